"""What a serving step does around its attention calls, and attention over a prefix that requests share.

Every case is one call, as a step of a serving instance makes it:

  maps     page maps of a step: blocks for the new tokens off the free list, block tables, cache slots, lengths and positions
  rope     queries and keys of one layer: norm of every head, rotation by positions with one or several axes, and K and V into
           the paged cache
  prefix   one layer's attention over the paged cache, of requests in groups that have the beginning of their context in common

Head counts, lengths and page sizes are those of synth_inputs.py: 16 heads of 80 with 256 to 4096 tokens per image (vision
encoder); 32 / 32 and 28 / 4 heads of 128 (language models), requests of an image part and a text part; cache blocks of 16
tokens.  Ragged lengths follow from the case alone (`shape`), values, page tables and slots from the seed.
"""
import math
import random

import torch

own = False

BLOCK = 16  # tokens per cache block
EPS = 1e-6  # of the norms

VIT = {"q_heads": 16, "kv_heads": 16, "head_dim": 80}
MHA = {"q_heads": 32, "kv_heads": 32, "head_dim": 128}
GQA = {"q_heads": 28, "kv_heads": 4, "head_dim": 128}
GQA64 = {"q_heads": 28, "kv_heads": 4, "head_dim": 64}


def listed():
    return [
        # decode step of a loaded instance: every request one token further, now and then into a new block
        dict(name="maps_decode", op="maps", kind="decode", requests=96, context_lo=128, context_hi=1800, short=False, shape=0),
        # the largest prefill: a thousand whole requests, whose blocks the step's scheduler has not quite got
        dict(name="maps_prefill", op="maps", kind="prefill", requests=1024, context_lo=0, context_hi=0, short=True, shape=0),
        # decode step of a few requests, heads normalised, K and V into the cache: latency
        dict(name="rope_decode_few", op="rope", kind="decode", **GQA, tokens=4, axes=3, norm=True, interleaved=False, shape=0),
        # the same for a loaded instance with one KV head per query head, one axis
        dict(name="rope_decode_mha", op="rope", kind="decode", **MHA, tokens=256, axes=1, norm=False, interleaved=False, shape=0),
        # prefill batch of requests with images, three axes, from one fused projection
        dict(name="rope_prefill", op="rope", kind="prefill", **GQA, tokens=30000, axes=3, norm=False, interleaved=False, shape=0),
        # vision encoder, rows and columns as axes, dynamic resolution, in place
        dict(name="rope_encode", op="rope", kind="encode", **VIT, tokens=65536, axes=2, norm=False, interleaved=False, shape=0),
        # two answers to one question about an image: latency
        dict(name="prefix_pair", op="prefix", **GQA, groups=1, requests=2, prefix=640, new_lo=1, new_hi=1, own_lo=20, own_hi=200, shape=0),
        # a loaded instance whose requests all begin with the same instructions and examples
        dict(name="prefix_decode", op="prefix", **GQA, groups=1, requests=48, prefix=4096, new_lo=1, new_hi=1, own_lo=32, own_hi=512, shape=0),
        # many users of one long document or video
        dict(name="prefix_decode_long", op="prefix", **GQA, groups=1, requests=128, prefix=16384, new_lo=1, new_hi=1, own_lo=16, own_hi=1024, shape=0),
        # several answers sampled for each of a dozen prompts
        dict(name="prefix_decode_groups", op="prefix", **GQA, groups=12, requests=96, prefix=1200, new_lo=1, new_hi=1, own_lo=16, own_hi=600, shape=0),
        # one KV head per query head: an image and its instructions, and questions about it being answered
        dict(name="prefix_decode_mha", op="prefix", **MHA, groups=2, requests=32, prefix=1024, new_lo=1, new_hi=1, own_lo=30, own_hi=400, shape=0),
        # the questions themselves, before the first answer's token
        dict(name="prefix_questions", op="prefix", **GQA, groups=1, requests=24, prefix=2304, new_lo=16, new_hi=150, own_lo=16, own_hi=150, shape=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["maps", "rope", "rope", "prefix", "prefix", "prefix"])
    shape = rng.randrange(1 << 20)
    if op == "maps":
        kind = rng.choice(["decode", "hybrid", "prefill"])
        hi = _log_int(rng, 100, 16384)
        return dict(op=op, kind=kind, requests=_log_int(rng, 1, 700 if kind == "prefill" else 2048), context_lo=0 if kind == "prefill" else max(1, hi // 10),
                    context_hi=0 if kind == "prefill" else hi, short=rng.random() < 0.25, shape=shape)
    if op == "rope":
        kind = rng.choice(["decode", "prefill", "encode"])
        heads = VIT if kind == "encode" else rng.choice([GQA, GQA, MHA, GQA64])
        most = 32768 if kind == "encode" else 1024 if kind == "decode" else 8192 if heads is MHA else 24000
        return dict(op=op, kind=kind, **heads, tokens=_log_int(rng, 1 if kind == "decode" else 200, most), axes=2 if kind == "encode" else rng.choice([1, 3]),
                    norm=rng.random() < 0.5, interleaved=kind != "encode" and rng.random() < 0.25, shape=shape)
    heads = rng.choice([GQA, GQA, MHA, GQA64])
    questions = rng.random() < 0.3
    groups = _log_int(rng, 1, 16)
    requests = max(groups, _log_int(rng, 2, 24 if questions else 48 if heads is MHA else 160))
    prefix = BLOCK * _log_int(rng, 4, max(5, min(1024, (128 if questions else 160 if heads is MHA else 1024) // groups)))
    new = _log_int(rng, 2, 100) if questions else 1
    own_hi = _log_int(rng, max(new, 16), 1024)
    return dict(op=op, **heads, groups=groups, requests=requests, prefix=prefix, new_lo=max(1, new // 4), new_hi=new, own_lo=max(new, own_hi // 20), own_hi=own_hi, shape=shape)


def _offsets(lengths):
    at, out = 0, [0]
    for n in lengths:
        at += n
        out.append(at)
    return out


# ---- maps ----------------------------------------------------------------------------------------------------


def _maps_lengths(case):
    """New tokens and tokens already cached of every request, and how many blocks the free list lacks."""
    rng = random.Random(case["shape"])
    new, context = [], []
    for b in range(case["requests"]):
        if case["kind"] == "prefill":
            new.append(_log_int(rng, 64, 1024) + rng.randint(32, 512))
            context.append(0)
        else:
            chunk = case["kind"] == "hybrid" and b % 25 == 7
            new.append(rng.randint(60, 512) if chunk else int(rng.random() < 0.95))  # (a slot whose request is done has none)
            context.append(_log_int(rng, max(1, case["context_lo"]), case["context_hi"]))
    if sum(new) == 0:
        new[0] = 1
    need = [-(-(c + n) // BLOCK) - -(-c // BLOCK) for n, c in zip(new, context)]
    return new, context, need, (sum(need) // 10 if case["short"] else 0)


def _maps_prepare(case, seed, dev, gen):
    new, context, need, lacking = _maps_lengths(case)
    batch, held = len(new), [-(-c // BLOCK) for c in context]
    free = max(sum(need) - lacking, 0) + (0 if lacking else 40)
    blocks = sum(held) + free + 8
    width = max(h + n for h, n in zip(held, need)) + 3
    ids = torch.randperm(blocks, generator=gen, device=dev).to(torch.int32)
    column = torch.arange(width, device=dev)
    starts = torch.tensor(_offsets(held)[:-1], device=dev)
    used = column[None, :] < torch.tensor(held, device=dev)[:, None]
    table = torch.where(used, ids[torch.where(used, starts[:, None] + column[None, :], 0)], -1).to(torch.int32).contiguous()
    list_ = torch.zeros(blocks, dtype=torch.int32, device=dev)  # (as long as the cache has blocks; the first `free` are on it)
    list_[:free] = ids[sum(held): sum(held) + free]
    total = sum(new)
    i32 = lambda *shape: torch.empty(shape, dtype=torch.int32, device=dev)  # noqa: E731
    # the step's token buffers are a little longer than its tokens, as those of a recorded graph are
    room = total + 5
    return {"case": case, "new": torch.tensor(new, dtype=torch.int32, device=dev), "context": torch.tensor(context, dtype=torch.int32, device=dev), "table": table,
            "free": list_, "n_free": torch.tensor([free], dtype=torch.int32, device=dev), "blocks": blocks, "room": room,
            "cu": i32(batch + 1), "kv": i32(batch), "slots": torch.empty(room, dtype=torch.int64, device=dev), "positions": i32(room), "next": i32(batch), "pool": i32(2)}


def _maps_run(s):
    if own:
        import paper_2505_12658_amd as hydra

        maps = hydra.PageMaps(s["cu"], s["kv"], s["slots"], s["positions"], s["next"], s["pool"])
        hydra.hydra_page_maps_build(s["new"], s["context"], s["table"], s["free"], s["n_free"], s["room"], BLOCK, s["blocks"], maps=maps)
        return s["cu"], s["kv"], s["slots"], s["positions"], s["next"], s["pool"], s["table"]
    new, context, table, room = s["new"].long(), s["context"].long(), s["table"], s["room"]
    batch, width = table.shape
    held = (context + BLOCK - 1) // BLOCK
    need = (context + new + BLOCK - 1) // BLOCK - held
    ends = torch.cumsum(need, 0)
    served = (need == 0) | (ends <= s["n_free"])  # in the order of the batch, until the list is used up
    zero = torch.zeros(1, dtype=torch.long, device=new.device)
    cu = torch.cat([zero, torch.cumsum(new, 0)])
    granted = torch.where(served, new, 0)
    kv = torch.where(served, context + new, 0)
    taken = torch.where(served, need, 0).sum()
    column = torch.arange(width, device=new.device)[None, :]
    fresh = (column >= held[:, None]) & (column < (held + need)[:, None]) & served[:, None]
    at = s["n_free"].long() - 1 - ((ends - need)[:, None] + column - held[:, None])
    torch.where(fresh, s["free"][at.clamp(0, s["free"].numel() - 1)], table, out=table)
    token = torch.arange(room, device=new.device)
    b = torch.searchsorted(cu[1:], token, right=True).clamp(max=batch - 1)
    real = token < cu[-1]
    position = context[b] + token - cu[b]
    block = table[b, (position // BLOCK).clamp(0, width - 1)].long()
    slots = torch.where(real & served[b], block * BLOCK + position % BLOCK, -1)
    pool = torch.stack([s["n_free"][0].long() - taken, (need.sum() - s["n_free"][0]).clamp(min=0)])
    i32 = torch.int32
    return cu.to(i32), kv.to(i32), slots, torch.where(real, position, 0).to(i32), (context + granted).to(i32), pool.to(i32), table


# ---- rope ----------------------------------------------------------------------------------------------------


def _frequencies(case, dev):
    """Angle per position of every pair of elements, and the axis whose position it takes."""
    half, axes = case["head_dim"] // 2, case["axes"]
    if case["kind"] == "encode":  # each axis has the frequencies of half a head
        per = half // 2
        f = 10000.0 ** -(torch.arange(per, dtype=torch.float64) / per)
        return torch.cat([f, f]).float().to(dev), torch.tensor([0] * per + [1] * per, dtype=torch.int32, device=dev)
    f = (1000000.0 if axes == 3 else 10000.0) ** -(torch.arange(half, dtype=torch.float64) / half)
    if axes == 1:
        return f.float().to(dev), None
    first = half // 4
    second = (half - first) // 2
    return f.float().to(dev), torch.tensor([0] * first + [1] * second + [2] * (half - first - second), dtype=torch.int32, device=dev)


def _rope_prepare(case, seed, dev, gen):
    n, hq, hkv, d = case["tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
    kind, axes = case["kind"], case["axes"]

    def normal(*shape, std=1.0):
        return (torch.randn(shape, generator=gen, device=dev) * std).to(torch.bfloat16)

    fused = normal(n, (hq + 2 * hkv) * d)  # one projection's output
    q, k, v = (t.view(n, -1, d) for t in fused.split([hq * d, hkv * d, hkv * d], dim=1))
    s = {"case": case, "q": q, "k": k, "v": v}
    s["inv_freq"], s["freq_axis"] = _frequencies(case, dev)
    if kind == "decode":  # one token of each request, at its own place
        p = torch.randint(1, 32768, (1, n), generator=gen, device=dev).expand(axes, n)
    elif kind == "prefill":  # requests of some 700 tokens, the first ones those of an image of 24 columns
        t = torch.arange(n, device=dev) % 700
        image = t < 480
        text = t - 480 + 24
        p = torch.stack([torch.where(image, 0, text), torch.where(image, t // 24, text), torch.where(image, t % 24, text)])
        p = p if axes == 3 else t[None, :]
    else:  # images of 52 columns
        t = torch.arange(n, device=dev) % 1976
        p = torch.stack([t // 52, t % 52])
    s["positions"] = p.to(torch.int32).contiguous()
    s["q_weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(torch.bfloat16) if case["norm"] else None
    s["k_weight"] = (1 + 0.1 * torch.randn(d, generator=gen, device=dev)).to(torch.bfloat16) if case["norm"] else None
    s["q_out"] = torch.empty((n, hq, d), dtype=torch.bfloat16, device=dev)
    if kind == "encode":
        s["k_out"] = torch.empty((n, hkv, d), dtype=torch.bfloat16, device=dev)
        return s
    blocks = -(-n // BLOCK) + 4
    s["slots"] = torch.randperm(blocks * BLOCK, generator=gen, device=dev)[:n].contiguous() if kind == "decode" else \
        (torch.randperm(blocks, generator=gen, device=dev)[:, None] * BLOCK + torch.arange(BLOCK, device=dev)).reshape(-1)[:n].contiguous()
    if n > 8:  # a padded token here and there
        s["slots"][torch.randperm(n, generator=gen, device=dev)[: n // 50 + 1]] = -1
    s["k_cache"], s["v_cache"] = normal(blocks, BLOCK, hkv, d), normal(blocks, BLOCK, hkv, d)
    return s


def _normed(x, weight):
    return x if weight is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * weight.float()


def _rotated(x, cos, sin, interleaved):
    half = x.shape[-1] // 2
    a, b = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :half], x[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)


def _rope_run(s):
    case = s["case"]
    cached = case["kind"] != "encode"
    if own:
        import paper_2505_12658_amd as hydra

        more = dict(v=s["v"], k_cache=s["k_cache"], v_cache=s["v_cache"], slot_mapping=s["slots"]) if cached else dict(k_out=s["k_out"])
        hydra.hydra_qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], freq_axis=s["freq_axis"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                                 eps=EPS, interleaved=case["interleaved"], q_out=s["q_out"], **more)
        return (s["q_out"], s["k_cache"], s["v_cache"]) if cached else (s["q_out"], s["k_out"])
    p = s["positions"]
    p = p[0][:, None] if s["freq_axis"] is None else p[s["freq_axis"].long()].T
    angle = p.double() * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    q = _rotated(_normed(s["q"].float(), s["q_weight"]), cos, sin, case["interleaved"]).to(torch.bfloat16)
    k = _rotated(_normed(s["k"].float(), s["k_weight"]), cos, sin, case["interleaved"]).to(torch.bfloat16)
    if not cached:
        return q, k
    keep = s["slots"] >= 0
    slots = s["slots"][keep]
    s["k_cache"].view(-1, *k.shape[1:])[slots] = k[keep]
    s["v_cache"].view(-1, *k.shape[1:])[slots] = s["v"][keep]
    return q, s["k_cache"], s["v_cache"]


def _rope_exact(case, seed):
    s = prepare(case, seed)
    n = case["tokens"]
    half = case["head_dim"] // 2
    f = s["inv_freq"].double()
    turn = torch.zeros((n, half), dtype=torch.complex128, device=f.device)
    for i in range(half):
        axis = 0 if s["freq_axis"] is None else int(s["freq_axis"][i])
        turn[:, i] = torch.exp(1j * (s["positions"][axis].double() * f[i]))

    def turned(x, weight):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
        pairs = x.reshape(*x.shape[:-1], half, 2) if case["interleaved"] else x.reshape(*x.shape[:-1], 2, half).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None, :])
        return (z if case["interleaved"] else z.transpose(-1, -2)).reshape(x.shape)

    q, k = turned(s["q"], s["q_weight"]), turned(s["k"], s["k_weight"])
    if case["kind"] == "encode":
        return q, k
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    keep = torch.nonzero(s["slots"] >= 0)[:, 0]
    at = s["slots"][keep]
    kc[at // BLOCK, at % BLOCK] = k[keep]
    vc[at // BLOCK, at % BLOCK] = s["v"].double()[keep]
    return q, kc, vc


# ---- prefix --------------------------------------------------------------------------------------------------


def _prefix_lengths(case):
    """Requests of each group, its common prefix, and every request's new tokens and tokens of its own (new ones included)."""
    rng = random.Random(case["shape"])
    groups, requests = case["groups"], case["requests"]
    cuts = sorted(rng.sample(range(1, requests), groups - 1))
    sizes = [b - a for a, b in zip([0] + cuts, cuts + [requests])]
    prefixes = [case["prefix"] if groups == 1 else BLOCK * max(1, round(case["prefix"] * rng.uniform(0.5, 1.5) / BLOCK)) for _ in sizes]
    new = [_log_int(rng, case["new_lo"], case["new_hi"]) for _ in range(requests)]
    mine = [max(n, _log_int(rng, case["own_lo"], case["own_hi"])) for n in new]
    return sizes, prefixes, new, mine


def _prefix_prepare(case, seed, dev, gen):
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    sizes, prefixes, new, mine = _prefix_lengths(case)
    group_of = [g for g, n in enumerate(sizes) for _ in range(n)]
    shared_blocks, own_blocks = [p // BLOCK for p in prefixes], [-(-m // BLOCK) for m in mine]
    blocks = sum(shared_blocks) + sum(own_blocks) + 8
    ids = torch.randperm(blocks, generator=gen, device=dev).to(torch.int32)
    width = max(shared_blocks[g] + o for g, o in zip(group_of, own_blocks))
    column = torch.arange(width, device=dev)[None, :]
    in_prefix = torch.tensor([shared_blocks[g] for g in group_of], device=dev)[:, None]
    first_shared = torch.tensor([_offsets(shared_blocks)[g] for g in group_of], device=dev)[:, None]
    first_own = sum(shared_blocks) + torch.tensor(_offsets(own_blocks)[:-1], device=dev)[:, None]
    used = column < in_prefix + torch.tensor(own_blocks, device=dev)[:, None]
    at = torch.where(column < in_prefix, first_shared + column, first_own + column - in_prefix)
    table = torch.where(used, ids[torch.where(used, at, 0)], -1).to(torch.int32).contiguous()

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev).to(torch.bfloat16)

    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    n = sum(new)
    return {"case": case, "q": normal(n, hq, d), "k_cache": normal(blocks, BLOCK, hkv, d), "v_cache": normal(blocks, BLOCK, hkv, d), "table": table,
            "cu": i32(_offsets(new)), "kv": i32([prefixes[g] + m for g, m in zip(group_of, mine)]), "groups": i32(_offsets(sizes)), "shared": i32(prefixes),
            "scale": 1.0 / math.sqrt(d), "out": torch.empty((n, hq, d), dtype=torch.bfloat16, device=dev), "workspace": None,
            # (sizes that the scheduler knows on the host)
            "most_new": max(new), "most_tokens": max(sum(new[a:b]) for a, b in zip(_offsets(sizes)[:-1], _offsets(sizes)[1:])), "most_prefix": max(prefixes),
            "most_own": max(mine)}


def _partial(q, keys, values, visible, scale):
    """Maximum, sum and unnormalised output of q [.., rows, d] over keys [.., n, d]; visible broadcasts to [.., rows, n]."""
    z = torch.matmul(q, keys.transpose(-1, -2).contiguous()) * scale
    z = torch.where(visible, z, -math.inf)
    top = z.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(z - top)
    return top, p.sum(-1, keepdim=True), torch.matmul(p, values)


def _prefix_run(s):
    if own:
        import paper_2505_12658_amd as hydra

        n, hq, d = s["q"].shape
        if s["workspace"] is None:  # kept by the program, like the output buffer
            need = hydra.hydra_attn_prefix_workspace_bytes(s["kv"].numel(), s["shared"].numel(), n, hq, s["case"]["kv_heads"], d)
            s["workspace"] = torch.empty(need, dtype=torch.uint8, device=s["q"].device)
        return hydra.hydra_attn_prefix_fwd(s["q"], s["k_cache"], s["v_cache"], s["table"], s["cu"], s["kv"], s["groups"], s["shared"], s["scale"],
                                           out=s["out"], workspace=s["workspace"])
    q, dev = s["q"], s["q"].device
    n, hq, d = q.shape
    hkv = s["case"]["kv_heads"]
    share = hq // hkv
    k_rows, v_rows = s["k_cache"].view(-1, hkv, d), s["v_cache"].view(-1, hkv, d)
    cu, kv, cu_groups, shared = s["cu"].long(), s["kv"].long(), s["groups"].long(), s["shared"].long()
    new = cu[1:] - cu[:-1]
    token = torch.arange(n, device=dev)
    request = torch.searchsorted(cu[1:], token, right=True)
    group = torch.searchsorted(cu_groups[1:], request, right=True)

    def rows(keys, table):  # rows of the cache that hold these keys; [.., keys]
        return torch.gather(table, -1, (keys // BLOCK).clamp(max=table.shape[-1] - 1)).long().clamp(min=0) * BLOCK + keys % BLOCK

    def heads_first(x):  # [a, b, heads, d] -> [a, heads, b, d] in 32 bits
        return x.float().transpose(1, 2).contiguous()

    def packed(which, count, place, places):  # the tokens' queries by `which` and place, and where they went; [count, hkv, places * share, d]
        full = torch.zeros((count, places, hkv, share, d), device=dev)
        full[which, place] = q.float().view(n, hkv, share, d)
        return full.permute(0, 2, 1, 3, 4).reshape(count, hkv, places * share, d)

    def unpacked(x, which, place, places):  # and back: [n, hkv, share, ..]
        return x.reshape(x.shape[0], hkv, places, share, -1).permute(0, 2, 1, 3, 4)[which, place]

    # the common prefixes, all of a group's tokens against them
    first = cu[cu_groups[:-1]]
    key = torch.arange(s["most_prefix"], device=dev)[None, :].expand(shared.numel(), -1)
    at = rows(key, s["table"][cu_groups[:-1]])
    place = token - first[group]
    a = _partial(packed(group, shared.numel(), place, s["most_tokens"]), heads_first(k_rows[at]), heads_first(v_rows[at]),
                 (key < shared[:, None])[:, None, None, :], s["scale"])
    m1, l1, o1 = (unpacked(x, group, place, s["most_tokens"]) for x in a)
    # what each request has of its own
    begin = shared[torch.searchsorted(cu_groups[1:], torch.arange(kv.numel(), device=dev), right=True)]
    key = begin[:, None] + torch.arange(s["most_own"], device=dev)[None, :]
    at = rows(key, s["table"])
    place = token - cu[request]
    last = (kv - new)[:, None] + torch.arange(s["most_new"], device=dev)[None, :]  # of a token's visible keys
    seen = (key[:, None, :] <= last[:, :, None]) & (key < kv[:, None])[:, None, :]
    a = _partial(packed(request, kv.numel(), place, s["most_new"]), heads_first(k_rows[at]), heads_first(v_rows[at]),
                 seen.repeat_interleave(share, 1)[:, None], s["scale"])
    m2, l2, o2 = (unpacked(x, request, place, s["most_new"]) for x in a)
    top = torch.maximum(m1, m2)
    w1, w2 = torch.exp(m1 - top), torch.exp(m2 - top)
    return ((w1 * o1 + w2 * o2) / (w1 * l1 + w2 * l2)).reshape(n, hq, d).to(torch.bfloat16)


def _prefix_exact(case, seed):
    s = prepare(case, seed)
    n, hq, d = s["q"].shape
    hkv = case["kv_heads"]
    out = torch.empty((n, hq, d), dtype=torch.float64, device=s["q"].device)
    cu, kv = s["cu"].tolist(), s["kv"].tolist()
    for b, length in enumerate(kv):
        pages = s["table"][b, : -(-length // BLOCK)].long()
        keys = s["k_cache"][pages].reshape(-1, hkv, d)[:length].double()
        values = s["v_cache"][pages].reshape(-1, hkv, d)[:length].double()
        count = cu[b + 1] - cu[b]
        hidden = torch.arange(length, device=keys.device)[None, :] > torch.arange(length - count, length, device=keys.device)[:, None]
        for h in range(hq):
            z = s["q"][cu[b]: cu[b + 1], h].double() @ keys[:, h * hkv // hq].T.contiguous() * s["scale"]
            z = z.masked_fill(hidden, -math.inf)
            out[cu[b]: cu[b + 1], h] = torch.softmax(z, -1) @ values[:, h * hkv // hq].contiguous()
    return out


# ---- what the measurement calls ------------------------------------------------------------------------------


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    return {"maps": _maps_prepare, "rope": _rope_prepare, "prefix": _prefix_prepare}[case["op"]](case, seed, dev, gen)


def run(s):
    return {"maps": _maps_run, "rope": _rope_run, "prefix": _prefix_run}[s["case"]["op"]](s)


def work(case):
    if case["op"] == "maps":  # lengths read, lengths and offsets written, blocks off the list into the table, a slot and a position per token
        new, context, need, lacking = _maps_lengths(case)
        return {"bytes": len(new) * (8 + 12) + (sum(need) - lacking) * 8 + sum(new) * 12 + 20, "flops": 0}
    if case["op"] == "rope":
        n, d = case["tokens"], case["head_dim"]
        q, k = n * case["q_heads"] * d, n * case["kv_heads"] * d
        cached = case["kind"] != "encode"
        moved = 2 * (q + k) * 2 + n * 4 * case["axes"] + (2 * k * 2 + n * 8 if cached else 0)
        return {"bytes": moved, "flops": (q + k) * (7 if case["norm"] else 3)}
    sizes, prefixes, new, mine = _prefix_lengths(case)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    group_of = [g for g, n in enumerate(sizes) for _ in range(n)]
    pairs = sum(n * (prefixes[g] + m - n) + n * (n + 1) // 2 for g, n, m in zip(group_of, new, mine))
    return {"bytes": (2 * sum(new) * hq + 2 * (sum(prefixes) + sum(mine)) * hkv) * d * 2, "flops": 4 * d * hq * pairs}


def exact(case, seed):
    if case["op"] == "maps":  # whole numbers
        return None
    return _rope_exact(case, seed) if case["op"] == "rope" else _prefix_exact(case, seed)
