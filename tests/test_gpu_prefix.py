"""Attention over the paged cache of requests that share prefixes, against the 64-bit oracle of the paged call."""
import numpy as np
import pytest
import torch

import synth_inputs as si
from oracle import reference

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HALF_STEP = torch.finfo(torch.bfloat16).eps / 2


def _f64(t):
    return reference.bf16_bits_to_f64(si.bf16_bits(t))


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


class Batch:
    """Groups of requests: sizes[g] requests behind prefixes[g] tokens whose blocks they share; mine[b] tokens of its own for each, q_lens[b]
    of them new.  Every cache row holds a random value, and entries past a request's last block are -1."""

    def __init__(self, sizes, prefixes, q_lens, mine, hq, hkv, d, block=16, seed=0):
        self.sizes, self.prefixes, self.q_lens, self.hq, self.hkv, self.d, self.block = sizes, prefixes, list(q_lens), hq, hkv, d, block
        rng = np.random.default_rng(seed)
        group_of = [g for g, n in enumerate(sizes) for _ in range(n)]
        self.kv_lens = [prefixes[g] + m for g, m in zip(group_of, mine)]
        need = [-(-k // block) for k in self.kv_lens]
        shared = [p // block for p in prefixes]  # (whole blocks are shared; the rest of a prefix is written per request, with equal values)
        total = sum(shared) + sum(n - shared[g] for g, n in zip(group_of, need)) + 3
        ids = rng.permutation(total).tolist()
        blocks_of = [[ids.pop() for _ in range(s)] for s in shared]
        self.tables = np.full((len(group_of), max(need + [1]) + 1), -1, np.int32)
        g_ = torch.Generator().manual_seed(seed)
        draw = lambda *shape: torch.randn(shape, generator=g_).to(torch.bfloat16)  # noqa: E731
        self.k_cache, self.v_cache = draw(total, block, hkv, d), draw(total, block, hkv, d)
        leaders = {}
        for b, g in enumerate(group_of):
            row = blocks_of[g] + [ids.pop() for _ in range(need[b] - shared[g])]
            self.tables[b, :need[b]] = row
            rest = prefixes[g] - shared[g] * block
            if rest and need[b] > shared[g]:
                if g in leaders:
                    for c in (self.k_cache, self.v_cache):
                        c[row[shared[g]], :rest] = c[leaders[g], :rest]
                else:
                    leaders[g] = row[shared[g]]
        self.q = draw(sum(q_lens), hq, d)
        self.cu = np.concatenate([[0], np.cumsum(q_lens)])
        self.cu_groups = np.concatenate([[0], np.cumsum(sizes)])
        self.scale = d ** -0.5

    def on_gpu(self, shared=None):
        return (self.q.to(DEV), self.k_cache.to(DEV), self.v_cache.to(DEV), _i32(self.tables), _i32(self.cu), _i32(self.kv_lens), _i32(self.cu_groups),
                _i32(self.prefixes if shared is None else shared), self.scale)

    def want(self, values=None, q=None):
        """(zeros for requests without output, which the oracle refuses)"""
        q, keys, values = _f64(self.q if q is None else q), _f64(self.k_cache), _f64(self.v_cache) if values is None else values
        out = np.zeros(q.shape)
        for b, (n, k) in enumerate(zip(self.q_lens, self.kv_lens)):
            if k >= n > 0:
                at = slice(self.cu[b], self.cu[b + 1])
                out[at] = reference.attn_paged(q[at], keys, values, self.tables[b: b + 1], [0, n], [k], self.scale)
        return out

    def check(self, out, q=None):
        """Probabilities are rounded to bf16 before the second product and the output once more, each by half a step at most:
        half a step of sum_j p_j |v_j|, and of the result; exponents of scores of a few units in fp32 and the sums add some 1e-6 of it."""
        want, size = self.want(q=q), self.want(np.abs(_f64(self.v_cache)), q)
        got = _f64(out)
        has = np.zeros(len(got), bool)
        for b, (n, k) in enumerate(zip(self.q_lens, self.kv_lens)):
            has[self.cu[b]: self.cu[b + 1]] = n > 0 and k >= n
        off, allowed = np.abs(got - want)[has], (HALF_STEP * (size + np.abs(want)) + 1e-4 * size)[has]
        assert np.isfinite(got[has]).all() and (off <= allowed).all(), f"off by {(off / allowed).max():.3f} of what is allowed"


def _call(planned, q, kc, vc, table, cu, kv, groups, shared, scale, out=None, workspace=None):
    """The whole call, which leaves small batches and long chunks to the paged kernels, or its two halves, which never do."""
    import paper_2505_12658_amd as hydra

    if not planned:
        return hydra.hydra_attn_prefix_fwd(q, kc, vc, table, cu, kv, groups, shared, scale, out=out, workspace=workspace)
    ws = hydra.hydra_attn_prefix_plan(cu, kv, groups, shared, q.shape[0], q.shape[1], kc.shape[2], q.shape[2], table.shape[1], kc.shape[1], workspace=workspace)
    return hydra.hydra_attn_prefix_fwd_planned(q, kc, vc, table, shared.numel(), scale, ws, out=out)


def _run(batch, planned, shared=None, **kw):
    out = _call(planned, *batch.on_gpu(shared), **kw)
    torch.cuda.synchronize()
    return out


both = pytest.mark.parametrize("planned", [True, False], ids=["planned", "whole"])


CASES = [
    # sizes, prefixes, q_lens, own tokens, Hq, Hkv, d, block
    ([1], [0], [1], [1], 1, 1, 64, 16),
    ([2], [64], [1, 1], [1, 2], 7, 1, 128, 16),
    ([2], [640], [1, 1], [20, 200], 28, 4, 128, 16),
    ([3, 1, 2], [130, 500, 64], [1, 1, 1, 1, 1, 1], [5, 70, 33, 9, 1, 400], 28, 4, 128, 16),
    ([5], [1000], [1] * 5, [1, 1, 2, 17, 129], 32, 32, 128, 16),
    ([9, 7], [333, 2048], [1] * 16, list(range(1, 17)), 4, 2, 64, 4),
    ([40], [700], [1] * 40, [3 + 7 * i for i in range(40)], 28, 4, 128, 16),
    ([40], [700], [1] * 40, [3 + 7 * i for i in range(40)], 28, 4, 64, 32),
    ([12], [256], [1 + (i * 5) % 9 for i in range(12)], [20 + i for i in range(12)], 8, 2, 80, 16),
    ([3], [400], [1, 17, 130], [60, 17, 200], 16, 16, 80, 8),
    ([4, 2], [100, 900], [33, 1, 64, 5, 200, 1], [40, 9, 64, 77, 200, 3], 7, 1, 128, 1),
    ([6], [1500], [50, 33, 80, 61, 20, 45], [50, 40, 80, 300, 20, 45], 28, 4, 128, 16),
    ([3], [300], [2, 1, 3], [9, 1, 5], 64, 1, 64, 256),
    ([2], [640], [1, 1], [3, 3], 48, 1, 128, 16),
    ([130], [128], [1] * 130, [1 + i % 50 for i in range(130)], 2, 1, 128, 16),
    ([2, 2], [64, 20000], [1, 1, 1, 1], [30, 40, 3000, 50], 7, 1, 128, 16),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0][0]}of{len(c[2])}-p{max(c[1])}-q{max(c[2])}-h{c[4]}k{c[5]}-d{c[6]}-b{c[7]}")
@both
def test_shared_prefixes(case, planned):
    batch = Batch(*case, seed=len(case[2]))
    batch.check(_run(batch, planned))


@pytest.mark.parametrize("seed", range(24))
@both
def test_random_groups(seed, planned):
    """Random groups (empty ones, groups of one), requests without new tokens or with more new tokens than context, claims of fewer and of more shared keys
    than the tokens can see, any head grouping, head_dim and block size; workspaces full of NaN."""
    import paper_2505_12658_amd as hydra

    rng = np.random.default_rng(500 + seed)
    hq, hkv = [(1, 1), (4, 1), (4, 2), (7, 1), (8, 8), (28, 4)][int(rng.integers(6))]
    sizes = rng.integers(0, 9, int(rng.integers(1, 6))).tolist() + [2]
    n = sum(sizes)
    prefixes = [int(rng.integers(0, 600)) for _ in sizes]
    q_lens = [int(rng.choice([0, 1, 1, 1, rng.integers(2, 6), rng.integers(6, 70)])) for _ in range(n)]
    if sum(q_lens) == 0:
        q_lens[0] = 1
    mine = [max(q, int(rng.integers(1, 200))) for q in q_lens]
    batch = Batch(sizes, prefixes, q_lens, mine, hq, hkv, [64, 80, 128][int(rng.integers(3))], [1, 4, 16, 64][int(rng.integers(4))], seed)
    if n > 3:
        batch.kv_lens[int(rng.integers(n))] = 0  # (a request without room in the cache)
    claims = [int(p + rng.choice([0, 0, -1, -64, -p])) for p in prefixes]
    group_of = np.repeat(np.arange(len(sizes)), sizes)
    for g in range(len(sizes)):  # more than can be seen by a group that has one request with new tokens: nothing else says so
        if sum(q_lens[b] > 0 for b in np.flatnonzero(group_of == g)) == 1:
            claims[g] += 1000
    need = hydra.hydra_attn_prefix_workspace_bytes(n, len(sizes), sum(q_lens), hq, hkv, batch.d)
    workspace = torch.full((need // 4 + 1,), float("nan"), device=DEV).view(torch.uint8)
    out = torch.full((sum(q_lens), hq, batch.d), 5.0, dtype=torch.bfloat16, device=DEV)
    batch.check(_run(batch, planned, claims, out=out, workspace=workspace))
    for b, (q, k) in enumerate(zip(q_lens, batch.kv_lens)):
        if k < q:
            assert (out[batch.cu[b]: batch.cu[b + 1]] == 5.0).all()


@both
def test_a_claim_beyond_what_the_shortest_request_sees(planned):
    """The last new token of a chunk sees all of the shared keys, its first one does not: fewer are taken as shared."""
    batch = Batch([4], [512], [1, 1, 1, 1], [70, 9, 30, 1], 7, 1, 128)
    batch.q_lens[3], batch.kv_lens[3] = 40, 500
    batch.cu = np.concatenate([[0], np.cumsum(batch.q_lens)])
    batch.q = torch.randn((43, 7, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    batch.check(_run(batch, planned))


@both
def test_strided_queries_and_results_bit_for_bit(planned):
    batch = Batch([6, 5], [500, 900], [1, 2, 1, 1, 3, 1, 1, 1, 1, 1, 1], [9, 80, 1, 30, 3, 500, 7, 7, 100, 1, 2], 14, 2, 128, seed=4)
    args = list(batch.on_gpu())
    first = _call(planned, *args)
    wide = torch.randn((batch.q.shape[0], 14 * 128 + 40), device=DEV).to(torch.bfloat16)
    view = wide[:, 16: 16 + 14 * 128].view(-1, 14, 128)
    view.copy_(args[0])
    args[0] = view
    for _ in range(3):
        again = _call(planned, *args)
        assert torch.equal(first.view(torch.int16), again.view(torch.int16))
    batch.check(first)


def test_large_batches_are_planned_by_the_whole_call():
    """Contexts beyond what is sooner read one by one: the whole call gives the halves' bits."""
    batch = Batch([12], [2048], [1] * 12, [9 + 5 * i for i in range(12)], 32, 32, 128, seed=5)
    whole, planned = _run(batch, False), _run(batch, True)
    batch.check(whole)
    assert torch.equal(whole.view(torch.int16), planned.view(torch.int16))


def test_one_plan_for_several_layers():
    import paper_2505_12658_amd as hydra

    layers = [Batch([7, 3], [640, 200], [1] * 9 + [20], [5, 80, 1, 30, 3, 500, 7, 9, 100, 41], 28, 4, 128, seed=9) for _ in range(2)]
    layers[1].q = torch.randn(layers[1].q.shape, generator=torch.Generator().manual_seed(77)).to(torch.bfloat16)
    layers[1].v_cache = layers[1].v_cache.roll(1, 3)
    q, kc, vc, table, cu, kv, groups, shared, scale = layers[0].on_gpu()
    ws = hydra.hydra_attn_prefix_plan(cu, kv, groups, shared, q.shape[0], 28, 4, 128, table.shape[1], 16)
    for layer in layers:
        q, kc, vc, table, *_ = layer.on_gpu()
        planned = hydra.hydra_attn_prefix_fwd_planned(q, kc, vc, table, 2, scale, ws)
        layer.check(planned)


@both
def test_recorded_step_with_growing_contexts(planned):
    """Planned and run inside a graph: replays act on the lengths, groups and queries that the buffers hold by then."""
    import paper_2505_12658_amd as hydra

    batch = Batch([5, 4], [320, 130], [1] * 9, [40] * 9, 28, 4, 128, seed=2)
    q, kc, vc, table, cu, kv, groups, shared, scale = batch.on_gpu()
    out = torch.zeros_like(q)
    ws = torch.empty(hydra.hydra_attn_prefix_workspace_bytes(9, 2, 9, 28, 4, 128), dtype=torch.uint8, device=DEV)

    def step():
        _call(planned, q, kc, vc, table, cu, kv, groups, shared, scale, out=out, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, lengths in enumerate([[320 + 1] * 5 + [130 + 7] * 4, [320 + 3 * j for j in range(1, 6)] + [130 + 9 * j for j in range(1, 5)], [0, 322, 345, 0, 360] + [0, 131, 0, 170]]):
        kv.copy_(_i32(lengths))
        shared.copy_(_i32([320, 130] if i != 1 else [0, 128]))
        fresh = torch.randn(q.shape, generator=torch.Generator().manual_seed(i)).to(torch.bfloat16)
        q.copy_(fresh.to(DEV))
        out.fill_(3.0)
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.fill_(3.0)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.int16), out.view(torch.int16))
        batch.kv_lens = lengths
        batch.check(got, q=fresh)
        assert all((got[b] == 3.0).all() for b in range(9) if lengths[b] == 0)


@pytest.mark.parametrize("requests, block", [(3, 16), (14, 16), (40, 16), (14, 4), (30, 2)])
@pytest.mark.parametrize("d", [64, 128])
@both
def test_large_scores_and_equal_keys(requests, block, d, planned):
    """Scores that lead the first keys' by far more than a fixed reference allows, in the prefix and behind it; rows whose keys are all the same."""
    batch = Batch([requests, 2], [576, 256], [1] * (requests + 2), [100, 40, 7] + [90] * (requests - 3) + [64, 1], 7, 1, d, block, seed=6)
    for b, j in ((0, 100), (0, 470), (1, 600), (requests, 30), (requests, 300)):
        at = (batch.tables[b, j // block], j % block)
        batch.k_cache[at] = batch.k_cache[at] * 60
    batch.q[2] = 0
    batch.check(_run(batch, planned))


@pytest.mark.parametrize("d", [64, 128])
@both
def test_large_scores_in_chunks(d, planned):
    """The same for requests of many rows: whole contexts in one piece, and contexts cut in parts."""
    batch = Batch([1, 1, 1], [0, 0, 0], [40, 70, 33], [900, 70, 1500], 7, 1, d, seed=8)
    for b, j in ((0, 500), (1, 40), (2, 64), (2, 1400)):
        at = (batch.tables[b, j // 16], j % 16)
        batch.k_cache[at] = batch.k_cache[at] * 60
    batch.check(_run(batch, planned))


@pytest.mark.parametrize("prefix, own, requests, q_len", [(2048, 3000, 300, 1), (0, 40000, 300, 1), (512, 9000, 500, 2), (1024, 3000, 60, 33)],
                         ids=["behind-a-prefix", "long", "pairs", "chunks"])
@both
def test_workspaces_hold_the_plans_of_many_long_contexts(prefix, own, requests, q_len, planned):
    """Many requests with long contexts of their own, which could be cut into more pieces than the chip has places for.  Eight requests over and over, so
    that eight tell what all of them give."""
    kinds, d, block = 8, 64, 16
    few = Batch([kinds], [prefix], [q_len] * kinds, [own - 150 * i for i in range(kinds)], 1, 1, d, block, seed=3)
    many = np.arange(requests) % kinds
    rows = (many[:, None] * q_len + np.arange(q_len)).ravel()
    args = list(few.on_gpu())
    args[0] = args[0][torch.from_numpy(rows).to(DEV)].contiguous()
    args[3], args[5] = args[3][torch.from_numpy(many).to(DEV)].contiguous(), _i32(np.asarray(few.kv_lens)[many])
    args[4], args[6] = _i32(np.arange(requests + 1) * q_len), _i32([0, requests])
    out = torch.full_like(args[0], float("nan"))
    _call(planned, *args, out=out)
    torch.cuda.synchronize()
    n = kinds * q_len
    results = few.want(), few.want(np.abs(_f64(few.v_cache)))
    few.want = lambda values=None, q=None: results[values is not None]
    for first in range(0, len(out), n):  # (rows of the last, broken-off turn are compared with the first turn's)
        here = out[first: first + n]
        few.check(torch.cat([here, out[len(here): n]]))


@both
def test_all_keys_shared(planned):
    """Several answers about to begin: contexts that are equal to the last key, which is the new token's own."""
    batch = Batch([20, 2], [640, 128], [1] * 22, [1] * 22, 14, 2, 128, seed=12)
    batch.kv_lens = [640] * 20 + [128] * 2
    batch.check(_run(batch, planned))


@pytest.mark.parametrize("sizes", [[2048], [1] * 2048, [0] * 1000 + [1024, 0, 1024] + [0] * 1045], ids=["one", "alone", "two"])
@both
def test_as_many_requests_and_groups_as_there_may_be(sizes, planned):
    batch = Batch(sizes, [256] * len(sizes) if len(sizes) < 2048 or 0 in sizes else [3] * len(sizes), [1] * 2048, [1 + i % 37 for i in range(2048)], 2, 1, 64, seed=13)
    batch.check(_run(batch, planned))


@both
def test_rows_behind_the_last_request_stay(planned):
    batch = Batch([6], [512], [1, 2, 1, 0, 3, 1], [9, 2, 30, 1, 3, 70], 7, 1, 128, seed=14)
    args = list(batch.on_gpu())
    args[0] = torch.cat([args[0], torch.full((5, 7, 128), float("nan"), dtype=torch.bfloat16, device=DEV)])
    out = torch.full_like(args[0], 3.0)
    _call(planned, *args, out=out)
    torch.cuda.synchronize()
    batch.check(out[:8])
    assert (out[8:] == 3.0).all()


@pytest.mark.parametrize("name, values", [("cu", [0, 1, 9, 2, 3]), ("cu", [-1, 1, 2, 3, 4]), ("cu", [0, 1, 2, 3, 5]), ("groups", [0, 3, 2, 4]), ("groups", [0, 1, 3, 3]),
                                          ("groups", [1, 2, 3, 4]), ("groups", [0, 2, 5, 4]), ("groups", [0, 2, 3, 5])])
def test_plans_of_offsets_that_are_none(name, values):
    """Offsets that decrease, or leave the batch: a plan without pieces."""
    batch = Batch([1, 2, 1], [640, 640, 70], [1] * 4, [9, 2, 30, 1], 7, 1, 128, seed=15)
    args = list(batch.on_gpu())
    args[4 if name == "cu" else 6] = _i32(values)
    out = torch.full_like(args[0], 3.0)
    _call(True, *args, out=out)
    torch.cuda.synchronize()
    assert (out == 3.0).all()


@both
def test_a_stream_of_its_own(planned):
    """On a side stream that is given as an argument, with outputs and workspaces that the calls allocate, while the current stream fills memory that it frees."""
    import paper_2505_12658_amd as hydra

    batch = Batch([12], [2048], [1] * 12, [9 + 5 * i for i in range(12)], 32, 32, 128, seed=5)
    args = batch.on_gpu()
    q, kc, vc, table, cu, kv, groups, shared, scale = args
    need = hydra.hydra_attn_prefix_workspace_bytes(12, 1, 12, 32, 32, 128)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        torch.empty(need, dtype=torch.uint8, device=DEV).fill_(255)
    if planned:
        ws = hydra.hydra_attn_prefix_plan(cu, kv, groups, shared, 12, 32, 32, 128, table.shape[1], 16, stream=side)
        out = hydra.hydra_attn_prefix_fwd_planned(q, kc, vc, table, 1, scale, ws, stream=side)
    else:
        out = hydra.hydra_attn_prefix_fwd(*args, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    batch.check(out)
    with pytest.raises((TypeError, ValueError, AttributeError)):
        hydra.hydra_attn_prefix_fwd(*args, stream=3)


FORMS = [([20, 3], [700, 130], [1 + 4 * (i % 2) for i in range(23)], [5 + 9 * i for i in range(23)], 32, 8, 128, 16),
         ([9], [500], [1, 2, 9, 1, 1, 30, 1, 1, 70], [70, 3, 90, 1, 65, 31, 2, 200, 71], 14, 2, 128, 2),
         ([20], [333], [1 + 4 * (i % 2) for i in range(20)], [5 + 9 * i for i in range(20)], 8, 2, 64, 64),
         ([6], [200], [1, 7, 1, 40, 1, 1], [5, 60, 1, 40, 129, 64], 4, 2, 80, 16)]


@pytest.mark.parametrize("case", FORMS, ids=lambda c: f"h{c[4]}k{c[5]}-d{c[6]}-b{c[7]}")
@both
def test_nothing_behind_the_contexts_is_used(case, planned):
    """NaN in every row of the cache that is in no context: behind the last key in its block, and in blocks that nobody has."""
    batch = Batch(*case, seed=16)
    in_context = torch.zeros(batch.k_cache.shape[:2], dtype=torch.bool)
    for row, n in zip(batch.tables, batch.kv_lens):
        in_context[row[np.arange(n) // batch.block], np.arange(n) % batch.block] = True
    want = batch.want(), batch.want(np.abs(_f64(batch.v_cache)))
    batch.want = lambda values=None, q=None: want[values is not None]
    for c in (batch.k_cache, batch.v_cache):
        c[~in_context] = float("nan")
    batch.check(_run(batch, planned))


@pytest.mark.parametrize("case", FORMS[:1], ids=lambda c: f"h{c[4]}k{c[5]}-d{c[6]}-b{c[7]}")
@both
def test_blocks_behind_the_first_four_gigabytes(case, planned):
    batch = Batch(*case, seed=17)
    blocks, block, hkv, d = batch.k_cache.shape
    apart = (5 << 30) // (block * hkv * d * 2) // blocks
    far = torch.arange(blocks, device=DEV) * apart + apart - 1
    args = list(batch.on_gpu())
    for i in (1, 2):
        wide = torch.zeros((blocks * apart, block, hkv, d), dtype=torch.bfloat16, device=DEV)
        wide[far] = args[i]
        args[i] = wide
    args[3] = torch.where(args[3] < 0, args[3], args[3] * apart + apart - 1)
    out = _call(planned, *args)
    torch.cuda.synchronize()
    batch.check(out)


@pytest.mark.parametrize("case", FORMS, ids=lambda c: f"h{c[4]}k{c[5]}-d{c[6]}-b{c[7]}")
@both
def test_a_scale_of_zero_takes_the_mean(case, planned):
    batch = Batch(*case, seed=18)
    batch.scale = 0.0
    batch.check(_run(batch, planned))


@pytest.mark.parametrize("case", FORMS, ids=lambda c: f"h{c[4]}k{c[5]}-d{c[6]}-b{c[7]}")
@both
def test_pages_outside_the_cache_harm_only_their_request(case, planned):
    """Entries of one request's own blocks that no cache has: wrong numbers for it, and the others as they are without it."""
    batch = Batch(*case, seed=19)
    bad = 4
    first = batch.prefixes[0] // batch.block
    args = list(batch.on_gpu())
    table = batch.tables.copy()
    table[bad, first: -(-batch.kv_lens[bad] // batch.block)] = [-7, 2 ** 31 - 1, 10 ** 6][bad % 3]
    args[3] = _i32(table)
    out = _call(planned, *args)
    torch.cuda.synchronize()
    assert torch.isfinite(out).all()
    mine = slice(batch.cu[bad], batch.cu[bad + 1])
    out[mine] = _run(batch, planned)[mine]
    batch.check(out)


@both
def test_two_recorded_steps_share_a_workspace(planned):
    """Two batches of different sizes, each recorded with its plan, replayed in turn over one workspace."""
    import paper_2505_12658_amd as hydra

    batches = [Batch([12], [2048], [1] * 12, [9 + 5 * i for i in range(12)], 32, 32, 128, seed=20), Batch([5, 20], [320, 700], [1] * 20 + [2] * 5, [9 + 7 * i for i in range(25)], 28, 4, 128, seed=21)]
    need = max(hydra.hydra_attn_prefix_workspace_bytes(len(b.kv_lens), len(b.sizes), b.q.shape[0], b.hq, b.hkv, b.d) for b in batches)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    steps = []
    for b in batches:
        args = b.on_gpu()
        out = torch.zeros_like(args[0])
        eager = _call(planned, *args, workspace=ws).clone()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            _call(planned, *args, out=out, workspace=ws)
        b.check(eager)
        steps.append((graph, out, eager, args))
    for _ in range(3):
        for graph, out, eager, _ in steps:
            out.fill_(7.0)
            graph.replay()
            assert torch.equal(out.view(torch.int16), eager.view(torch.int16))


def test_binding_refuses_mismatched_tensors():
    import paper_2505_12658_amd as hydra

    batch = Batch([3], [64], [1] * 3, [4] * 3, 4, 2, 64)
    names = ("q", "k_cache", "v_cache", "block_tables", "cu_seqlens_q", "kv_lens", "cu_groups", "shared_lens", "softmax_scale")
    good = dict(zip(names, batch.on_gpu()))
    for bad in (dict(q=good["q"][:, :, :32]), dict(q=good["q"].float()), dict(v_cache=good["v_cache"][:1]), dict(block_tables=good["block_tables"][:2]),
                dict(cu_seqlens_q=good["cu_seqlens_q"][:3]), dict(kv_lens=good["kv_lens"].long()), dict(cu_groups=good["cu_groups"][:1]), dict(shared_lens=good["shared_lens"].cpu()),
                dict(out=torch.empty_like(good["q"])[:2]), dict(workspace=torch.empty(1 << 20, dtype=torch.uint8))):
        with pytest.raises((TypeError, ValueError)):
            hydra.hydra_attn_prefix_fwd(**{**good, **bad})
    with pytest.raises(hydra.HydraError) as e:
        hydra.hydra_attn_prefix_fwd(**good, workspace=torch.empty(64, dtype=torch.uint8, device=DEV))
    assert e.value.status == 3
