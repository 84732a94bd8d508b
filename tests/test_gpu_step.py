"""Page maps and norm + rotation against the 64-bit oracle, on the GPU."""
import numpy as np
import pytest
import torch

import synth_inputs as si
from oracle import reference

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _f64(t):
    return reference.bf16_bits_to_f64(si.bf16_bits(t))


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


# ---- page maps -----------------------------------------------------------------------------------------------


def _maps_case(seed, batch, q_most, context_most, block, lacking=0, total_more=0, empty=0.2):
    """Lengths, a table whose used entries are blocks of their own, and a free list."""
    rng = np.random.default_rng(seed)
    q = rng.integers(1, q_most + 1, batch) * (rng.random(batch) >= empty)
    context = rng.integers(0, context_most + 1, batch)
    held, after = -(-context // block), -(-(context + q) // block)
    need = int((after - held).sum())
    free = max(need - lacking, 0) + (0 if lacking else 3)
    blocks = int(held.sum()) + max(free, need) + 5
    ids = rng.permutation(blocks).astype(np.int32)
    width = int(after.max(initial=0)) + 2
    tables = np.full((batch, width), -1, np.int32)
    at = 0
    for b in range(batch):
        tables[b, :held[b]] = ids[at: at + held[b]]
        at += held[b]
    list_ = np.full(free + 4, -77, np.int32)  # (longer than what is on it)
    list_[:free] = ids[at: at + free]
    return q, context, tables, list_, free, int(q.sum()) + total_more, blocks


def _maps_run(q, context, tables, list_, n_free, total, block, blocks, deltas=None, **kw):
    import paper_2505_12658_amd as hydra

    table = _i32(tables)
    got = hydra.hydra_page_maps_build(_i32(q), _i32(context), table, _i32(list_), _i32([n_free]), total, block, blocks,
                                      position_deltas=None if deltas is None else _i32(deltas), **kw)
    torch.cuda.synchronize()
    return [t.cpu().numpy() for t in got] + [table.cpu().numpy()]


def _maps_check(got, want):
    for name, g, w in zip(("cu_seqlens_q", "kv_lens", "slot_mapping", "positions", "next_context", "pool", "block_tables"), got, want):
        assert np.array_equal(g, np.asarray(w)), name


@pytest.mark.parametrize("batch, q_most, context_most, block, lacking, more", [
    (1, 1, 0, 16, 0, 0), (1, 1, 31, 16, 0, 3), (3, 40, 50, 1, 0, 0), (5, 17, 33, 16, 4, 1), (64, 1, 700, 16, 0, 0), (65, 1, 700, 16, 3, 7), (130, 90, 300, 8, 0, 0),
    (200, 300, 10, 32, 200, 11), (1023, 1, 60, 4, 0, 0), (1024, 3, 60, 2, 5, 0), (1025, 9, 20, 16, 0, 1), (2500, 2, 90, 16, 9, 0), (40, 1200, 0, 16, 0, 5),
    (7, 5000, 3000, 64, 0, 0), (33, 2, 100, 256, 1, 40),
    (256, 9, 30, 4, 0, 0), (257, 9, 30, 4, 2, 3), (900, 2000, 100, 16, 30, 7), (65535, 3, 40, 8, 0, 5),
])
def test_page_maps(batch, q_most, context_most, block, lacking, more):
    q, context, tables, list_, free, total, blocks = _maps_case(batch * 7 + block, batch, q_most, context_most, block, lacking, more)
    deltas = np.random.default_rng(batch).integers(-500, 500, batch)
    args = (q, context, tables, list_, free, total, block, blocks)
    _maps_check(_maps_run(*args, deltas=deltas), reference.page_maps(*args, position_deltas=deltas))
    _maps_check(_maps_run(*args), reference.page_maps(*args))


@pytest.mark.parametrize("batch, q_most, lacking", [(1500, 1, 0), (2300, 1, 40), (300, 50, 0), (1100, 400, 9)])
def test_page_maps_of_large_batches_in_place(batch, q_most, lacking):
    """Context lengths and free list overwritten by the call that reads them, in several rounds and several workgroups."""
    import paper_2505_12658_amd as hydra

    q, context, tables, list_, free, total, blocks = _maps_case(batch, batch, q_most, 90, 16, lacking)
    e = lambda n, t=torch.int32: torch.empty(n, dtype=t, device=DEV)  # noqa: E731
    table, d_context, pool = _i32(tables), _i32(context), _i32([free, 0])
    maps = hydra.PageMaps(e(batch + 1), e(batch), e(total, torch.int64), e(total), d_context, pool)
    hydra.hydra_page_maps_build(_i32(q), d_context, table, _i32(list_), pool, total, 16, blocks, maps=maps)
    torch.cuda.synchronize()
    _maps_check([t.cpu().numpy() for t in (*maps, table)], reference.page_maps(q, context, tables, list_, free, total, 16, blocks))


def test_page_maps_of_lengths_that_do_not_fit():
    """Requests beyond their row of the table, beyond total_tokens, with negative lengths; block ids outside the cache."""
    q = [5, -3, 20, 4, 0, 1 << 29, 3, 2, 0]
    context = [10, 4, 60, -7, 33, 2, 15, 30, 7]
    tables = np.arange(9 * 5, dtype=np.int32).reshape(9, 5)
    tables[0, 0] = 99
    tables[7, 1] = -4
    list_ = [50, 51, 120, 53]
    for total in (16, 20, 29, 36, 60):
        for n_free in (-2, 0, 1, 2, 4, 9):
            args = (q, context, tables, list_, n_free, total, 16, 60)
            _maps_check(_maps_run(*args), reference.page_maps(*args))


@pytest.mark.parametrize("total_more", [0, 9000])
def test_page_maps_moving_on_in_place(total_more):
    """Context lengths, free list and tables that every step leaves as the next one needs them, in one workgroup and in several; recorded once
    into a graph and replayed, until blocks are lacking."""
    import paper_2505_12658_amd as hydra

    rng = np.random.default_rng(3)
    batch, block, blocks = 37, 4, 300
    context, tables, list_ = np.zeros(batch, int), np.full((batch, 20), -1, np.int32), rng.permutation(blocks).astype(np.int32)
    n_free, room = 150, 3 * batch + total_more
    d_q, d_context, d_table, d_list, d_pool = _i32(np.zeros(batch)), _i32(context), _i32(tables), _i32(list_), _i32([n_free, 0])
    e = lambda n, t=torch.int32: torch.empty(n, dtype=t, device=DEV)  # noqa: E731
    maps = hydra.PageMaps(e(batch + 1), e(batch), e(room, torch.int64), e(room), d_context, d_pool)

    def step():
        hydra.hydra_page_maps_build(d_q, d_context, d_table, d_list, d_pool, room, block, blocks, maps=maps)

    step()  # (a step without tokens changes nothing)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    lacked = 0
    for i in range(14):
        q = rng.integers(0, 4, batch)
        d_q.copy_(_i32(q))
        graph.replay()
        torch.cuda.synchronize()
        want = reference.page_maps(q, context, tables, list_, n_free, room, block, blocks)
        _maps_check([t.cpu().numpy() for t in maps] + [d_table.cpu().numpy()], want)
        context, tables, n_free = np.array(want[4]), want[6], want[5][0]
        lacked += want[5][1]
    assert lacked > 0


def test_page_maps_leave_what_is_not_theirs():
    """Optional outputs left out; buffers longer than the step keep what is behind total_tokens."""
    import paper_2505_12658_amd as hydra

    q, context, tables, list_, free, total, blocks = _maps_case(5, 20, 6, 40, 16)
    slots = torch.full((total + 6,), 12345, dtype=torch.int64, device=DEV)
    e = lambda n: torch.empty(n, dtype=torch.int32, device=DEV)  # noqa: E731
    maps = hydra.PageMaps(e(21), e(20), slots, None, None, e(2))
    hydra.hydra_page_maps_build(_i32(q), _i32(context), _i32(tables), _i32(list_), _i32([free]), total, 16, blocks, maps=maps)
    want = reference.page_maps(q, context, tables, list_, free, total, 16, blocks)
    assert np.array_equal(slots.cpu().numpy(), np.concatenate([want[2], np.full(6, 12345)]))
    assert np.array_equal(maps.cu_seqlens_q.cpu().numpy(), want[0])


# ---- norm and rotation ---------------------------------------------------------------------------------------

# Per element, relative to the two elements of its pair after the norm: sine and cosine of the hardware are off by 2^-22.3 at most (measured
# over 2^28 arguments), two products and a sum by 3 2^-24: together below 2^-21.  With a norm also the scale of the row: 16
# products and sums one after the other and three more, halved by the root, root, quotient and two products: below 2^-20.
# Then the rounding to bf16, half a step.
HALF_STEP = torch.finfo(torch.bfloat16).eps / 2


def _allowed(want, x, normed, interleaved, pairs):
    size = np.abs(x)
    other = size.copy()
    for i in range(pairs):
        l, u = (2 * i, 2 * i + 1) if interleaved else (i, i + pairs)
        other[:, :, l], other[:, :, u] = size[:, :, l] + size[:, :, u], size[:, :, l] + size[:, :, u]
    return HALF_STEP * np.abs(want) * (1 + 2.0 ** -10) + (2.0 ** -21 + (2.0 ** -20 if normed else 0)) * other + 1e-38


def _near(got, x, weight, eps, positions, freq, axis, interleaved):
    want = reference.qk_norm_rope(x, weight, eps, positions, freq, axis, interleaved)
    flat = reference.qk_norm_rope(x, weight, eps, positions, [], None, interleaved)
    off = np.abs(_f64(got) - want)
    allowed = _allowed(want, flat, weight is not None, interleaved, len(freq))
    assert np.isfinite(off).all() and (off <= allowed).all(), f"off by {(off / allowed).max():.3f} of what is allowed"


def _draw(seed, n, hq, hkv, d):
    g = torch.Generator().manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g).to(torch.bfloat16)  # noqa: E731
    return normal(n, hq, d), normal(n, hkv, d), normal(n, hkv, d), (1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16), (1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16)


def _freq(pairs, base=10000.0):
    return (base ** (-np.arange(pairs) / max(pairs, 1))).astype(np.float32)


ROPE_CASES = [
    # tokens, Hq, Hkv, d, rotary, axes, norm, interleaved, cache
    (1, 1, 1, 64, 64, 1, False, False, False), (1, 28, 4, 128, 128, 3, True, False, True), (2, 28, 4, 128, 128, 3, False, False, True),
    (3, 32, 32, 128, 128, 1, True, False, True), (5, 16, 16, 80, 80, 2, False, False, False), (5, 16, 16, 80, 80, 2, True, False, False),
    (7, 3, 1, 80, 48, 4, True, True, True), (17, 5, 5, 64, 32, 2, True, True, True), (33, 7, 1, 128, 64, 1, False, True, True), (130, 28, 4, 64, 64, 3, True, False, True),
    (257, 2, 2, 80, 16, 1, False, False, True), (1000, 9, 3, 128, 96, 2, True, False, False), (4099, 4, 1, 64, 0, 1, True, False, True), (4100, 4, 2, 128, 128, 3, False, False, True),
    (8193, 1, 1, 80, 80, 1, True, False, False), (300, 13, 1, 128, 0, 1, False, False, True),
]


@pytest.mark.parametrize("case", ROPE_CASES, ids=lambda c: "-".join(map(str, c)))
def test_norm_and_rotation(case):
    import paper_2505_12658_amd as hydra

    n, hq, hkv, d, rotary, axes, norm, interleaved, cache = case
    q, k, v, qw, kw = _draw(n + d, n, hq, hkv, d)
    rng = np.random.default_rng(n)
    positions = rng.integers(0, 40000, (axes, n))
    freq, axis = _freq(rotary // 2), rng.integers(0, axes, rotary // 2)
    more = {}
    if cache:
        block = 16 if n % 2 else 5
        blocks = -(-n // block) + 2
        slots = rng.permutation(blocks * block)[:n].astype(np.int64)
        slots[rng.random(n) < 0.2] = -1
        kc0, vc0 = (si.make_cache_sentinel(blocks, block, hkv, d, seed=s) for s in (1, 2))
        kc, vc = (torch.from_numpy(c.view(np.int16).copy()).view(torch.bfloat16).to(DEV) for c in (kc0, vc0))
        more = dict(v=v.to(DEV), k_cache=kc, v_cache=vc, slot_mapping=torch.from_numpy(slots).to(DEV), k_out=torch.empty_like(k, device=DEV) if n % 3 else None)
    q_out, k_out = hydra.hydra_qk_norm_rope(q.to(DEV), k.to(DEV), _i32(positions), torch.from_numpy(freq).to(DEV), freq_axis=_i32(axis), q_weight=qw.to(DEV) if norm else None,
                                            k_weight=kw.to(DEV) if norm else None, eps=1e-5, interleaved=interleaved, **more)
    torch.cuda.synchronize()
    _near(q_out, _f64(q), _f64(qw) if norm else None, 1e-5, positions, freq, axis, interleaved)
    assert (k_out is None) == (cache and n % 3 == 0)
    if k_out is not None:
        _near(k_out, _f64(k), _f64(kw) if norm else None, 1e-5, positions, freq, axis, interleaved)
    if cache:
        keep = slots >= 0
        rows = kc.view(-1, hkv, d)[torch.from_numpy(slots[keep]).to(DEV)]
        _near(rows, _f64(k)[keep], _f64(kw) if norm else None, 1e-5, positions[:, keep], freq, axis, interleaved)
        want_v = vc0.reshape(-1, hkv, d)
        want_v[slots[keep]] = si.bf16_bits(v)[keep]
        assert np.array_equal(si.bf16_bits(vc).reshape(-1, hkv, d), want_v)
        others = np.setdiff1d(np.arange(blocks * block), slots[keep])
        assert np.array_equal(si.bf16_bits(kc).reshape(-1, hkv, d)[others], kc0.reshape(-1, hkv, d)[others])


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("d", [64, 80, 128])
def test_in_place_on_views_of_one_buffer(d, norm):
    """q and k are parts of one projection's rows and are rotated where they lie; the rows' other parts keep their bits."""
    import paper_2505_12658_amd as hydra

    n, hq, hkv = 77, 6, 2
    g = torch.Generator().manual_seed(d)
    fused = torch.randn((n, (hq + 2 * hkv) * d + 24), generator=g).to(torch.bfloat16)
    dev = fused.to(DEV)
    part = lambda t, at, heads: t[:, at: at + heads * d].view(n, heads, d)  # noqa: E731
    q, k = part(dev, 0, hq), part(dev, hq * d, hkv)
    weight = (1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16)
    positions, freq = np.arange(n)[None, :] * 3, _freq(d // 2)
    w = weight.to(DEV) if norm else None
    a, b = hydra.hydra_qk_norm_rope(q, k, _i32(positions[0]), torch.from_numpy(freq).to(DEV), q_weight=w, k_weight=w, q_out=q, k_out=k)
    torch.cuda.synchronize()
    assert a.data_ptr() == q.data_ptr() and b.data_ptr() == k.data_ptr()
    for got, at, heads in ((q, 0, hq), (k, hq * d, hkv)):
        _near(got.contiguous(), _f64(part(fused, at, heads).contiguous()), _f64(weight) if norm else None, 1e-6, positions, freq, None, False)
    rest = (hq + hkv) * d
    assert torch.equal(dev[:, rest:].cpu().view(torch.int16), fused[:, rest:].view(torch.int16))


def test_far_positions_and_frequencies():
    """Every int32 position, frequencies above 1 and negative ones, axes outside their range."""
    import paper_2505_12658_amd as hydra

    positions = np.array([[0, 1, -1, 2**31 - 1, -2**31, 123456789, -987654321, 131072, 1 << 24], [5, 4, 3, 2, 1, 0, -1, -2, -3]])
    freq = np.concatenate([_freq(24), [1.0, 2.5, -3.75, 100.0, 1e-9, 0.0, -1e-3, 6.2831855]]).astype(np.float32)
    axis = np.array([0, 1, -5, 7] * 8)
    q, k, *_ = _draw(9, 9, 2, 1, 64)
    q_out, k_out = hydra.hydra_qk_norm_rope(q.to(DEV), k.to(DEV), _i32(positions), torch.from_numpy(freq).to(DEV), freq_axis=_i32(axis))
    for got, x in ((q_out, q), (k_out, k)):
        _near(got, _f64(x), None, 0.0, positions, freq, axis, False)


def test_one_norm_only_zero_rows_and_infinities_beside_the_rotated_part():
    import paper_2505_12658_amd as hydra

    q, k, _, qw, kw = _draw(4, 6, 4, 2, 128)
    q[2, 1] = 0
    q[3, 0, 70:] = float("inf")  # (k has no norm here and its last elements do not rotate)
    k[0, 1, 100] = float("inf")
    k[1, 0, 127] = float("nan")
    positions, freq = np.arange(6)[None, :] + 9, _freq(32)
    args = (_i32(positions), torch.from_numpy(freq).to(DEV))
    _, k_out = hydra.hydra_qk_norm_rope(q.to(DEV), k.to(DEV), *args, q_weight=qw.to(DEV))
    bits, want = si.bf16_bits(k_out)[:, :, 64:], si.bf16_bits(k)[:, :, 64:]
    assert np.array_equal(bits, want)
    q_out, _ = hydra.hydra_qk_norm_rope(q.to(DEV), k.to(DEV), *args, k_weight=kw.to(DEV))
    assert torch.equal(q_out[..., 64:].cpu().view(torch.int16), q[..., 64:].view(torch.int16))
    q[3, 0, 70:] = 1
    q_out, _ = hydra.hydra_qk_norm_rope(q.to(DEV), k.to(DEV), *args, q_weight=qw.to(DEV), eps=1e-6)
    _near(q_out, _f64(q), _f64(qw), 1e-6, positions, freq, None, False)
    assert (q_out[2, 1] == 0).all()


def test_slots_outside_the_cache_are_not_written():
    import paper_2505_12658_amd as hydra

    q, k, v, *_ = _draw(8, 4, 2, 2, 64)
    caches = torch.full((2, 3, 16, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)  # (the calls get the middle block)
    slots = torch.tensor([16, -1, 3, 1 << 40], dtype=torch.int64, device=DEV)
    hydra.hydra_qk_norm_rope(q.to(DEV), k.to(DEV), None, None, v=v.to(DEV), k_cache=caches[0, 1:2], v_cache=caches[1, 1:2], slot_mapping=slots)
    want = torch.full((2, 3, 16, 2, 64), 7.0, dtype=torch.bfloat16)
    want[0, 1, 3], want[1, 1, 3] = k[2], v[2]
    assert torch.equal(caches.cpu(), want)


def test_slots_behind_the_first_four_gigabytes():
    import paper_2505_12658_amd as hydra

    q, k, v, _, _ = (t.to(DEV) for t in _draw(3, 5, 4, 8, 128))
    slots = torch.tensor([2621500, 0, 2300000, 2621439, 17], device=DEV)  # (rows of 2 KB: 5.4 GB)
    kc, vc = (torch.zeros((163900, 16, 8, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    _, none = hydra.hydra_qk_norm_rope(q, k, None, None, v=v, k_cache=kc, v_cache=vc, slot_mapping=slots)
    for cache, rows in ((kc, k), (vc, v)):
        assert torch.equal(cache.view(-1, 8, 128)[slots], rows)
        assert int((cache.view(-1, 1024) != 0).any(1).sum()) == 5


def test_step_calls_on_a_stream_of_their_own():
    """Both calls, one after the other on a side stream that is given as an argument, allocating their outputs."""
    import paper_2505_12658_amd as hydra

    q_lens, context, tables, list_, free, total, blocks = _maps_case(11, 30, 3, 100, 16)
    q, k, v, qw, kw = (t.to(DEV) for t in _draw(11, total, 4, 2, 128))
    kc, vc = torch.zeros((2, blocks, 16, 2, 128), dtype=torch.bfloat16, device=DEV)
    inv_freq = torch.from_numpy(_freq(64)).to(DEV)
    args = [_i32(x) for x in (q_lens, context, tables, list_, [free])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    maps = hydra.hydra_page_maps_build(*args, total, 16, blocks, stream=side)
    q_out, none = hydra.hydra_qk_norm_rope(q, k, maps.positions, inv_freq, v=v, k_cache=kc, v_cache=vc, slot_mapping=maps.slot_mapping, stream=side)
    side.synchronize()
    want = reference.page_maps(q_lens, context, tables, list_, free, total, 16, blocks)
    assert none is None and np.array_equal(maps.slot_mapping.cpu().numpy(), want[2])
    positions = want[3][None, :]
    _near(q_out, _f64(q), None, 0.0, positions, _freq(64), None, False)
    _near(kc.view(-1, 2, 128)[maps.slot_mapping], _f64(k), None, 0.0, positions, _freq(64), None, False)
    assert torch.equal(vc.view(-1, 2, 128)[maps.slot_mapping], v)


def test_binding_refuses_mismatched_tensors():
    import paper_2505_12658_amd as hydra

    q, k, v, qw, kw = (t.to(DEV) for t in _draw(1, 4, 4, 2, 64))
    freq = torch.from_numpy(_freq(32)).to(DEV)
    p = _i32(range(4))
    kc, vc = torch.zeros((2, 2, 16, 2, 64), dtype=torch.bfloat16, device=DEV)
    slots = torch.arange(4, device=DEV)
    for bad in (dict(positions=p[:3]), dict(positions=None), dict(positions=p.long()), dict(inv_freq=freq.double()), dict(freq_axis=p), dict(q_weight=qw[:32]), dict(q_weight=qw.float()),
                dict(k_cache=kc), dict(k_cache=kc, v_cache=vc, slot_mapping=slots), dict(v=v, k_cache=kc, v_cache=vc, slot_mapping=slots.int()),
                dict(v=v, k_cache=kc, v_cache=vc[:1], slot_mapping=slots), dict(q_out=q[:3]), dict(k_out=q), dict(q_weight=qw.cpu()), dict(k=k[:, :, :32])):
        with pytest.raises((TypeError, ValueError)):
            hydra.hydra_qk_norm_rope(**{**dict(q=q, k=k, positions=p, inv_freq=freq), **bad})
    with pytest.raises(hydra.HydraError):
        hydra.hydra_qk_norm_rope(q, k, p, freq[:12])  # (24 of 64 elements rotated: no whole pieces)
    i = _i32([1, 2])
    with pytest.raises(ValueError):
        hydra.hydra_page_maps_build(i, i[:1], i.view(2, 1), i, i[:1], 4, 16, 8)
    with pytest.raises(hydra.HydraError):
        hydra.hydra_page_maps_build(i, i, i.view(2, 1), i, i[:1], 4, 12, 8)
