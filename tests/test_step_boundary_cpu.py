"""Host-side checks of include/hydra_step.h that need no GPU: every declared call is exported, and bad arguments are refused before
anything is launched (the addresses are never dereferenced)."""
import os
import re

import pytest
import torch

import paper_2505_12658_amd as hydra

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(hydra.library_path()):
        from paper_2505_12658_amd import build

        build.build()
    return hydra.load_library()


def test_declared_calls_are_exported_and_public(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "hydra_step.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(hydra_[a-z_0-9]+)\s*\(", text)))
    assert "hydra_page_maps_build" in names and "hydra_qk_norm_rope" in names
    for n in names:
        assert getattr(lib, n) is not None and callable(getattr(hydra, n))


def _maps(lib, q=16, context=16, table=16, width=4, free=16, capacity=8, n_free=16, deltas=None, batch=2, total=8, block=16, blocks=32, cu=16, kv=16, slots=16,
          positions=16, nxt=16, pool=16):
    return lib.hydra_page_maps_build(q, context, table, width, free, capacity, n_free, deltas, batch, total, block, blocks, cu, kv, slots, positions, nxt, pool, None)


@pytest.mark.parametrize("change, status", [
    (dict(q=None), INVALID), (dict(context=None), INVALID), (dict(table=None), INVALID), (dict(free=None), INVALID), (dict(n_free=None), INVALID),
    (dict(cu=None), INVALID), (dict(kv=None), INVALID), (dict(slots=None), INVALID), (dict(pool=None), INVALID), (dict(batch=-1), INVALID), (dict(total=-1), INVALID),
    (dict(width=-1), INVALID), (dict(capacity=-1), INVALID), (dict(blocks=-1), INVALID), (dict(block=0), INVALID), (dict(block=-16), INVALID),
    (dict(block=24), UNSUPPORTED), (dict(batch=65536), UNSUPPORTED), (dict(total=(1 << 20) + 1), UNSUPPORTED), (dict(blocks=1 << 27), UNSUPPORTED),
    (dict(width=(1 << 26) + 1), UNSUPPORTED), (dict(batch=0), OK),
], ids=str)
def test_page_maps_refusals(lib, change, status):
    assert _maps(lib, **change) == status


def _rope(lib, q=16, k=16, v=16, qs=128, ks=128, vs=128, qo=32, ko=32, qos=128, kos=128, qw=None, kw=None, eps=1e-6, positions=16, axis_stride=8, axes=1, freq=16, axis=None,
          rotary=64, interleaved=0, kc=16, vc=16, slots=16, block=16, blocks=4, tokens=8, hq=2, hkv=2, d=64):
    return lib.hydra_qk_norm_rope(q, k, v, qs, ks, vs, qo, ko, qos, kos, qw, kw, eps, positions, axis_stride, axes, freq, axis, rotary, interleaved, kc, vc, slots, block, blocks,
                                  tokens, hq, hkv, d, None)


@pytest.mark.parametrize("change, status", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(qo=None), INVALID), (dict(ko=None, kc=None, vc=None, slots=None), INVALID),
    (dict(kc=None), INVALID), (dict(vc=None), INVALID), (dict(slots=None), INVALID), (dict(positions=None), INVALID), (dict(freq=None), INVALID),
    (dict(q=8), INVALID), (dict(ko=8), INVALID), (dict(vc=8), INVALID), (dict(qw=8), INVALID), (dict(qs=120), INVALID), (dict(kos=64), INVALID), (dict(vs=132), INVALID),
    (dict(qos=132), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(axes=0), INVALID),
    (dict(axis_stride=-8), INVALID), (dict(tokens=-1), INVALID), (dict(hq=0), INVALID), (dict(hkv=0), INVALID), (dict(rotary=-16), INVALID), (dict(rotary=80), INVALID),
    (dict(block=0), INVALID), (dict(blocks=-1), INVALID), (dict(qo=16, qos=256), INVALID), (dict(ko=16, kos=256), INVALID),
    (dict(axes=5), UNSUPPORTED), (dict(rotary=24), UNSUPPORTED), (dict(d=96), UNSUPPORTED), (dict(d=0), UNSUPPORTED), (dict(tokens=(1 << 25) + 1), UNSUPPORTED),
    (dict(hq=65535, qs=1 << 23, qos=1 << 23), UNSUPPORTED), (dict(blocks=1 << 60), UNSUPPORTED), (dict(tokens=0), OK),
], ids=str)
def test_norm_and_rotation_refusals(lib, change, status):
    assert _rope(lib, **change) == status


def _prefix(lib, q=16, out=32, qs=128, kc=16, vc=16, table=16, width=4, cu=16, kv=16, groups=16, shared=16, batch=3, n_groups=1, total=3, hq=2, hkv=2, d=64, block=16, blocks=32,
            scale=0.125, ws=16, ws_bytes=1 << 30):
    return lib.hydra_attn_prefix_fwd(q, out, qs, kc, vc, table, width, cu, kv, groups, shared, batch, n_groups, total, hq, hkv, d, block, blocks, scale, ws, ws_bytes, None)


@pytest.mark.parametrize("change, status", [
    (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(kc=None), INVALID), (dict(vc=None), INVALID), (dict(table=None), INVALID), (dict(cu=None), INVALID), (dict(kv=None), INVALID),
    (dict(groups=None), INVALID), (dict(shared=None), INVALID), (dict(q=8), INVALID), (dict(out=8), INVALID), (dict(vc=24), INVALID), (dict(qs=120), INVALID), (dict(qs=132), INVALID),
    (dict(batch=-1), INVALID), (dict(n_groups=-1), INVALID), (dict(n_groups=0), INVALID), (dict(total=-1), INVALID), (dict(hq=3), INVALID), (dict(hkv=0), INVALID), (dict(width=0), INVALID),
    (dict(blocks=0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=float("inf")), INVALID), (dict(d=96), UNSUPPORTED),
    (dict(batch=2049), UNSUPPORTED), (dict(n_groups=2049), UNSUPPORTED), (dict(total=(1 << 23) + 1), UNSUPPORTED), (dict(block=24), UNSUPPORTED), (dict(block=0), UNSUPPORTED),
    (dict(blocks=1 << 27), UNSUPPORTED), (dict(width=(1 << 26) + 1), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(ws=24), WORKSPACE), (dict(ws_bytes=1000), WORKSPACE),
    (dict(batch=0), OK), (dict(total=0), OK), (dict(batch=0, n_groups=0), OK),
], ids=str)
def test_prefix_attention_refusals(lib, change, status):
    assert _prefix(lib, **change) == status


def test_prefix_plan_and_planned_refusals(lib):
    plan = lambda cu=16, width=4, block=16, ws=16, n=1 << 30: lib.hydra_attn_prefix_plan(cu, 16, 16, 16, 3, 1, 3, 2, 2, 64, width, block, ws, n, None)  # noqa: E731
    assert plan(cu=None) == INVALID and plan(width=0) == INVALID and plan(block=0) == INVALID
    assert plan(block=12) == UNSUPPORTED and plan(ws=None) == WORKSPACE and plan(n=64) == WORKSPACE
    run = lambda q=16, table=16, ws=16, n=1 << 30: lib.hydra_attn_prefix_fwd_planned(q, 32, 128, 16, 16, table, 4, 3, 1, 3, 2, 2, 64, 16, 32, 0.125, ws, n, None)  # noqa: E731
    assert run(q=None) == INVALID and run(table=None) == INVALID and run(ws=None) == WORKSPACE and run(n=64) == WORKSPACE


def test_prefix_workspace_bytes(lib):
    size = hydra.hydra_attn_prefix_workspace_bytes
    assert size(3, 1, 3, 3, 2, 64) == 0 and size(3, 1, 3, 2, 2, 96) == 0 and size(2049, 1, 3, 2, 2, 64) == 0
    assert 0 < size(3, 1, 3, 2, 2, 64) < size(300, 1, 3000, 2, 2, 64) < size(300, 1, 3000, 2, 2, 128)


def test_binding_refuses_what_is_no_gpu_tensor():
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        hydra.hydra_qk_norm_rope(q, q, None, None)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        hydra.hydra_page_maps_build(i, i, i.view(4, 1), i, i[:1], 4, 16, 8)
