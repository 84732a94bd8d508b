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
    (dict(hq=65535, qs=1 << 23, qos=1 << 23), UNSUPPORTED), (dict(tokens=0), OK),
], ids=str)
def test_norm_and_rotation_refusals(lib, change, status):
    assert _rope(lib, **change) == status


def test_binding_refuses_what_is_no_gpu_tensor():
    q = torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        hydra.hydra_qk_norm_rope(q, q, None, None)
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        hydra.hydra_page_maps_build(i, i, i.view(4, 1), i, i[:1], 4, 16, 8)
