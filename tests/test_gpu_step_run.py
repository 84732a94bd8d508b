"""Steps of a serving instance, as its layers run them: page maps, norm and rotation with the cache write, and attention over the prefixes
that requests share; eagerly and recorded into a graph.  What every request should see is kept apart, densely and in 64 bits."""
import numpy as np
import pytest
import torch

import synth_inputs as si
from oracle import reference

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BLOCK, HQ, HKV, D = 16, 14, 2, 128
HALF_STEP = torch.finfo(torch.bfloat16).eps / 2


def _f64(t):
    return reference.bf16_bits_to_f64(si.bf16_bits(t))


class Instance:
    """Two groups of requests behind prompts of their own, whose whole blocks they share; the prompts' tokens are in the cache."""

    def __init__(self, prompts, sizes, room, seed):
        self.rng, self.gen = np.random.default_rng(seed), torch.Generator().manual_seed(seed)
        self.sizes, self.prompts = sizes, prompts
        self.group_of = [g for g, n in enumerate(sizes) for _ in range(n)]
        self.batch, self.room = sum(sizes), room
        self.blocks = sum(p // BLOCK for p in prompts) + 30 * self.batch
        ids = self.rng.permutation(self.blocks).astype(np.int32)
        shared = [p // BLOCK for p in prompts]
        width = max(shared) + 24
        tables = np.full((self.batch, width), -1, np.int32)
        at = 0
        for g, n in enumerate(shared):
            for b in range(self.batch):
                if self.group_of[b] == g:
                    tables[b, :n] = ids[at: at + n]
            at += n
        i32 = lambda x: torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)  # noqa: E731
        draw = lambda *shape: torch.randn(shape, generator=self.gen).to(torch.bfloat16)  # noqa: E731
        self.k_cache, self.v_cache = (torch.full((self.blocks, BLOCK, HKV, D), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        prefix = []
        for g, n in enumerate(shared):
            k, v = draw(n, BLOCK, HKV, D), draw(n, BLOCK, HKV, D)
            rows = torch.from_numpy(ids[sum(shared[:g]): sum(shared[:g]) + n].astype(np.int64)).to(DEV)
            self.k_cache[rows], self.v_cache[rows] = k.to(DEV), v.to(DEV)
            prefix.append((_f64(k).reshape(-1, HKV, D), _f64(v).reshape(-1, HKV, D)))
        self.keys, self.values = [prefix[g][0] for g in self.group_of], [prefix[g][1] for g in self.group_of]
        self.table, self.context = i32(tables), i32([shared[g] * BLOCK for g in self.group_of])
        self.free, self.pool = i32(np.concatenate([ids[at:], np.zeros(at, np.int32)])), i32([self.blocks - at, 0])
        self.cu_groups, self.shared = i32(np.concatenate([[0], np.cumsum(sizes)])), i32([n * BLOCK for n in shared])
        self.q_lens, self.deltas = i32(np.zeros(self.batch)), i32(self.rng.integers(-40, 40, self.batch))
        self.fused = torch.zeros((room, (HQ + 2 * HKV) * D), dtype=torch.bfloat16, device=DEV)
        self.weights = [(1 + 0.2 * torch.randn(D, generator=self.gen)).to(torch.bfloat16) for _ in range(2)]
        self.weights_on = [w.to(DEV) for w in self.weights]
        self.freq = (1000000.0 ** -(np.arange(D // 2) / (D // 2))).astype(np.float32)
        self.axis = np.arange(D // 2, dtype=np.int32) % 3
        self.freq_on, self.axis_on = torch.from_numpy(self.freq).to(DEV), torch.from_numpy(self.axis).to(DEV)
        e = lambda n, t=torch.int32: torch.empty(n, dtype=t, device=DEV)  # noqa: E731
        import paper_2505_12658_amd as hydra

        self.hydra = hydra
        self.maps = hydra.PageMaps(e(self.batch + 1), e(self.batch), e(room, torch.int64), e(room), self.context, self.pool)
        self.q, self.out = (torch.empty((room, HQ, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        self.workspace = e(hydra.hydra_attn_prefix_workspace_bytes(self.batch, len(sizes), room, HQ, HKV, D), torch.uint8)

    def layer(self, planned):
        hydra, m = self.hydra, self.maps
        hydra.hydra_page_maps_build(self.q_lens, self.context, self.table, self.free, self.pool, self.room, BLOCK, self.blocks, position_deltas=self.deltas, maps=m)
        q, k, v = (x.view(self.room, -1, D) for x in self.fused.split([HQ * D, HKV * D, HKV * D], dim=1))
        positions = m.positions.unsqueeze(0).expand(3, -1)  # (text: the same on every axis)
        hydra.hydra_qk_norm_rope(q, k, positions, self.freq_on, freq_axis=self.axis_on, q_weight=self.weights_on[0], k_weight=self.weights_on[1], q_out=self.q, v=v,
                                 k_cache=self.k_cache, v_cache=self.v_cache, slot_mapping=m.slot_mapping)
        if planned:
            hydra.hydra_attn_prefix_plan(m.cu_seqlens_q, m.kv_lens, self.cu_groups, self.shared, self.room, HQ, HKV, D, self.table.shape[1], BLOCK, workspace=self.workspace)
            hydra.hydra_attn_prefix_fwd_planned(self.q, self.k_cache, self.v_cache, self.table, len(self.sizes), D ** -0.5, self.workspace, out=self.out)
        else:
            hydra.hydra_attn_prefix_fwd(self.q, self.k_cache, self.v_cache, self.table, m.cu_seqlens_q, m.kv_lens, self.cu_groups, self.shared, D ** -0.5, out=self.out,
                                        workspace=self.workspace)

    def new_step(self, q_lens):
        self.now = list(q_lens)
        self.q_lens.copy_(torch.tensor(q_lens, dtype=torch.int32))
        fused = torch.randn(self.fused.shape, generator=self.gen).to(torch.bfloat16)
        self.fused.copy_(fused)
        self.out.fill_(9.0)
        self.host = _f64(fused).reshape(self.room, -1, D)

    def check(self):
        """Rotated rows are off by half a step of bf16, queries and keys: that moves a score of a few units by some 2^-8 of it, on average far less, and
        the output by as much of the values' size; with the probabilities' and the output's own half steps under 4 of them."""
        torch.cuda.synchronize()
        out, at = _f64(self.out), 0
        for b, n in enumerate(self.now):
            rows = self.host[at: at + n]
            positions = np.arange(n)[None, :].repeat(3, 0) + len(self.keys[b]) + int(self.deltas[b])
            turned = lambda x, w: reference.qk_norm_rope(x, _f64(w), 1e-6, positions, self.freq, self.axis, False)  # noqa: E731
            q = turned(rows[:, :HQ], self.weights[0])
            self.keys[b] = np.concatenate([self.keys[b], turned(rows[:, HQ: HQ + HKV], self.weights[1])])
            self.values[b] = np.concatenate([self.values[b], rows[:, HQ + HKV:]])
            if n:
                length = len(self.keys[b])
                table, cu = np.arange(length)[None, :], [0, n]
                want = reference.attn_paged(q, self.keys[b][:, None], self.values[b][:, None], table, cu, [length], D ** -0.5)
                size = np.sqrt((self.values[b] ** 2).mean())
                off = np.abs(out[at: at + n] - want)
                assert np.isfinite(off).all() and (off <= 4 * HALF_STEP * (size + np.abs(want))).all(), (b, off.max())
            at += n
        assert (out[at:] == 9.0).all()  # tokens behind the last request


STEPS = [[1, 1, 1, 1, 1, 1, 1], [1, 0, 1, 9, 1, 1, 2], [1, 1, 1, 1, 0, 20, 1], [0, 1, 1, 1, 1, 1, 1]]


@pytest.mark.parametrize("planned", [True, False], ids=["planned", "whole"])
@pytest.mark.parametrize("recorded", [False, True], ids=["eager", "recorded"])
def test_steps_of_requests_behind_shared_prompts(recorded, planned):
    instance = Instance([330, 700], [4, 3], 40, seed=1)
    instance.new_step([0] * 7)
    instance.layer(planned)  # (a step without tokens; everything is loaded by then)
    instance.check()
    graph = None
    if recorded:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            instance.layer(planned)
    for q_lens in STEPS:
        instance.new_step(q_lens)
        torch.cuda.synchronize()
        if recorded:
            graph.replay()
        else:
            instance.layer(planned)
        instance.check()


def test_two_instances_on_two_streams():
    """Two instances with workspaces of their own, their steps enqueued side by side."""
    instances = [Instance([330, 700], [4, 3], 40, seed=2), Instance([1000, 64], [3, 4], 33, seed=3)]
    streams = [torch.cuda.Stream() for _ in instances]
    for q_lens in STEPS:
        for instance in instances:
            instance.new_step(q_lens)
        torch.cuda.synchronize()
        for instance, stream in zip(instances, streams):
            with torch.cuda.stream(stream):
                instance.layer(True)
        for instance in instances:
            instance.check()
