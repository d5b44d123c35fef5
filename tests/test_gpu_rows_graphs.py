"""A verification step as it is served, appending the drafts and attending over their tree, captured once and replayed with
other tokens, two of them at once with a cache and a workspace each."""

import numpy as np
import pytest
import torch

from paper_2506_03781_gb300 import api
from tests import kv_cases as C
from tests.rows_cases import signed, tree_masks
from tests.test_gpu_append import rope_table

pytestmark = pytest.mark.gpu
H, KV, HD, PAGE, DRAFTS = 8, 2, 128, 16, 12


class Step:
    """Three sequences, `DRAFTS` rows each, of which counts[b] are drafts; what the cache holds before is the same for all."""

    def __init__(self, fmt, dtype):
        self.lens, self.counts = [40, 200, 9], [12, 5, 1]
        d = lambda a, t: torch.tensor(a, dtype=t, device=C.dev())
        self.cache = api.empty_kv_cache(40, KV, PAGE, HD, C.FMT[fmt], C.dev())
        C.poison(self.cache)
        self.table = torch.from_numpy(np.random.default_rng(1).permutation(40).astype(np.int32)[:39].reshape(3, 13)).to(C.dev())
        self.len = d(self.lens, torch.int32)
        self.rope = torch.from_numpy(rope_table(300, HD)).to(C.dev())
        masks = [tree_masks(DRAFTS, b) for b in range(3)]
        self.tree = d([signed(m) for m in masks], torch.int64)
        place = [[n - c + i if i < c else -1 for i in range(DRAFTS)] for n, c in zip(self.lens, self.counts)]
        depth = [[n - c + bin(m & ((1 << c) - 1)).count("1") - 1 if i < c else 0 for i, m in enumerate(ms)]
                 for n, c, ms in zip(self.lens, self.counts, masks)]
        rows = torch.arange(3, device=C.dev()).repeat_interleave(DRAFTS)
        self.slots = api.kv_slots(self.table, rows, d(sum(place, []), torch.int64).clamp(min=0), PAGE)
        self.slots[d(sum(place, []), torch.int64) < 0] = -1
        self.pos = d(sum(depth, []), torch.int64)
        self.n = d(self.counts, torch.int32)
        gen = torch.Generator("cuda").manual_seed(3)
        before = torch.randn(2, 3 * 13 * PAGE, KV, HD, device=C.dev(), generator=gen).to(C.DT[dtype])
        api.uq_kv_write(self.cache, before[0], before[1], torch.arange(3 * 13 * PAGE, device=C.dev()))
        self.fused = torch.zeros(3 * DRAFTS, H + 2 * KV, HD, dtype=C.DT[dtype], device=C.dev())
        self.q = torch.zeros(3, DRAFTS, H, HD, dtype=C.DT[dtype], device=C.dev())
        self.out, self.lse = torch.empty_like(self.q), torch.empty(3, DRAFTS, H, device=C.dev())
        self.ws = api.paged_rows_workspace(H, KV, HD, C.dev())

    def run(self):
        f = self.fused
        api.uq_kv_append(self.cache, f[:, H:H + KV], f[:, H + KV:], self.slots, self.pos, self.rope, q=f[:, :H], q_out=self.q.view(-1, H, HD))
        api.uq_paged_tree_attn(self.cache, self.q, self.tree, self.table, self.len, self.out, counts=self.n, lse=self.lse,
                               window=60, sinks=4, workspace=self.ws)


@pytest.mark.parametrize("fmt", ("bf16", "int8", "int4"))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_replayed_steps_are_the_eager_ones(fmt, dtype):
    base, steps = Step(fmt, dtype), []
    for _ in range(2):
        s, stream, g = Step(fmt, dtype), torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            s.run()
            with torch.cuda.graph(g, stream=stream):
                s.run()
        steps.append((s, stream, g))
    torch.cuda.synchronize()
    last = None
    for i in range(4):
        x = torch.randn(base.fused.shape, device=C.dev(), generator=torch.Generator("cuda").manual_seed(i)).to(C.DT[dtype])
        for s in (base, *(s for s, _, _ in steps)):
            s.fused.copy_(x)
            s.out.fill_(7)
            s.lse.fill_(7)
        base.run()
        torch.cuda.synchronize()
        for s, stream, g in steps:
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        for s, _, _ in steps:
            assert torch.equal(s.out, base.out) and torch.equal(s.lse, base.lse)
            for name in base.cache:
                assert torch.equal(s.cache[name].view(torch.uint8), base.cache[name].view(torch.uint8))
        assert (base.out[0] != 7).all() and (base.out[1, 5:] == 7).all() and (base.out[2, 1:] == 7).all()
        assert last is None or not torch.equal(last, base.out)
        last = base.out.clone()
