"""uq_paged_prompt_attn, uq_paged_tree_attn and uq_paged_attn_sinks on the GPU against the oracle in 64 bits.  Every
cache's unused places hold NaN and every unused table entry an invalid page."""

import numpy as np
import pytest
import torch

from oracle import kv as OK
from paper_2506_03781_gb300 import api
from tests import kv_cases as C
from tests.rows_cases import Rows, signed

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "int8", "int4")
TYPES = ("bf16", "f32")


# --- one new token, sinks

class Sinks(C.Case):
    def check(self, window, sinks):
        H = self.kv * self.r
        ws = api.paged_attn_workspace(H, self.kv, self.hd, C.dev()).fill_(255)
        scale = self.hd ** -0.5
        api.uq_paged_attn_sinks(self.cache, self.q, self.tab, self.len, self.out, lse=self.lse, scale=scale, window=window,
                                sinks=sinks, workspace=ws)
        torch.cuda.synchronize()
        out, lse = self.out.float().cpu().numpy(), self.lse.cpu().numpy()
        for b, n in enumerate(self.lens):
            t = np.arange(n)
            pos = t[OK.window_sees(n - 1, t, window, sinks)]
            K, V = self.K[b][:, pos], self.V[b][:, pos]
            ref, ref_lse = OK.attend(self.qv[b], K, V, scale)
            if n == 0:
                assert np.array_equal(out[b], ref) and np.array_equal(lse[b], ref_lse)
                continue
            tol, tol_lse = C.tolerance(self.qv[b], K, V, scale, ref, ref_lse, self.dtype)
            assert (np.abs(out[b] - ref) <= tol).all() and (np.abs(lse[b] - ref_lse) <= tol_lse).all(), f"sequence {b} of {n}"


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd,kv,r,page", [(64, 2, 5, 16), (128, 2, 4, 64), (256, 1, 12, 32)])
@pytest.mark.parametrize("window,sinks", [(1, 1), (17, 4), (100, 33), (100, 0), (64, 64), (300, 2 ** 40), (0, 9), (2 ** 40, 3)])
def test_one_token_with_sinks(fmt, dtype, hd, kv, r, page, window, sinks):
    Sinks(fmt, dtype, hd, kv, r, page, [1, 0, 15, 64, 65, 97, 101, 130, 300, 1000], seed=window % 97 + sinks % 89).check(window, sinks)


@pytest.mark.parametrize("fmt", FORMATS)
def test_one_token_of_long_sequences_with_sinks(fmt):
    Sinks(fmt, "bf16", 128, 2, 4, 64, [70001, 3, 4100, 20000], seed=3).check(4096, 4)


@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_between_sinks_and_window_are_not_read(fmt):
    """The table's entries between them are invalid, and no page that is gone hides another's positions."""
    c = Sinks(fmt, "f32", 64, 2, 3, 16, [400, 90], seed=5)
    c.tab[0, 1:18] = 2 ** 31 - 1                     # the window of 100 begins in page 18
    c.check(100, 7)


# --- prompts

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd,kv,r,page", [(64, 2, 4, 16), (128, 2, 4, 32), (256, 1, 2, 128), (128, 1, 7, 16), (64, 1, 16, 64),
                                          (128, 3, 1, 16), (64, 1, 37, 256)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 4)])
def test_prompts(fmt, dtype, hd, kv, r, page, window, sinks):
    Rows(fmt, dtype, hd, kv, r, page, [1, 0, 130, 64, 257, 300, 17, 400], [1, 0, 130, 33, 1, 65, 0, 7], seed=kv + r).check(
        window=window, sinks=sinks, every=3)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,new", [(1, 1), (2000, 1), (3000, 700), (5000, 40)])
def test_single_prompts(fmt, dtype, n, new):
    """One sequence: little work that is cut over the GPU, or a triangle of it."""
    for window, sinks in ((0, 0), (129, 64), (1000, 4)):
        Rows(fmt, dtype, 128, 2, 4, 64, [n], [new], seed=n).check(window=window, sinks=sinks, every=max(1, new // 11))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 3), (127, 130), (128, 128), (129, 1), (2 ** 40, 5), (300, 2 ** 40)])
def test_windows_of_prompts(fmt, window, sinks):
    Rows(fmt, "f32", 64, 2, 5, 16, [500, 130, 1, 777], [260, 130, 1, 3], seed=window % 97).check(window=window, sinks=sinks, every=13)


def test_many_prompts():
    """Hundreds of sequences with few new tokens each, some with none."""
    lens = [(i * 37) % 300 for i in range(400)]
    Rows("int8", "bf16", 64, 1, 4, 16, lens, [min(n, i % 7) for i, n in enumerate(lens)], seed=2).check(every=2)


@pytest.mark.parametrize("fmt", FORMATS)
def test_large_and_small_scores(fmt):
    for scale in (30.0, 0.0, -0.3, 1e-6):
        Rows(fmt, "bf16", 128, 2, 4, 16, [300, 40], [200, 40], seed=8).check(scale=scale, every=17)


@pytest.mark.parametrize("fmt", ("int8", "int4"))
@pytest.mark.parametrize("dtype", TYPES)
def test_value_scales_of_all_sizes(fmt, dtype):
    for s in (1e-20, 1e20):
        Rows(fmt, dtype, 128, 2, 4, 16, [200, 3], [70, 3], seed=9, scale_v=s).check(every=5)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("trees", (False, True))
def test_pages_that_are_not_there(fmt, trees):
    r = Rows(fmt, "f32", 64, 2, 4, 32, [300, 64, 96], [40, 30, 5], trees=trees, seed=2)
    hidden = {0: np.r_[32:64, 288:300], 1: np.arange(64)}
    for b, p, e in ((0, 1, -1), (0, 9, 2 ** 31 - 1), (1, 0, -2 ** 31), (1, 1, r.c.pages)):
        r.c.tab[b, p] = e
    r.check(hidden=hidden)


@pytest.mark.parametrize("trees", (False, True))
def test_lengths_beyond_the_table_below_zero_and_below_the_new(trees):
    """Longer than the table: as long as it; shorter than what is new: the first ones have no place and see nothing."""
    r = Rows("bf16", "f32", 64, 1, 2, 16, [64, 10, 30], [20, 10, 30], trees=trees, seed=4)
    r.c.len.copy_(torch.tensor([10 ** 9, -5, 12]))
    out, lse = r.run()
    out, lse = out.cpu().numpy(), lse.cpu().numpy()
    for b, n in ((0, 64), (1, 0), (2, 12)):
        k = r.new[b]
        for i in range(k):
            if trees:
                d = [j for j in range(k) if r.masks[b][i] >> j & 1 and n - k + j >= 0]
                pos = list(range(max(0, n - k))) + [n - k + j for j in d]
            else:
                pos = list(range(max(0, n - k + i + 1)))
            ref, ref_lse = OK.attend(r.qv[r.at(b, i)], r.c.K[b][:, pos], r.c.V[b][:, pos], 64 ** -0.5)
            assert np.abs(out[r.at(b, i)] - ref).max() < 1e-5, (b, i)
            assert np.array_equal(np.isinf(lse[r.at(b, i)]), np.isinf(ref_lse))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("value", (float("nan"), float("inf"), -float("inf")))
def test_what_a_token_does_not_see_does_not_reach_it(dtype, value):
    """Rows of later tokens, of tokens before the window and of other branches are no numbers: only who sees them has it.
    The others' results may be computed another way then: both are within (2^-8 + 2^-8) of sum p |v| <= max |v| of the
    exact ones in bf16 (rows_cases.tolerance), fp32 within 4e-6 of it."""
    n, new = 400, 200
    for trees, window, sinks in ((False, 0, 0), (False, 90, 3), (True, 0, 0)):
        k = 50 if trees else new
        r = Rows("bf16", dtype, 64, 1, 4, 16, [n], [k], trees=trees, seed=6)
        clean, _ = r.run(window=window, sinks=sinks)
        clean = clean.clone()
        bad = np.array([n - 1, n - k // 2, n - k + 1, n - k + 11])      # all of them new
        for t in bad:
            page, off = int(r.c.table[0, t // 16]), t % 16
            r.c.cache["v"][page, 0, off, (t % 3)::5] = value
            if t % 2:
                r.c.cache["k"][page, 0, off, t % 7] = value
        out, _ = r.run(window=window, sinks=sinks)
        sees = r.sees(0, window, sinks)[:, bad].any(1)
        assert sees.any() and not sees.all()
        for i in range(k):
            got, want = out[r.at(0, i)].float(), clean[r.at(0, i)].float()
            if not sees[i]:
                assert (got - want).abs().max() <= 2 * (2.0 ** -7 if dtype == "bf16" else 4e-6) * np.abs(r.c.V[0]).max(), i
            else:
                assert not torch.isfinite(got).all(), i


# --- trees

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("hd,kv,r,page", [(64, 2, 4, 16), (128, 2, 4, 32), (256, 1, 2, 128), (128, 1, 7, 16), (64, 1, 16, 64), (128, 3, 1, 16)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (33, 4)])
def test_trees(fmt, dtype, hd, kv, r, page, window, sinks):
    Rows(fmt, dtype, hd, kv, r, page, [64, 0, 130, 65, 257, 300, 17, 1000], [64, 0, 13, 64, 1, 33, 0, 60], trees=True,
         seed=kv + r).check(window=window, sinks=sinks, every=2)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", TYPES)
def test_one_tree_of_a_long_sequence(fmt, dtype):
    Rows(fmt, dtype, 128, 2, 4, 64, [20011], [16], trees=True, seed=1).check()
    Rows(fmt, dtype, 128, 2, 4, 64, [20011, 9000], [16, 5], trees=True, most=20, seed=1).check(window=5000, sinks=4)


@pytest.mark.parametrize("fmt", FORMATS)
def test_long_trees_of_few_rows_between_large_ones(fmt):
    """One tile of rows of a block has no part in the trees of 32 rows, for dozens of tiles of positions, and then in those
    of 240."""
    Rows(fmt, "bf16", 64, 4, 4, 64, [4000 + 37 * i for i in range(24)], [8 if i % 2 else 60 for i in range(24)], trees=True, seed=4).check(every=13)


def test_masks_of_all_kinds():
    """A chain, all apart, bits of drafts behind the last one, of later drafts, and a draft that does not see itself."""
    r = Rows("int8", "f32", 64, 1, 2, 16, [100, 100, 100], [10, 10, 10], trees=True, most=12, seed=3)
    r.masks[0] = [(2 << i) - 1 for i in range(12)]
    r.masks[1] = [1 << i for i in range(12)]
    r.masks[2] = [0, 2, 1 << 9 | 4, 15, 0x3ff, 16, 32, 64, 128, 256, 0, 0]
    r.tree.copy_(torch.tensor([signed([m | (1 << 63) | (3 << 10) for m in ms]) for ms in r.masks]))
    for window, sinks in ((0, 0), (5, 2)):
        r.check(window=window, sinks=sinks)


def test_a_chain_is_a_prompt():
    for fmt in FORMATS:
        t = Rows(fmt, "f32", 128, 2, 4, 16, [90, 300], [30, 30], trees=True, seed=7)
        t.masks = [[(2 << i) - 1 for i in range(30)]] * 2
        t.tree.copy_(torch.tensor([signed(m) for m in t.masks]))
        p = Rows(fmt, "f32", 128, 2, 4, 16, [90, 300], [30, 30], seed=7)
        p.q[:60] = t.q.view(60, 8, 128)
        for window, sinks in ((0, 0), (50, 4)):
            a, _ = t.run(window=window, sinks=sinks)
            b, _ = p.run(window=window, sinks=sinks)
            assert (a.view(60, 8, 128) - b[:60]).abs().max() < 1e-5


def test_counts_left_out_and_beyond():
    r = Rows("bf16", "bf16", 64, 1, 4, 16, [100, 40], [9, 9], trees=True, seed=5).check()
    want = r.out.clone()
    for counts in (None, torch.tensor([9, 2 ** 31 - 1], dtype=torch.int32, device=C.dev())):
        r.out.fill_(7)
        api.uq_paged_tree_attn(r.c.cache, r.q, r.tree, r.c.tab, r.c.len, r.out, counts=counts)
        assert torch.equal(r.out, want)
    r.counts = torch.tensor([-3, 0], dtype=torch.int32, device=C.dev())
    r.out.fill_(7)
    assert (r.run()[0] == 7).all()


# --- strides, streams, repeats

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("trees", (False, True))
def test_strides(dtype, trees):
    r = Rows("int8", dtype, 128, 2, 4, 16, [5, 130, 77], [5, 40, 9], trees=trees, seed=6)
    shape = r.q.shape[:-2]
    fused = torch.zeros(*shape, 12, 128, dtype=C.DT[dtype], device=C.dev())
    fused[..., :8, :] = r.q
    r.q = fused[..., :8, :]
    room = torch.full((8, *shape, 128), 7.0, dtype=C.DT[dtype], device=C.dev())
    r.out = room.movedim(0, -2)
    wide = torch.full((3, 20), 2 ** 31 - 1, dtype=torch.int32, device=C.dev())
    wide[:, 3:3 + r.c.tab.shape[1]] = r.c.tab
    r.c.tab = wide[:, 3:3 + r.c.tab.shape[1]]
    if trees:
        far = torch.zeros(3, 70, dtype=torch.int64, device=C.dev())
        far[:, 5:5 + r.most] = r.tree
        r.tree = far[:, 5:5 + r.most]
    r.check()


@pytest.mark.parametrize("trees", (False, True))
@pytest.mark.parametrize("dtype", TYPES)
def test_repeats_are_equal_whatever_the_workspace_holds(trees, dtype):
    r = Rows("int4", dtype, 128, 2, 4, 16, [3000, 17, 900, 0, 4001], [60, 17, 1, 0, 33], trees=trees, seed=1)
    ws = api.paged_rows_workspace(8, 2, 128, C.dev())
    first = None
    for fill in (255, 0, 1, None, None, 127):
        if fill is not None:
            ws.fill_(fill)
        out, lse = r.run(workspace=ws)
        if first is None:
            first = out.clone(), lse.clone()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
        r.out.fill_(7)
    r.lse = None                                      # not wanted; a workspace of the call's own
    assert torch.equal(r.run(workspace=None)[0], first[0])


def test_streams_and_graphs():
    """A verification step (append, attend over the tree) replayed from two graphs with a workspace each on two streams."""
    rng = np.random.default_rng(0)
    base = Rows("int8", "bf16", 128, 2, 4, 16, [40, 333], [8, 5], trees=True, seed=3)
    steps = []
    for s in range(2):
        r = Rows("int8", "bf16", 128, 2, 4, 16, [40, 333], [8, 5], trees=True, seed=3)
        stream = torch.cuda.Stream()
        ws = api.paged_rows_workspace(8, 2, 128, C.dev())
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            r.run(workspace=ws)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                api.uq_paged_tree_attn(r.c.cache, r.q, r.tree, r.c.tab, r.c.len, r.out, counts=r.counts, lse=r.lse, workspace=ws)
        steps.append((r, stream, g, ws))
    torch.cuda.synchronize()
    for _ in range(3):
        q = torch.from_numpy(rng.standard_normal(tuple(base.q.shape)).astype(np.float32)).to(C.dev()).to(torch.bfloat16)
        base.q.copy_(q)
        want, _ = base.run()
        for r, _, _, _ in steps:
            r.q.copy_(q)
            r.out.fill_(7)
        torch.cuda.synchronize()
        for r, stream, g, _ in steps:
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        for r, _, _, _ in steps:
            assert torch.equal(r.out, want)


def test_nothing_to_do():
    c = C.Case("int8", "bf16", 64, 1, 2, 16, [20], seed=1)
    q = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=C.dev())
    api.uq_paged_prompt_attn(c.cache, q, torch.zeros(2, dtype=torch.int32, device=C.dev()), c.tab, c.len, q.clone())
    q = torch.zeros(1, 0, 2, 64, dtype=torch.bfloat16, device=C.dev())
    api.uq_paged_tree_attn(c.cache, q, torch.zeros(1, 0, dtype=torch.int64, device=C.dev()), c.tab, c.len, q.clone())
    q = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device=C.dev())
    api.uq_paged_attn_sinks(c.cache, q, c.tab[:0], c.len[:0], q.clone(), window=3, sinks=1)
