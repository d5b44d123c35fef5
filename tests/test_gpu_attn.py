"""uq_paged_attn on the GPU against the oracle in 64 bits, within tolerances
derived from its arithmetic (kv_cases.tolerance).  Every cache's unused places
hold NaN and every unused table entry an invalid page."""

import numpy as np
import pytest
import torch

from paper_2506_03781_gb300 import api
from tests import kv_cases as C

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "int8", "int4")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hd", (64, 128, 256))
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("kv,r,page", [(1, 1, 16), (2, 4, 32), (8, 8, 16), (3, 3, 64), (1, 16, 256), (2, 12, 128),
                                       (1, 37, 16)])
def test_lengths(fmt, hd, dtype, kv, r, page):
    C.Case(fmt, dtype, hd, kv, r, page, [1, 0, 2, 15, 16, 17, 31, 64, 65, 127, 300, 1023], seed=kv + r).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("lens", [[1], [0], [0, 0, 0], [70001], [5000, 3], [1] * 300, [129] * 77, [40000, 0, 1, 20000, 6]])
def test_shares_of_the_work(fmt, dtype, lens):
    """One long sequence cut over the whole GPU, many short ones, very different ones."""
    C.Case(fmt, dtype, 128, 2, 4, 16 if max(lens) < 50000 else 64, lens, seed=len(lens)).check()


@pytest.mark.parametrize("fmt,dtype,hd,kv,r", [("int8", "bf16", 128, 1, 1), ("bf16", "f32", 64, 1, 9),
                                               ("int4", "bf16", 256, 1, 2), ("int4", "f32", 128, 2, 3)])
def test_many_sequences(fmt, dtype, hd, kv, r):
    """Thousands of them: every lane of the search has many; with and without long ones among them."""
    C.Case(fmt, dtype, hd, kv, r, 16, [i % 5 for i in range(2500)], seed=r).check()
    C.Case(fmt, dtype, hd, kv, r, 16, [(7000 if i % 900 == 450 else i % 40) for i in range(1900)], seed=r).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("window", [1, 2, 15, 16, 17, 100, 129, 4096, 2 ** 40])
def test_windows(fmt, window):
    C.Case(fmt, "f32", 64, 2, 5, 16, [1, 0, 16, 100, 101, 300, 1000], seed=window % 97).check(window=window)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_pages_that_are_not_there(fmt, dtype):
    """Table entries in use that are negative or beyond the pool hide their positions; a sequence whose pages are all
    hidden is empty."""
    c = C.Case(fmt, dtype, 128, 2, 4, 32, [300, 64, 96, 33], seed=2)
    hidden = {0: np.r_[32:64, 96:128, 288:300], 1: np.arange(64), 3: np.arange(32, 33)}
    for b, p, e in ((0, 1, -1), (0, 3, c.pages), (0, 9, 2 ** 31 - 1), (1, 0, -2 ** 31), (1, 1, -7), (3, 1, c.pages + 9)):
        c.tab[b, p] = e
    c.check(hidden=hidden)


@pytest.mark.parametrize("fmt", FORMATS)
def test_lengths_beyond_the_table_and_below_zero(fmt):
    c = C.Case(fmt, "f32", 64, 1, 2, 16, [64, 64, 10], seed=4)
    c.len.copy_(torch.tensor([10 ** 9, 2 ** 31 - 1, -5]))
    c.lens[2], c.K[2], c.V[2] = 0, c.K[2][:, :0], c.V[2][:, :0]
    c.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_scales_and_large_scores(fmt, dtype):
    """Scores of hundreds (one position takes all the weight), none at all, and a negative scale."""
    for scale in (30.0, 0.0, -0.3, 1e-6):
        C.Case(fmt, dtype, 128, 2, 4, 16, [1, 50, 700], seed=8).check(scale=scale)


@pytest.mark.parametrize("fmt", ("int8", "int4"))
def test_value_scales_of_all_sizes(fmt):
    for s in (1e-20, 1e20):
        C.Case(fmt, "f32", 128, 2, 4, 16, [200, 3], seed=9, scale_v=s).check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_strides(dtype):
    """Queries from a fused projection, a slice of a wider table, results into a wider tensor."""
    c = C.Case("int8", dtype, 128, 2, 4, 16, [5, 130, 77], seed=6)
    fused = torch.zeros(3, 12, 128, dtype=C.DT[dtype], device=C.dev())
    fused[:, :8] = c.q
    c.q = fused[:, :8]
    wide = torch.full((3, 20), 2 ** 31 - 1, dtype=torch.int32, device=C.dev())
    wide[:, 3:3 + c.tab.shape[1]] = c.tab
    c.tab = wide[:, 3:3 + c.tab.shape[1]]
    room = torch.full((8, 5, 128), 3.0, dtype=C.DT[dtype], device=C.dev())
    c.out = room[:, 1:4].transpose(0, 1)
    c.check()
    assert (room[:, 0] == 3).all() and (room[:, 4] == 3).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_repeats_are_equal_whatever_the_workspace_holds(fmt):
    c = C.Case(fmt, "f32", 128, 2, 4, 16, [3000, 17, 900, 0, 4001], seed=1)
    ws = api.paged_attn_workspace(8, 2, 128, C.dev())
    first = None
    for fill in (255, 0, 1, None, None, 127):
        if fill is not None:
            ws.fill_(fill)
        c.out.fill_(float("nan"))
        c.lse.fill_(float("nan"))
        out, lse = c.run(workspace=ws)
        if first is None:
            first = out.clone(), lse.clone()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    api.uq_paged_attn(c.cache, c.q, c.tab, c.len, c.out, lse=None)          # no lse, a workspace of its own
    assert torch.equal(c.out, first[0])


def test_streams_and_graphs():
    """A decode step (write, then attend) on a stream of its own and replayed from a graph: the replay sees new tokens."""
    c = C.Case("int8", "bf16", 128, 2, 4, 16, [40, 33, 1000], seed=3)
    n = torch.tensor([c.lens]).T - 1
    table = c.tab.long().cpu()
    slots = (table.gather(1, n // 16) * 16 + n % 16)[:, 0].to(C.dev())
    ws = api.paged_attn_workspace(8, 2, 128, C.dev())
    k, v = (torch.randn(3, 2, 128, device=C.dev()).bfloat16() for _ in range(2))
    k2, v2 = k.flip(0).contiguous(), v.flip(1).contiguous()

    def step(stream=None):
        api.uq_kv_write(c.cache, k, v, slots, stream=stream)
        api.uq_paged_attn(c.cache, c.q, c.tab, c.len, c.out, lse=c.lse, workspace=ws, stream=stream)

    step()
    torch.cuda.synchronize()
    want = c.out.clone()
    c.out.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    api.uq_paged_attn(c.cache, c.q, c.tab, c.len, c.out, stream=side)       # a workspace taken on that stream
    side.synchronize()
    assert torch.equal(c.out, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for kk, vv in ((k2, v2), (k.clone(), v.clone())):
        k.copy_(kk)
        v.copy_(vv)
        g.replay()
        g.replay()
        torch.cuda.synchronize()
        got = c.out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, c.out)
    assert torch.equal(got, want)


@pytest.mark.parametrize("fmt", FORMATS)
def test_pools_beyond_32_bit_offsets(fmt):
    """The pages of the sequences are the last ones of a pool of more than 2^32 bytes."""
    c = C.Case(fmt, "f32", 256, 8, 2, 256, [300, 500], seed=5, spare=0)
    row = c.cache["k"][0].numel() * c.cache["k"].element_size()
    more = 2 ** 32 // row + 1
    for name, t in list(c.cache.items()):
        big = torch.empty(more + t.shape[0], *t.shape[1:], dtype=t.dtype, device=t.device)
        big.view(torch.uint8).fill_(255)
        big[more:] = t
        c.cache[name] = big
    need = [-(-n // 256) for n in c.lens]
    for b, n in enumerate(need):
        c.tab[b, :n] += more
    for b, n in enumerate(need):
        c.tab[b, n:] = -1
    c.check()


def test_not_finite_inputs_stay_in_their_sequence():
    """A NaN or an infinity in a sequence's values or queries shows in that sequence and nowhere else."""
    for fmt in FORMATS:
        c = C.Case(fmt, "f32", 64, 1, 2, 16, [40, 40, 40], seed=7)
        name = "k" if fmt == "bf16" else "v_scale"
        c.cache[name][int(c.table[1, 1]), 0, 2] = float("nan")     # position 18 of sequence 1
        out, lse = c.run()
        assert torch.isnan(out[1]).all() if fmt == "bf16" else torch.isnan(out[1]).any()
        c.lens[1], c.K[1], c.V[1] = 40, c.K[0], c.V[0]
        c.tab[1] = c.tab[0]
        c.qv[1] = c.qv[0]
        c.q[1] = c.q[0]
        c.check()
        c.q[2, 0, 3] = float("nan")
        out, lse = c.run()
        assert torch.isnan(out[2, 0]).all() and torch.isnan(lse[2, 0]) and torch.isfinite(out[:2]).all()
        assert torch.isfinite(out[2, 1]).all()


def test_refusals():
    d = C.dev()
    c = C.Case("int4", "bf16", 64, 2, 2, 16, [20, 3])
    ws = api.paged_attn_workspace(4, 2, 64, d)
    call = lambda **m: api.uq_paged_attn(**{**dict(cache=c.cache, q=c.q, block_table=c.tab, seq_lens=c.len, out=c.out,
                                                   lse=c.lse, workspace=ws), **m})
    call()
    for more, match in ((dict(q=c.q[:1]), "out has shape"), (dict(out=c.out.float()), "out has dtype"),
                        (dict(block_table=c.tab.long()), "block_table"), (dict(block_table=c.tab[:1]), "block_table"),
                        (dict(block_table=c.tab.T.contiguous().T), "block_table"),
                        (dict(seq_lens=c.len[:1]), "seq_lens"), (dict(seq_lens=c.len.long()), "seq_lens"),
                        (dict(lse=c.lse[:, :1]), "lse"), (dict(lse=c.lse.double()), "lse"),
                        (dict(q=c.q.half(), out=c.out.half()), "float32 or bfloat16"),
                        (dict(workspace=ws.cpu()), "workspace")):
        with pytest.raises(ValueError, match=match):
            call(**more)
    for more, status in ((dict(window=-1), api.UQ_ERR_ARG), (dict(scale=float("nan")), api.UQ_ERR_ARG),
                         (dict(scale=float("inf")), api.UQ_ERR_ARG), (dict(workspace=ws[:-1]), api.UQ_ERR_ARG),
                         (dict(workspace=ws[8:]), api.UQ_ERR_ALIGN)):
        with pytest.raises(api.UQError) as e:
            call(**more)
        assert e.value.status == status
    q3 = torch.zeros(2, 3, 64, dtype=torch.bfloat16, device=d)
    with pytest.raises(api.UQError) as e:                              # heads that the key/value heads do not divide
        call(q=q3, out=q3.clone(), lse=None)
    assert e.value.status == api.UQ_ERR_ARG
    with pytest.raises(ValueError):
        api.paged_attn_workspace(3, 2, 64, d)
    none = torch.empty(0, 4, 64, dtype=torch.bfloat16, device=d)
    call(q=none, out=none.clone(), lse=None, block_table=c.tab[:0], seq_lens=c.len[:0])
    torch.cuda.synchronize()
