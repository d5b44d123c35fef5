"""The deployed block over chunks of prompts, windows with sinks and drafted trees: the same tokens one way and another,
and with a window against the attention's definition on the cache's values.

The cache's rows are the same whichever way a token came, so hidden states differ by fp32 sums alone: by what
tests/test_gpu_serve.py allows against fp64, twice."""

import numpy as np
import pytest
import torch

from paper_2506_03781_gb300 import api, recon, serve, synth

pytestmark = pytest.mark.gpu
FMT = {"bf16": api.KV_BF16, "int8": api.KV_INT8, "int4": api.KV_INT4}
# (a key near the middle of two codes may go either way where sums of its projection differ: 4 bits)
BOUND = {"bf16": 4e-3, "int8": 4e-3, "int4": 1e-2}


@pytest.fixture(scope="module")
def block():
    shape = synth.BLOCKS["tiny"]
    weights = {n: raw for n, (raw, _) in synth.block_weights(shape, 1).items()}
    return recon.BlockReconstructor(shape, weights, q=3, g=64, G=4, T=2)


def decoder(block, fmt, **more):
    pool = serve.PagePool(40, block.shape.kv_heads, block.shape.head_dim, page_size=16, fmt=FMT[fmt], sequences=6)
    return serve.BlockDecoder.of(block, pool, **more)


def same(got, want, X, fmt):
    off = (got - want).norm(dim=-1) / (want - X).norm(dim=-1)
    assert off.max() <= BOUND[fmt], float(off.max())


@pytest.mark.parametrize("fmt", sorted(FMT))
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_chunks_single_tokens_and_one_go(block, fmt, window, sinks):
    dec = decoder(block, fmt, window=window, sinks=sinks)
    gen = torch.Generator("cuda").manual_seed(5)
    X = torch.randn(70, block.shape.d, device="cuda", generator=gen)
    Y = torch.randn(33, block.shape.d, device="cuda", generator=gen)
    a, b, c, e = (dec.pool.open() for _ in range(4))
    whole = dec.prefill(a, X)
    other = dec.prefill(e, Y)
    parts = [dec.extend([b, c], torch.cat([X[:40], Y[:1]]), [40, 1]), dec.extend([c, b], torch.cat([Y[1:], X[40:69]]), [32, 29])]
    last = dec.decode([b], X[69:])
    got = torch.cat([parts[0][:40], parts[1][32:], last])
    same(got, whole, X, fmt)
    same(torch.cat([parts[0][40:], parts[1][:32]]), other, Y, fmt)
    assert [dec.pool.length[s] for s in (a, b, c)] == [70, 70, 33]


@pytest.mark.parametrize("fmt", sorted(FMT))
@pytest.mark.parametrize("window,sinks", [(0, 0), (12, 2)])
def test_drafts_and_what_stays_of_them(block, fmt, window, sinks):
    """A path of the tree gives what its tokens give one after the other, and after it is kept the next token does too."""
    dec = decoder(block, fmt, window=window, sinks=sinks)
    gen = torch.Generator("cuda").manual_seed(6)
    X = torch.randn(30, block.shape.d, device="cuda", generator=gen)
    D = torch.randn(2, 6, block.shape.d, device="cuda", generator=gen)
    Z = torch.randn(1, block.shape.d, device="cuda", generator=gen)
    parents = [[-1, 0, 0, 2, 1, 3], [-1, -1, 1, 2, 3, 4]]
    a, b, c = (dec.pool.open() for _ in range(3))
    for s in (a, b, c):
        dec.prefill(s, X)
    got = dec.verify([a, c], D, parents)
    path = [0, 2, 3, 5]
    steps = torch.cat([dec.decode([b], D[0, i:i + 1]) for i in path])
    same(got[0, path], steps, D[0, path], fmt)
    dec.pool.keep(a, 6, path)
    assert dec.pool.length[a] == dec.pool.length[b] == 34 and len(dec.pool.owned[a]) == 3
    same(dec.decode([a], Z), dec.decode([b], Z), Z, fmt)
    dec.pool.keep(c, 6, [])
    assert dec.pool.length[c] == 30


def test_the_window_is_the_definitions(block):
    """Tokens that a window hides do not matter: other ones in their place change nothing."""
    dec = decoder(block, "bf16", window=16, sinks=4)
    gen = torch.Generator("cuda").manual_seed(7)
    X = torch.randn(60, block.shape.d, device="cuda", generator=gen)
    Y = X.clone()
    Y[10:30] = torch.randn(20, block.shape.d, device="cuda", generator=gen)
    a, b = dec.pool.open(), dec.pool.open()
    x, y = dec.prefill(a, X), dec.prefill(b, Y)
    assert torch.equal(x[46:], y[46:]) and torch.equal(x[:10], y[:10]) and not torch.equal(x[30:46], y[30:46])
    z = torch.randn(1, block.shape.d, device="cuda", generator=gen)
    assert torch.equal(dec.decode([a], z), dec.decode([b], z))
