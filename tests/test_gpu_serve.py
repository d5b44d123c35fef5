"""The deployed block (serve.BlockDecoder) against the same block in fp64 on
the exported weights, attending over the values that the cache holds.

Those values are checked by themselves: each within half a step of the fp64 key
or value (and what the rounding of a group's minimum and scale to bf16 adds); a key
near the middle of two codes, or a minimum near the middle of two bf16 values, may go
either way, so they are not computed twice.  The rest is fp32 sums: the bounds on
what the block adds to its input leave them a factor of hundreds."""

import numpy as np
import pytest
import torch

import oracle as O
from oracle import kv as OK
from paper_2506_03781_gb300 import api, recon, serve, synth
from tests import kv_cases as C

pytestmark = pytest.mark.gpu
FMT = {"bf16": api.KV_BF16, "int8": api.KV_INT8, "int4": api.KV_INT4}
BOUND = {"bf16": 2e-3, "int8": 2e-3, "int4": 5e-3}


def dense(exported, g):
    planes, a, z = (t.cpu().numpy() for t in exported)
    q, out, words = planes.shape
    bits = (planes.view(np.uint32)[..., None] >> np.arange(32, dtype=np.uint32)) & 1
    c = bits.reshape(q, out, words * 32).astype(np.float64) * 2 - 1
    return sum(c[j] * np.repeat(a[..., j].astype(np.float64), g, 1) for j in range(q)) + np.repeat(z.astype(np.float64), g, 1)


def reference(shape, W, X, fmt, kept):
    """The whole sequence at once, in fp64, on the cache's values of K and V (kept: as kv_cases.cache_rows)."""
    rms = lambda x: x / np.sqrt((x * x).mean(-1, keepdims=True) + shape.eps)
    n, hd = X.shape[0], shape.head_dim
    inv = shape.theta ** (-np.arange(hd // 2) * 2.0 / hd)
    ang = np.arange(n)[:, None, None] * inv
    def rot(x):
        x1, x2 = x[..., :hd // 2], x[..., hd // 2:]
        return np.concatenate([x1 * np.cos(ang) - x2 * np.sin(ang), x1 * np.sin(ang) + x2 * np.cos(ang)], -1)
    h = rms(X)
    q = rot((h @ W["q_proj"].T).reshape(n, shape.heads, hd))
    k = rot((h @ W["k_proj"].T).reshape(n, shape.kv_heads, hd))
    v = (h @ W["v_proj"].T).reshape(n, shape.kv_heads, hd)
    k, v = (held(t, rows, fmt).transpose(1, 0, 2) for t, rows in ((k, kept["k"]), (v, kept["v"])))
    o = np.stack([OK.attend(q[t], k[:, :t + 1], v[:, :t + 1], hd ** -0.5)[0] for t in range(n)])
    X1 = X + o.reshape(n, -1) @ W["o_proj"].T
    h = rms(X1)
    gate = h @ W["gate_proj"].T
    return X1 + (gate / (1 + np.exp(-gate)) * (h @ W["up_proj"].T)) @ W["down_proj"].T


def held(x, rows, fmt):
    """The values of a cache's rows, which have to be x to half a step."""
    val = OK.row_values(rows, fmt)
    _, s, m = rows
    if fmt == "bf16":
        room = 2.0 ** -8 * np.abs(x)
    elif fmt == "int8":
        room = 0.501 * s.astype(np.float64)[..., None]
    else:
        s, m = (np.repeat(t.astype(np.float64), 64, -1) for t in (s, m))
        room = 0.501 * s + 2.0 ** -8 * (np.abs(m) + 15 * s)
    assert (np.abs(val - x) <= room + 1e-5).all()
    return val


@pytest.mark.parametrize("fmt", sorted(FMT))
def test_prompts_and_tokens(fmt):
    shape = synth.BLOCKS["tiny"]
    weights = {n: raw for n, (raw, _) in synth.block_weights(shape, 1).items()}
    block = recon.BlockReconstructor(shape, weights, q=3, g=64, G=4, T=2)
    pool = serve.PagePool(24, shape.kv_heads, shape.head_dim, page_size=16, fmt=FMT[fmt], sequences=4)
    dec = serve.BlockDecoder.of(block, pool)
    W = {n: dense(e, 64) for n, e in dec.exported.items()}
    assert np.abs(W["o_proj"][:4] - O.bcq_gemv(*(t.cpu().numpy().view(np.uint32) if t.dtype == torch.int32 else t.cpu().numpy()
                                                 for t in dec.exported["o_proj"]),
                                               np.eye(W["o_proj"].shape[1], dtype=np.float32), 64).T[:4]).max() < 1e-6
    rng = np.random.default_rng(3)
    lens, new = [70, 1, 15], 20
    X = [rng.standard_normal((n + new, shape.d)).astype(np.float32) for n in lens]
    ids = [pool.open() for _ in lens]
    got = [[dec.prefill(s, torch.from_numpy(x[:n]).cuda())] for s, x, n in zip(ids, X, lens)]
    for t in range(new):
        order = [2, 0, 1] if t % 2 else [0, 1, 2]
        y = dec.decode([ids[b] for b in order], torch.from_numpy(np.stack([X[b][lens[b] + t] for b in order])).cuda())
        for i, b in enumerate(order):
            got[b].append(y[i:i + 1])
    for b, x in enumerate(X):
        y = torch.cat(got[b]).cpu().numpy().astype(np.float64)
        n = pool.length[ids[b]]
        slots = api.kv_slots(pool.table, torch.full((n,), ids[b]).cuda(), torch.arange(n).cuda(), 16).cpu().numpy()
        kept = {name: C.cache_rows(pool.cache, fmt, name, slots) for name in ("k", "v")}
        ref = reference(shape, W, x.astype(np.float64), fmt, kept)
        off = np.linalg.norm(y - ref, axis=1) / np.linalg.norm(ref - x, axis=1)
        assert off.max() <= BOUND[fmt], f"sequence {b}: {off.max():.3g}"
        assert pool.length[ids[b]] == lens[b] + new


def test_pages_come_back():
    pool = serve.PagePool(4, 2, 64, page_size=16, sequences=2)
    a, b = pool.open(), pool.open()
    pool.append([a], [33])
    with pytest.raises(RuntimeError):
        pool.append([b], [17])
    assert pool.length[b] == 0 and len(pool.free) == 1                  # nothing was taken
    with pytest.raises(RuntimeError):
        pool.open()
    pool.close(a)
    slots, pos = pool.append([b], [50])
    assert len(set(slots.tolist())) == 50 and pos.tolist() == list(range(50)) and (pool.table[a] == -1).all()


def test_the_example_runs(capsys):
    serve.main()
    assert capsys.readouterr().out.count("tokens cached") == 3
