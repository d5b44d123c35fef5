"""Oracle of the paged key-value cache and of the attention over it.

Written from the definitions: the rows' codes and scales are decided in IEEE
fp32 with the stated operation order (they decide integers and what is kept in
few bits), values, scores and sums are fp64.  The cache here is a plain list
of rows; pages only say which row a position is."""

from __future__ import annotations

import numpy as np

F32, F64 = np.float32, np.float64
TINY = F32(2.0 ** -100)
GROUP = 64
FORMATS = ("bf16", "int8", "int4")


def to_bf16(x):
    """fp32 -> bf16 -> fp32, nearest even; infinities and NaN kept."""
    x = np.ascontiguousarray(x, F32)
    b = x.view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint32) << 16
    y = r.astype(np.uint32).view(F32)
    return np.where(np.isfinite(x), y, x).astype(F32)


def quantise_rows(x, fmt):
    """x [..., hd] fp32 -> (codes or bf16 values, scales, minima) as the cache keeps them.

    int8: scales [...]; int4: scales, minima [..., hd / 64]."""
    x = np.asarray(x, F32)
    with np.errstate(all="ignore"):
        if fmt == "bf16":
            return to_bf16(x), None, None
        if fmt == "int8":
            a = np.abs(x).max(-1)                              # NaN stays
            fine, some = np.isfinite(a), np.isfinite(a) & (a >= TINY)
            inv = np.where(some, F32(127) / a, F32(0)).astype(F32)
            c = np.rint((x * inv[..., None]).astype(F32))
            c = np.where(some[..., None], c, 0).astype(np.int8)
            scale = np.where(some, (a / F32(127)).astype(F32), np.where(fine, F32(0), F32(np.nan))).astype(F32)
            return c, scale, None
        g = x.reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
        lo, hi = g.min(-1), g.max(-1)
        s, m = to_bf16(((hi - lo).astype(F32) / F32(15)).astype(F32)), to_bf16(lo)
        fine = np.isfinite(s) & np.isfinite(m)
        some = fine & (s >= TINY)
        inv = np.where(some, F32(1) / s, F32(0)).astype(F32)
        c = np.rint(((g - m[..., None]).astype(F32) * inv[..., None]).astype(F32))
        c = np.where(some[..., None], np.clip(c, 0, 15), 0).astype(np.uint8).reshape(x.shape)
        nan = F32(np.nan)
        return c, np.where(some, s, np.where(fine, F32(0), nan)).astype(F32), np.where(fine, m, nan).astype(F32)


def row_values(kept, fmt):
    """fp64 values of what quantise_rows returned."""
    c, s, m = kept
    if fmt == "bf16":
        return np.asarray(c, F64)
    if fmt == "int8":
        return np.asarray(c, F64) * np.asarray(s, F64)[..., None]
    g = np.asarray(c, F64).reshape(*c.shape[:-1], c.shape[-1] // GROUP, GROUP)
    return (g * np.asarray(s, F64)[..., None] + np.asarray(m, F64)[..., None]).reshape(c.shape)


def attend(q, k, v, scale):
    """q [heads, hd]; k, v [kv, n, hd] fp64 values of the n positions that count -> (out [heads, hd], lse [heads])."""
    q, k, v = (np.asarray(t, F64) for t in (q, k, v))
    H, kv, n = q.shape[0], k.shape[0], k.shape[1]
    if n == 0:
        return np.zeros_like(q), np.full(H, -np.inf)
    x = np.einsum("grd,gnd->grn", q.reshape(kv, H // kv, -1), k) * scale
    m = x.max(-1, keepdims=True)
    p = np.exp(x - m)
    l = p.sum(-1, keepdims=True)
    return (np.einsum("grn,gnd->grd", p, v) / l).reshape(q.shape), (np.log(l) + m).reshape(H)


def attend_mass(q, k, v, scale):
    """What rounding errors of an attention are measured in: (sum_t p_t |v_t|, the largest sum_d |scale q_d k_td|),
    shapes [heads, hd] and [heads]."""
    q, k, v = (np.asarray(t, F64) for t in (q, k, v))
    H, kv, n = q.shape[0], k.shape[0], k.shape[1]
    if n == 0:
        return np.zeros_like(q), np.zeros(H)
    out, _ = attend(q, k, np.abs(v), scale)
    reach = np.einsum("grd,gnd->grn", np.abs(q).reshape(kv, H // kv, -1), np.abs(k)).max(-1) * abs(scale)
    return out, reach.reshape(H)


def rotate(x, rope, positions, rotated):
    """x [n, heads, hd] fp32, channels (j, j + rotated / 2) turned by rope[position, j] = (c, s), every product, sum and
    difference in fp32; NaN where rope has no such position."""
    x = np.asarray(x, F32)
    half = rotated // 2
    there = (positions >= 0) & (positions < len(rope))
    cs = np.where(there[:, None, None], rope[np.where(there, positions, 0)][:, :half], F32(np.nan)).astype(F32)[:, None]
    c, s = cs[..., 0], cs[..., 1]
    a, b = x[..., :half], x[..., half:rotated]
    with np.errstate(invalid="ignore"):
        return np.concatenate([(a * c).astype(F32) - (b * s).astype(F32), (a * s).astype(F32) + (b * c).astype(F32),
                               x[..., rotated:]], -1).astype(F32)


def window_sees(p, t, window, sinks):
    """Whether position t is in the window of position p, or a sink."""
    return (t > p - window) | (t < sinks) if window else np.ones(np.broadcast_shapes(np.shape(p), np.shape(t)), bool)


def prompt_sees(n, new, window=0, sinks=0):
    """[new, n]: what the last `new` of n tokens see."""
    p, t = np.arange(n - new, n)[:, None], np.arange(n)[None]
    return (t <= p) & window_sees(p, t, window, sinks)


def tree_sees(n, masks, window=0, sinks=0):
    """[drafts, n]: what the drafts, the last of n tokens, see; masks: their ancestors' bits (Python integers)."""
    c = len(masks)
    kin = np.array([[(m >> j) & 1 for j in range(c)] for m in masks], bool).reshape(c, c)
    ctx = n - c
    p = ctx + kin.sum(1) - 1
    t = np.concatenate([np.arange(max(ctx, 0)), p[max(0, -ctx):]])          # positions of the places
    sees = np.concatenate([np.ones((c, max(ctx, 0)), bool), kin[:, max(0, -ctx):]], 1)
    return sees & window_sees(p[:, None], t[None], window, sinks)
