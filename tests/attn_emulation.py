"""The arithmetic of the attention for fp32 queries, restated on the CPU, with
its terms as parameters: what an error bound has to let through, and what it
must not.

A product of 16 channels (positions) on the tensor cores is added to its fp32
accumulator and cut off to 24 bits; everything else is fp32, rounded to
nearest.  One chain of positions, as one warp adds them, with the maximum
known beforehand."""

from __future__ import annotations

import numpy as np

from oracle import kv as OK

F32, F64 = np.float32, np.float64

# How far fp32 results may be off, in units of sum_t p_t |v_t| (kv_cases has the
# worst case, whose sums of rounding errors grow with the positions; these inputs have
# scores of order 1, and errors of either sign).  By the emulation the full
# arithmetic stays below 1.2e-6, and an exponential that is off by 2^-22 adds 2.4e-7
# to a weight; a dropped term costs 6.5e-6 and more (test_attn_accuracy_cpu.py).
FP32_BOUND = 4e-6


def _cut(x):
    """fp64 -> fp32, toward zero."""
    y = x.astype(F32)
    return np.where(np.abs(y.astype(F64)) > np.abs(x), np.nextafter(y, F32(0)), y)


def _bf16_terms(x, n):
    parts, rest = [], np.ascontiguousarray(x, F32)
    for _ in range(n - 1):
        parts.append((rest.view(np.uint32) & np.uint32(0xFFFF0000)).view(F32))
        rest = rest - parts[-1]
    return parts + [OK.to_bf16(rest)]


def _fp16_terms(x, n):
    parts, rest = [], np.asarray(x, F32)
    for _ in range(n):
        parts.append(rest.astype(np.float16).astype(F32))
        rest = rest - parts[-1]
    return parts


def attend_fp32(q, kept_k, kept_v, fmt, scale, query_terms=None, weight_terms=3, fp32_sums=True):
    """q [r, hd] fp32; kept_k, kept_v: oracle.kv.quantise_rows of [n, hd] -> out [r, hd]."""
    n, hd = kept_k[0].shape
    k, v = kept_k[0].astype(F64), kept_v[0].astype(F64)
    if fmt == "bf16":
        terms, per, weight = _bf16_terms(q, query_terms or 3), F32(1), F32(1)
    else:
        exponent = 14 - np.frexp(np.abs(q).max(1, keepdims=True))[1]
        terms = _fp16_terms(np.ldexp(q, exponent).astype(F32), query_terms or 2)
        per, weight = np.ldexp(kept_k[1][None], -exponent).astype(F32), kept_v[1][None]
    sums = [np.zeros((len(q), n), F32), np.zeros((len(q), n), F32)]
    for lo in range(0, hd, 16):
        for i, t in enumerate(terms):
            at = min(i, 1)
            sums[at] = _cut(sums[at].astype(F64) + t[:, lo:lo + 16].astype(F64) @ k[:, lo:lo + 16].T)
    x = (sums[0] + sums[1]) * per * (F32(scale) * F32(1.4426950408889634))
    p = np.exp2((x - x.max(1, keepdims=True)).astype(F64)).astype(F32)
    weights = _bf16_terms(p * weight, weight_terms)
    o = np.zeros((len(q), hd), F32)
    for lo in range(0, n, 16):
        if fp32_sums:
            d = np.zeros_like(o)
            for t in weights[::-1]:
                d = _cut(d.astype(F64) + t[:, lo:lo + 16].astype(F64) @ v[lo:lo + 16])
            o = o + d
        else:
            for t in weights:
                o = _cut(o.astype(F64) + t[:, lo:lo + 16].astype(F64) @ v[lo:lo + 16])
    return o / p.astype(F64).sum(1, keepdims=True)
