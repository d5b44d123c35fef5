"""Helpers of the key-value cache tests: caches filled from the oracle's rows,
and the tolerances of the attention (derived here, from its arithmetic)."""

from __future__ import annotations

import numpy as np
import torch

from oracle import kv as OK
from paper_2506_03781_gb300 import api

F32, F64 = np.float32, np.float64
FMT = {"bf16": api.KV_BF16, "int8": api.KV_INT8, "int4": api.KV_INT4}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def dev():
    return torch.device("cuda:0")


def typed(x, dtype):
    """(device tensor of that type, the fp32 values it holds)."""
    x = np.ascontiguousarray(x, F32)
    t = torch.from_numpy(x).to(dev()).to(DT[dtype])
    return t, t.float().cpu().numpy()


def rows_to_cache(cache, fmt, name, kept, slots):
    """Stores the oracle's rows kept = (codes, scales, minima) [n, kv, ...] at `slots`."""
    codes, scales, minima = kept
    page_size = cache[name].shape[2]
    at, off = torch.as_tensor(slots // page_size), torch.as_tensor(slots % page_size)
    d = cache[name].device
    at, off = at.to(d), off.to(d)
    if fmt == "bf16":
        cache[name][at, :, off] = torch.from_numpy(codes).to(d).to(torch.bfloat16)
    elif fmt == "int8":
        cache[name][at, :, off] = torch.from_numpy(codes).to(d)
        cache[name + "_scale"][at, :, off] = torch.from_numpy(scales).to(d)
    else:
        packed = (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)
        cache[name][at, :, off] = torch.from_numpy(packed).to(d)
        pair = np.stack([scales, minima], -1)
        cache[name + "_scale"][at, :, off] = torch.from_numpy(pair).to(d).to(torch.bfloat16)


def cache_rows(cache, fmt, name, slots):
    """(codes, scales, minima) of the rows at `slots`, as numpy arrays like the oracle's."""
    page_size = cache[name].shape[2]
    at, off = torch.as_tensor(slots // page_size).to(dev()), torch.as_tensor(slots % page_size).to(dev())
    rows = cache[name][at, :, off]
    if fmt == "bf16":
        return rows.float().cpu().numpy(), None, None
    scales = cache[name + "_scale"][at, :, off].float().cpu().numpy()
    rows = rows.cpu().numpy()
    if fmt == "int8":
        return rows, scales, None
    codes = np.stack([rows & 15, rows >> 4], -1).reshape(*rows.shape[:-1], -1)
    return codes, scales[..., 0], scales[..., 1]


def poison(cache):
    """Every bit set: NaN in bf16 rows and in all scales."""
    for t in cache.values():
        t.view(torch.uint8).fill_(255)


class Case:
    """Sequences of `lens` tokens in a shuffled pool whose unused places are NaN, their values and one new token's
    queries."""

    def __init__(self, fmt, dtype, hd, kv, r, page, lens, seed=0, spare=3, width=None, scale_v=0.5):
        rng = np.random.default_rng(seed)
        self.fmt, self.dtype, self.hd, self.kv, self.r, self.page, self.lens = fmt, dtype, hd, kv, r, page, list(lens)
        B = len(lens)
        need = [-(-n // page) for n in lens]
        self.pages = sum(need) + spare
        order = rng.permutation(self.pages)
        width = width or max(1, max(need))
        # entries that no position needs: beyond the pool, negative, or another sequence's page
        self.table = rng.choice(np.array([-1, self.pages, 2 ** 31 - 1, -2 ** 31, 0], np.int64), (B, width)).astype(np.int32)
        first = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[first:first + n]
            first += n
        self.cache = api.empty_kv_cache(self.pages, kv, page, hd, FMT[fmt], dev())
        poison(self.cache)
        self.K, self.V = [], []                       # fp64 values [kv, n, hd] of every sequence
        for b, n in enumerate(lens):
            pos = np.arange(n)
            slots = self.table[b].astype(np.int64)[pos // page] * page + pos % page
            k = rng.standard_normal((n, kv, hd)).astype(F32)
            k[..., :: max(1, hd // 4)] *= 3
            v = (rng.standard_normal((n, kv, hd)) * scale_v).astype(F32)
            for name, x, keep in (("k", k, self.K), ("v", v, self.V)):
                kept = OK.quantise_rows(x, fmt)
                if n:
                    rows_to_cache(self.cache, fmt, name, kept, slots)
                keep.append(OK.row_values(kept, fmt).transpose(1, 0, 2))
        self.q, self.qv = typed(rng.standard_normal((B, kv * r, hd)), dtype)
        self.tab = torch.from_numpy(self.table).to(dev())
        self.len = torch.tensor(self.lens, dtype=torch.int32, device=dev())
        self.out = torch.full((B, kv * r, hd), float("nan"), dtype=DT[dtype], device=dev())
        self.lse = torch.full((B, kv * r), float("nan"), device=dev())

    def run(self, **more):
        H = self.kv * self.r
        ws = api.paged_attn_workspace(H, self.kv, self.hd, dev())
        ws.fill_(255)                                 # its contents do not matter
        more.setdefault("workspace", ws)
        api.uq_paged_attn(self.cache, self.q, self.tab, self.len, self.out, lse=self.lse, **more)
        torch.cuda.synchronize()
        return self.out, self.lse

    def check(self, scale=None, window=0, hidden=None, **more):
        """Runs and compares with the oracle; hidden: {sequence: positions that do not count}."""
        scale = self.hd ** -0.5 if scale is None else scale
        out, lse = self.run(scale=scale, window=window, **more)
        out, lse = out.float().cpu().numpy(), lse.cpu().numpy()
        for b, n in enumerate(self.lens):
            pos = np.arange(max(0, n - window) if window else 0, n)
            if hidden and b in hidden:
                pos = np.setdiff1d(pos, hidden[b])
            K, V = self.K[b][:, pos], self.V[b][:, pos]
            ref, ref_lse = OK.attend(self.qv[b], K, V, scale)
            tol, tol_lse = tolerance(self.qv[b], K, V, scale, ref, ref_lse, self.dtype)
            if len(pos) == 0:
                assert np.array_equal(out[b], ref) and np.array_equal(lse[b], ref_lse), f"sequence {b} of {n}"
                continue
            err, err_lse = np.abs(out[b] - ref), np.abs(lse[b] - ref_lse)
            assert np.isfinite(out[b]).all(), f"sequence {b} of {n} tokens: not finite"
            assert (err <= tol).all(), f"sequence {b} of {n} tokens: {(err / tol).max():.3g} x tolerance"
            assert (err_lse <= tol_lse).all(), f"sequence {b} of {n}: lse {(err_lse / tol_lse).max():.3g} x tolerance"


def tolerance(q, K, V, scale, ref, ref_lse, dtype):
    """How far the kernel may be from the fp64 result.

    A score is a sum of hd products in fp32, scaled and taken to base 2 (a few
    roundings more): off by (hd + 20) u reach, reach = max_t scale sum_d |q_d
    k_td|.  That and 16 u of the exponential are the relative error of a
    weight, which enters numerator and denominator.  A weight is then the sum
    of two bf16 for bf16 results (2^-16) and of three for fp32 (2^-24).  Sums over n positions
    are chains of at most n / 8 + 64 additions, each off by up to 2 u (the
    tensor cores truncate).  A bf16 result is rounded once more, by 2^-8 of
    itself."""
    n, hd = K.shape[1], q.shape[1]
    mass, reach = OK.attend_mass(q, K, V, scale)
    d = (hd + 20) * U * reach + 16 * U
    chain = (n / 8 + 64) * 2 * U
    split = 2.0 ** -16 if dtype == "bf16" else 2.0 ** -24
    tol = (2 * d[:, None] + 2 * chain + split) * mass + 1e-30
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * np.abs(ref)
    return tol, d + chain + 4 * U * np.abs(ref_lse) + 1e-7
