"""Helpers of the tests of attention over several new tokens of a sequence."""

from __future__ import annotations

import random

import numpy as np
import torch

from oracle import kv as OK
from paper_2506_03781_gb300 import api
from tests import kv_cases as C


def tree_masks(T, seed, wide=4):
    """Ancestors of T drafts: the first one is the root, every other a child of one of the few before it."""
    r = random.Random(seed)
    masks = []
    for i in range(T):
        masks.append((masks[r.randrange(max(0, i - wide), i)] if i else 0) | 1 << i)
    return masks


def signed(masks):
    return [m - (1 << 64) if m >> 63 else m for m in masks]


def tolerance(q, K, V, scale, ref, ref_lse, dtype, weighted):
    """As kv_cases.tolerance, but weights of bf16 results are rounded to bf16 once: half a step, 2^-8 of what each
    multiplies.  That is the value itself; of 4 bits it is s (c - 7.5), because a value is s (c - 7.5) + (m + 7.5 s) and
    the second part meets the sum of the weights before they are rounded: |s (c - 7.5)| may be larger than |value| (c = 8,
    m = -8 s: s / 2, 0).  `weighted`: what the weights multiply, as V."""
    tol, tol_lse = C.tolerance(q, K, V, scale, ref, ref_lse, dtype)
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * OK.attend_mass(q, K, weighted, scale)[0]
    return tol, tol_lse


class Rows:
    """Sequences of `lens` tokens, new[b] of them new, on kv_cases.Case's pool; trees: masks of every sequence's drafts,
    `most` rows each."""

    def __init__(self, fmt, dtype, hd, kv, r, page, lens, new, trees=False, most=None, seed=0, **more):
        self.c = C.Case(fmt, dtype, hd, kv, r, page, lens, seed=seed, **more)
        self.new, self.trees, self.dtype, self.lens = list(new), trees, dtype, list(lens)
        self.H, self.hd, self.kv = kv * r, hd, kv
        rng = np.random.default_rng(seed + 1)
        B = len(lens)
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        if trees:
            self.most = most or max(1, max(new))
            self.masks = [tree_masks(self.most, seed + b) for b in range(B)]
            shape = (B, self.most)
            self.tree = torch.tensor([signed(m) for m in self.masks], dtype=torch.int64).to(C.dev())
            self.counts = torch.tensor(self.new, dtype=torch.int32, device=C.dev())
        else:
            shape = (int(self.starts[-1]) + 3,)        # three rows behind the last sequence
            self.starts_d = torch.from_numpy(self.starts).to(C.dev())
        self.q, self.qv = C.typed(rng.standard_normal((*shape, self.H, hd)), dtype)
        self.out = torch.full((*shape, self.H, hd), 7.0, dtype=C.DT[dtype], device=C.dev())
        self.lse = torch.full((*shape, self.H), 7.0, device=C.dev())

    def run(self, **more):
        c = self.c
        if "workspace" not in more:
            more["workspace"] = api.paged_rows_workspace(self.H, self.kv, self.hd, C.dev()).fill_(255)
        if self.trees:
            api.uq_paged_tree_attn(c.cache, self.q, self.tree, c.tab, c.len, self.out, counts=self.counts, lse=self.lse, **more)
        else:
            api.uq_paged_prompt_attn(c.cache, self.q, self.starts_d, c.tab, c.len, self.out, lse=self.lse, **more)
        torch.cuda.synchronize()
        return self.out, self.lse

    def sees(self, b, window, sinks):
        n, k = self.lens[b], self.new[b]
        return OK.tree_sees(n, self.masks[b][:k], window, sinks) if self.trees else OK.prompt_sees(n, k, window, sinks)

    def weighted(self, b):
        """What the weights multiply, [kv, n, hd] (see tolerance)."""
        if self.c.fmt != "int4" or self.lens[b] == 0:
            return self.c.V[b]
        t = np.arange(self.lens[b])
        slots = self.c.table[b].astype(np.int64)[t // self.c.page] * self.c.page + t % self.c.page
        codes, s, _ = C.cache_rows(self.c.cache, "int4", "v", slots)
        return ((np.asarray(codes, np.float64) - 7.5) * np.repeat(np.asarray(s, np.float64), OK.GROUP, -1)).transpose(1, 0, 2)

    def at(self, b, i):
        return (b, i) if self.trees else (int(self.starts[b]) + i,)

    def check(self, scale=None, window=0, sinks=0, hidden=None, every=1, **more):
        """Runs and compares with the oracle, every `every`-th new token; hidden: {sequence: positions that do not count}."""
        scale = self.hd ** -0.5 if scale is None else scale
        out, lse = self.run(scale=scale, window=window, sinks=sinks, **more)
        out, lse = out.float().cpu().numpy(), lse.cpu().numpy()
        left = np.ones(out.shape[:-2], bool)
        for b, (n, k) in enumerate(zip(self.lens, self.new)):
            sees, weighted = self.sees(b, window, sinks), self.weighted(b)
            if hidden and b in hidden:
                sees[:, hidden[b]] = False
            for i in range(k):
                left[self.at(b, i)] = False
            for i in sorted(set(range(0, k, every)) | {k - 1} if k else ()):
                where = self.at(b, i)
                pos = np.nonzero(sees[i])[0]
                K, V, q = self.c.K[b][:, pos], self.c.V[b][:, pos], self.qv[where]
                ref, ref_lse = OK.attend(q, K, V, scale)
                if len(pos) == 0:
                    assert np.array_equal(out[where], ref) and np.array_equal(lse[where], ref_lse), (b, i)
                    continue
                tol, tol_lse = tolerance(q, K, V, scale, ref, ref_lse, self.dtype, weighted[:, pos])
                assert np.isfinite(out[where]).all(), f"sequence {b} of {n}, new token {i} of {k}: not finite"
                err, err_lse = np.abs(out[where] - ref), np.abs(lse[where] - ref_lse)
                assert (err <= tol).all(), f"sequence {b} of {n}, new token {i} of {k}: {(err / tol).max():.3g} x tolerance"
                assert (err_lse <= tol_lse).all(), f"sequence {b}, new token {i}: lse {(err_lse / tol_lse).max():.3g} x tolerance"
        assert (out[left] == 7).all() and (lse[left] == 7).all()          # rows of no token
        return self
