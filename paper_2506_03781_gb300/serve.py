"""A quantized decoder block in deployment: prompts and single tokens.

The block of ``recon.py`` (RMSNorm, rotary grouped-query attention, RMSNorm,
SwiGLU MLP) after training: its seven weights are multiplied from the exported
bit-planes (uq_bcq_gemv), and its keys and values live in a paged cache in
bf16, 8 or 4 bits that the library writes (uq_kv_write), reads back for a
prompt's own attention (uq_kv_read) and attends over for single tokens
(uq_paged_attn).  A prompt is taken in one go: a prefill begins a sequence.  Norms, rotations, the prompt's attention and
the MLP's product are torch operations.

``python -m paper_2506_03781_gb300.serve`` quantizes a small synthetic block,
prefills two prompts of different lengths and decodes tokens of both.
"""

from __future__ import annotations

import torch
import torch.nn.functional as F

from . import api
from .recon import NAMES, _rms_norm

MOST_TOKENS = 64                            # rows of one uq_bcq_gemv


class PagePool:
    """A key-value cache and who has its pages: tables of pages on the device (as uq_paged_attn takes them), free
    pages and lengths on the host."""

    def __init__(self, pages, kv_heads, head_dim, page_size=64, fmt=api.KV_INT8, sequences=MOST_TOKENS, max_pages=None,
                 device="cuda"):
        self.cache = api.empty_kv_cache(pages, kv_heads, page_size, head_dim, fmt, device)
        self.page_size, self.device = page_size, torch.device(device)
        self.max_pages = max_pages or pages
        self.table = torch.full((sequences, self.max_pages), -1, dtype=torch.int32, device=self.device)
        self.free = list(range(pages - 1, -1, -1))
        self.unused = list(range(sequences - 1, -1, -1))
        self.length, self.owned = {}, {}

    def open(self) -> int:
        """A new, empty sequence."""
        if not self.unused:
            raise RuntimeError("no sequence is unused")
        s = self.unused.pop()
        self.length[s], self.owned[s] = 0, []
        return s

    def close(self, s):
        """Gives a sequence's pages back."""
        self.free.extend(self.owned.pop(s))
        del self.length[s]
        self.table[s] = -1
        self.unused.append(s)

    def append(self, sequences, counts):
        """Room for counts[i] more tokens of sequences[i], each named once: (slots, positions) of all, in that order."""
        if len(set(sequences)) != len(sequences):
            raise ValueError("a sequence is named twice")
        if len(counts) != len(sequences) or any(n < 0 for n in counts):
            raise ValueError("every sequence needs a count of tokens, 0 at least")
        need = {s: -(-(self.length[s] + n) // self.page_size) for s, n in zip(sequences, counts)}
        if any(n > self.max_pages for n in need.values()) or sum(
                n - len(self.owned[s]) for s, n in need.items()) > len(self.free):
            raise RuntimeError("no page is free for these tokens")
        rows, cols, pages = [], [], []
        for s, n in need.items():
            for at in range(len(self.owned[s]), n):
                rows.append(s)
                cols.append(at)
                pages.append(self.free.pop())
                self.owned[s].append(pages[-1])
        if pages:
            at = torch.tensor([rows, cols, pages], device=self.device)
            self.table[at[0], at[1]] = at[2].to(torch.int32)
        size, slots, pos = self.page_size, [], []
        for s, n in zip(sequences, counts):
            lo, hi = self.length[s], self.length[s] + n
            for at in range(lo // size, -(-hi // size)):
                first = (self.owned[s][at] - at) * size
                slots += range(first + max(lo, at * size), first + min(hi, (at + 1) * size))
            pos += range(lo, hi)
            self.length[s] = hi
        return tuple(torch.tensor([slots, pos], dtype=torch.int64, device=self.device))


class BlockDecoder:
    """One block on its exported weights: {name: (bitplanes, alpha_star, zb_star)} for ``recon.NAMES``.  It has one
    workspace: its calls belong on one stream."""

    def __init__(self, shape, exported, g, pool: PagePool):
        self.shape, self.exported, self.g, self.pool = shape, exported, g, pool
        self.workspace = api.paged_attn_workspace(shape.heads, shape.kv_heads, shape.head_dim, pool.device)

    @classmethod
    def of(cls, block, pool):
        """The decoder of a ``recon.BlockReconstructor``'s current state."""
        exported = {}
        for n in NAMES:
            out, n_in = block.W[n].shape
            f = dict(dtype=torch.float32, device=block.device)
            exported[n] = (torch.empty(block.q, out, n_in // 32, dtype=torch.int32, device=block.device),
                           torch.empty(out, n_in // block.g, block.q, **f), torch.empty(out, n_in // block.g, **f))
            api.uq_export_bcq(block.W[n], block.q, block.g, block.P[n], block.codes[n], *exported[n])
        return cls(block.shape, exported, block.g, pool)

    def _check(self, X, rows=None):
        """X's shape, before a page is taken for its tokens."""
        if len(X.shape) != 2 or X.shape[1] != self.shape.d or rows not in (None, X.shape[0]):
            raise ValueError(f"X has shape {tuple(X.shape)}, expected ({'tokens' if rows is None else rows}, {self.shape.d})")

    def _linear(self, x, name):
        """x [tokens, in] fp32 -> [tokens, out] fp32."""
        planes, a, z = self.exported[name]
        y = torch.empty(x.shape[0], planes.shape[1], dtype=torch.float32, device=x.device)
        for lo in range(0, x.shape[0], MOST_TOKENS):
            api.uq_bcq_gemv(planes, a, z, x[lo:lo + MOST_TOKENS].contiguous(), y[lo:lo + MOST_TOKENS], self.g)
        return y

    def _rotated(self, x, positions):
        """x [tokens, heads, head_dim], rotated by its tokens' positions (as recon._rotary)."""
        half = x.shape[-1] // 2
        inv = self.shape.theta ** (-torch.arange(half, device=x.device, dtype=torch.float32) * 2.0 / x.shape[-1])
        angle = positions.float()[:, None, None] * inv
        c, s = torch.cos(angle), torch.sin(angle)
        x1, x2 = x[..., :half], x[..., half:]
        return torch.cat([x1 * c - x2 * s, x1 * s + x2 * c], dim=-1)

    def _qkv(self, X, positions):
        sh, n = self.shape, X.shape[0]
        h = _rms_norm(X, sh.eps)
        q = self._linear(h, "q_proj").view(n, sh.heads, sh.head_dim)
        k = self._linear(h, "k_proj").view(n, sh.kv_heads, sh.head_dim)
        v = self._linear(h, "v_proj").view(n, sh.kv_heads, sh.head_dim)
        return self._rotated(q, positions), self._rotated(k, positions), v

    def _rest(self, X, o):
        X1 = X + self._linear(o.reshape(X.shape[0], -1), "o_proj")
        h = _rms_norm(X1, self.shape.eps)
        return X1 + self._linear(F.silu(self._linear(h, "gate_proj")) * self._linear(h, "up_proj"), "down_proj")

    @torch.no_grad()
    def prefill(self, sequence, X):
        """The tokens X [n, d] (fp32) that begin a sequence: their hidden states after the block.  The prompt attends
        over its keys and values as the cache holds them, like the tokens that follow it will."""
        self._check(X)
        sh, n = self.shape, X.shape[0]
        if self.pool.length[sequence]:
            raise ValueError(f"sequence {sequence} has {self.pool.length[sequence]} tokens: a prefill begins a sequence")
        if n == 0:
            return torch.empty_like(X)
        slots, pos = self.pool.append([sequence], [n])
        q, k, v = self._qkv(X, pos)
        api.uq_kv_write(self.pool.cache, k, v, slots)
        api.uq_kv_read(self.pool.cache, slots, k, v)
        r = sh.heads // sh.kv_heads
        q, k, v = (t.transpose(0, 1)[None] for t in (q, k, v))
        o = F.scaled_dot_product_attention(q, k.repeat_interleave(r, 1), v.repeat_interleave(r, 1), is_causal=True,
                                           scale=sh.head_dim ** -0.5)
        return self._rest(X, o[0].transpose(0, 1))

    @torch.no_grad()
    def decode(self, sequences, X):
        """One more token of each of the sequences, X [len(sequences), d] (fp32): their hidden states after the block."""
        self._check(X, len(sequences))
        if not sequences:
            return torch.empty_like(X)
        slots, pos = self.pool.append(sequences, [1] * len(sequences))
        q, k, v = self._qkv(X, pos)
        api.uq_kv_write(self.pool.cache, k, v, slots)
        rows = torch.tensor(sequences, device=X.device)
        longest = max(len(self.pool.owned[s]) for s in sequences)
        o = torch.empty_like(q)
        api.uq_paged_attn(self.pool.cache, q, self.pool.table[rows, :longest], (pos + 1).to(torch.int32), o,
                          workspace=self.workspace)
        return self._rest(X, o)


def main():
    from . import recon, synth
    shape = synth.BLOCKS["small"]
    weights = {n: raw for n, (raw, _) in synth.block_weights(shape, 0).items()}
    block = recon.BlockReconstructor(shape, weights, q=3, g=64, G=8, T=4)
    for name, fmt in (("bf16", api.KV_BF16), ("int8", api.KV_INT8), ("int4", api.KV_INT4)):
        pool = PagePool(16, shape.kv_heads, shape.head_dim, page_size=16, fmt=fmt)
        dec = BlockDecoder.of(block, pool)
        prompts = [torch.randn(n, shape.d, device="cuda", generator=torch.Generator("cuda").manual_seed(n)) for n in (37, 5)]
        ids = [pool.open() for _ in prompts]
        for s, X in zip(ids, prompts):
            dec.prefill(s, X)
        x = torch.randn(2, shape.d, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
        for _ in range(8):
            y = dec.decode(ids, x)
        torch.cuda.synchronize()
        used = sum(t.numel() * t.element_size() for t in pool.cache.values()) / (16 * 16)
        print(f"{name}: {[pool.length[s] for s in ids]} tokens cached, {used:.0f} bytes a token; |y| = {y.norm().item():.3f}")


if __name__ == "__main__":
    main()
