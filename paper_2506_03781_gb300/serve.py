"""A quantized decoder block in deployment: prompts and single tokens.

The block of ``recon.py`` (RMSNorm, rotary grouped-query attention, RMSNorm,
SwiGLU MLP) after training: its seven weights are multiplied from the exported
bit-planes (uq_bcq_gemv), and its keys and values live in a paged cache in
bf16, 8 or 4 bits, into which the library rotates and appends them
(uq_kv_append) and over which it attends for prompts and chunks of them
(uq_paged_prompt_attn; long prompts of heads of 256 channels read their rows
back, uq_kv_read, for torch's attention), single tokens (uq_paged_attn, with a window
uq_paged_attn_sinks) and trees of drafted tokens (uq_paged_tree_attn).  A prefill
begins a sequence, extend adds chunks, decode single tokens; verify takes drafts,
of which keep leaves a path.  Norms and the MLP's product are torch operations.

``python -m paper_2506_03781_gb300.serve`` quantizes a small synthetic block,
prefills two prompts of different lengths and decodes tokens of both.
"""

from __future__ import annotations

import torch
import torch.nn.functional as F

from . import api
from .recon import NAMES, _rms_norm

MOST_TOKENS = 64                            # rows of one uq_bcq_gemv
# Tokens from which on a prompt of fp32 heads of 256 channels attends over rows that are read back: uq_paged_prompt_attn does
# such heads one row at a time.  Reading back and torch's attention / uq_paged_prompt_attn, us, rows of bf16: 4 heads over one of
# K and V: 64 tokens 109 / 29, 256 tokens 109 / 97, 700 tokens 113 / 381, 4096 tokens 864 / 5700; 32 over 8: 64 tokens 109 / 36,
# 256 tokens 113 / 215, 700 tokens 265 / 1280, 2048 tokens 1371 / 9978; 8 and 4 bits alike.
LONG_PROMPT = 256


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
        self.drafted = {}                   # sequences that end in drafts (verify): tokens before them, the drafts' parents

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
        self.drafted.pop(s, None)
        self.table[s] = -1
        self.unused.append(s)

    def append(self, sequences, counts):
        """Room for counts[i] more tokens of sequences[i], each named once: (slots, positions) of all, in that order."""
        if len(set(sequences)) != len(sequences):
            raise ValueError("a sequence is named twice")
        if len(counts) != len(sequences) or any(n < 0 for n in counts):
            raise ValueError("every sequence needs a count of tokens, 0 at least")
        for s, n in zip(sequences, counts):
            _, parents = self.drafted.get(s, (0, []))
            if n and not chain(parents, range(len(parents))):
                raise ValueError(f"sequence {s} ends in a tree of drafts: keep leaves a path of them, behind which more may come")
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
            if n:
                self.drafted.pop(s, None)
        return tuple(torch.tensor([slots, pos], dtype=torch.int64, device=self.device))

    def truncate(self, s, n):
        """The first n tokens of a sequence stay; pages behind them are given back."""
        if not 0 <= n <= self.length[s]:
            raise ValueError(f"sequence {s} has {self.length[s]} tokens: 0 to as many may stay, not {n}")
        keep = -(-n // self.page_size)
        self.free.extend(reversed(self.owned[s][keep:]))
        del self.owned[s][keep:]
        self.table[s, keep:] = -1
        self.length[s] = n
        if s in self.drafted:
            before, parents = self.drafted.pop(s)
            if n > before:
                self.drafted[s] = before, parents[:n - before]

    def keep(self, s, drafts, path):
        """Of a sequence's last `drafts` tokens those of `path` stay (increasing places among them, a chain of the tree):
        their rows move up behind the tokens before, the rest is given back.  Drafts that verify has put there stay only
        behind the one that they follow: their keys are rotated for no other place."""
        path = list(path)
        first = self.length[s] - drafts
        if drafts < 0 or first < 0:
            raise ValueError(f"sequence {s} has {self.length[s]} tokens, fewer than {drafts}")
        if any(not 0 <= i < drafts for i in path) or any(a >= b for a, b in zip(path, path[1:])):
            raise ValueError(f"path must be increasing places below {drafts}")
        before, parents = self.drafted.get(s, (self.length[s], []))
        old = [j for j in path if first + j < before]                         # tokens that are no drafts
        stay = [*range(before, first), *(first + j for j in path[len(old):])]
        if not chain(parents, [t - before for t in stay]) or (stay and len(old) < before - first):
            raise ValueError(f"path is no chain of the drafts of sequence {s}")
        moved = [(i, j) for i, j in enumerate(path) if i != j]
        if moved:
            place = lambda t: [self.owned[s][t // self.page_size], t % self.page_size]
            to = torch.tensor([place(first + i) for i, _ in moved], device=self.device).T
            at = torch.tensor([place(first + j) for _, j in moved], device=self.device).T
            for rows in self.cache.values():
                rows[to[0], :, to[1]] = rows[at[0], :, at[1]]              # (all are read before the first is written)
        self.truncate(s, first + len(path))
        self.drafted.pop(s, None)


def chain(parents, drafts):
    """Whether each of the drafts follows the one before it, and the first one none."""
    return [parents[i] for i in drafts] == [-1, *drafts][:len(drafts)]


def ancestors(parents):
    """[batch, drafts] parents (places of the same row's earlier drafts, -1: the last token before the drafts) as int64
    masks for uq_paged_tree_attn, and the drafts' depths."""
    masks, depths = [], []
    for row in parents:
        bits, deep = [], []
        for i, p in enumerate(row):
            if not -1 <= p < i or i >= 64:
                raise ValueError("a draft's parent is an earlier one of 64 at most, or -1")
            bits.append(1 << i | (bits[p] if p >= 0 else 0))
            deep.append(deep[p] + 1 if p >= 0 else 0)
        masks.append([m - (1 << 64) if m >> 63 else m for m in bits])
        depths.append(deep)
    return masks, depths


class BlockDecoder:
    """One block on its exported weights: {name: (bitplanes, alpha_star, zb_star)} for ``recon.NAMES``.  Its tokens see the
    last ``window`` positions (0: all) and the first ``sinks``.  It has one workspace, for single tokens (several
    take one of the allocator's, which all decoders share): its calls belong on one stream."""

    def __init__(self, shape, exported, g, pool: PagePool, window=0, sinks=0):
        if window < 0 or sinks < 0:
            raise ValueError(f"window={window} and sinks={sinks} must be 0 at least")
        self.shape, self.exported, self.g, self.pool = shape, exported, g, pool
        self.window, self.sinks = window, sinks
        self.workspace = api.paged_attn_workspace(shape.heads, shape.kv_heads, shape.head_dim, pool.device)
        self.rope = torch.empty(0, shape.head_dim // 2, 2, device=pool.device)

    def _rotations(self):
        """(cos, sin) of at least the positions that the pool's sequences have so far (as recon._rotary): a table that doubles
        as they grow, since each decoder has its own and a pool's every page for one sequence would be 268 MB of it (8192
        pages of 64, 128 channels)."""
        n = max(self.pool.length.values())
        if n > len(self.rope):
            half = self.shape.head_dim // 2
            inv = self.shape.theta ** (-torch.arange(half, device=self.rope.device, dtype=torch.float32) * 2.0 / self.shape.head_dim)
            angle = torch.arange(max(1024, 1 << (n - 1).bit_length()), device=self.rope.device).float()[:, None] * inv
            self.rope = torch.stack([torch.cos(angle), torch.sin(angle)], -1)
        return self.rope

    @classmethod
    def of(cls, block, pool, **more):
        """The decoder of a ``recon.BlockReconstructor``'s current state."""
        exported = {}
        for n in NAMES:
            out, n_in = block.W[n].shape
            f = dict(dtype=torch.float32, device=block.device)
            exported[n] = (torch.empty(block.q, out, n_in // 32, dtype=torch.int32, device=block.device),
                           torch.empty(out, n_in // block.g, block.q, **f), torch.empty(out, n_in // block.g, **f))
            api.uq_export_bcq(block.W[n], block.q, block.g, block.P[n], block.codes[n], *exported[n])
        return cls(block.shape, exported, block.g, pool, **more)

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

    def _append(self, X, slots, positions):
        """The tokens' rotated queries; their keys and values go into the cache."""
        sh, n = self.shape, X.shape[0]
        h = _rms_norm(X, sh.eps)
        q = self._linear(h, "q_proj").view(n, sh.heads, sh.head_dim)
        k = self._linear(h, "k_proj").view(n, sh.kv_heads, sh.head_dim)
        v = self._linear(h, "v_proj").view(n, sh.kv_heads, sh.head_dim)
        api.uq_kv_append(self.pool.cache, k, v, slots, positions, self._rotations(), q=q, q_out=q)
        return q

    def _tables(self, sequences):
        """(block table, lengths) of sequences on the device."""
        rows = torch.tensor(sequences, device=self.pool.device)
        longest = max(1, max(len(self.pool.owned[s]) for s in sequences))
        lens = torch.tensor([self.pool.length[s] for s in sequences], dtype=torch.int32, device=self.pool.device)
        return self.pool.table[rows, :longest], lens

    def _rest(self, X, o):
        X1 = X + self._linear(o.reshape(X.shape[0], -1), "o_proj")
        h = _rms_norm(X1, self.shape.eps)
        return X1 + self._linear(F.silu(self._linear(h, "gate_proj")) * self._linear(h, "up_proj"), "down_proj")

    @torch.no_grad()
    def prefill(self, sequence, X):
        """The tokens X [n, d] (fp32) that begin a sequence: their hidden states after the block.  The prompt attends
        over its keys and values as the cache holds them, like the tokens that follow it will."""
        self._check(X)
        if self.pool.length[sequence]:
            raise ValueError(f"sequence {sequence} has {self.pool.length[sequence]} tokens: a prefill begins a sequence")
        if self.shape.head_dim == 256 and not self.window and X.shape[0] >= LONG_PROMPT:
            return self._prefill_read_back(sequence, X)
        return self.extend([sequence], X, [X.shape[0]])

    def _prefill_read_back(self, sequence, X):
        """The same with the cache's rows read back and torch's attention over them."""
        sh, n = self.shape, X.shape[0]
        slots, pos = self.pool.append([sequence], [n])
        q = self._append(X, slots, pos)
        k, v = (q.new_empty(n, sh.kv_heads, sh.head_dim) for _ in range(2))
        api.uq_kv_read(self.pool.cache, slots, k, v)
        r = sh.heads // sh.kv_heads
        q, k, v = (t.transpose(0, 1)[None] for t in (q, k, v))
        o = F.scaled_dot_product_attention(q, k.repeat_interleave(r, 1), v.repeat_interleave(r, 1), is_causal=True,
                                           scale=sh.head_dim ** -0.5)
        return self._rest(X, o[0].transpose(0, 1))

    @torch.no_grad()
    def extend(self, sequences, X, counts):
        """The next counts[i] tokens of sequences[i], all in X [sum of counts, d] (fp32), on top of what is cached of them:
        their hidden states after the block."""
        if any(n < 0 for n in counts) or len(counts) != len(sequences):
            raise ValueError("every sequence needs a count of tokens, 0 at least")
        self._check(X, sum(counts))
        if X.shape[0] == 0:
            return torch.empty_like(X)
        slots, pos = self.pool.append(sequences, counts)
        q = self._append(X, slots, pos)
        starts = torch.tensor([0, *counts], device=X.device).cumsum(0).to(torch.int32)
        table, lens = self._tables(sequences)
        o = torch.empty_like(q)
        api.uq_paged_prompt_attn(self.pool.cache, q, starts, table, lens, o, window=self.window, sinks=self.sinks)
        return self._rest(X, o)

    @torch.no_grad()
    def verify(self, sequences, X, parents):
        """Drafted tokens X [len(sequences), drafts, d] (fp32, 64 drafts at most) of sequences, parents[i][j] the draft that
        draft j of sequence i follows (an earlier one; -1: the sequence's last token): their hidden states after the
        block.  They stay in the cache as the sequences' last tokens until pool.keep leaves a path of them; behind a tree no
        more tokens may come before."""
        B, T = len(sequences), len(parents[0]) if len(parents) else 0
        if len(parents) != B or any(len(p) != T for p in parents):
            raise ValueError("every sequence needs its drafts' parents, as many for each")
        if tuple(X.shape) != (B, T, self.shape.d):
            raise ValueError(f"X has shape {tuple(X.shape)}, expected {(B, T, self.shape.d)}")
        masks, depths = ancestors(parents)
        if B * T == 0:
            return torch.empty_like(X)
        before = [self.pool.length[s] for s in sequences]
        slots, _ = self.pool.append(sequences, [T] * B)
        self.pool.drafted.update((s, (n, list(row))) for s, n, row in zip(sequences, before, parents))
        pos = torch.tensor([n + d for n, row in zip(before, depths) for d in row], dtype=torch.int64, device=X.device)
        flat = X.reshape(B * T, -1)
        q = self._append(flat, slots, pos).view(B, T, self.shape.heads, self.shape.head_dim)
        table, lens = self._tables(sequences)
        o = torch.empty_like(q)
        api.uq_paged_tree_attn(self.pool.cache, q, torch.tensor(masks, device=X.device), table, lens, o, window=self.window,
                               sinks=self.sinks)
        return self._rest(flat, o).view(B, T, -1)

    @torch.no_grad()
    def decode(self, sequences, X):
        """One more token of each of the sequences, X [len(sequences), d] (fp32): their hidden states after the block."""
        self._check(X, len(sequences))
        if not sequences:
            return torch.empty_like(X)
        slots, pos = self.pool.append(sequences, [1] * len(sequences))
        q = self._append(X, slots, pos)
        table, lens = self._tables(sequences)
        o = torch.empty_like(q)
        if self.window:
            api.uq_paged_attn_sinks(self.pool.cache, q, table, lens, o, window=self.window, sinks=self.sinks,
                                    workspace=self.workspace)
        else:
            api.uq_paged_attn(self.pool.cache, q, table, lens, o, workspace=self.workspace)
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
