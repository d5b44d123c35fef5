"""What the operators around the paged key-value cache are timed on: new tokens'
keys and values rotated by their positions and appended to the cache, and
attention over it with a sliding window and first tokens that stay visible
(sinks), of one new token, of prompts' chunks and of trees of drafted tokens.

Cache.  A pool of pages; a page holds `page` consecutive tokens of one
sequence, for every key/value head: k, v [pages, kv_heads, page, row], with a
row of `hd` channels kept as

* "bf16"  the values, rounded to nearest even;
* "int8"  codes c in -127..127 and one fp32 scale per row: amax = max |x|,
          scale = amax / 127, c = rint(x * (127 / amax)), value = c * scale;
* "int4"  codes c in 0..15, two to a byte (even channel low), and a bf16 pair
          (scale, minimum) per 64 channels: scale = bf16((max - min) / 15),
          minimum = bf16(min), c = clamp(rint((x - minimum) * (1 / scale)),
          0, 15), value = c * scale + minimum.

Every quotient, product and difference is rounded to fp32; ties of rint go to
even.  A slot is page * page_size + offset; a negative slot is written nowhere
and read as zeros.

Rotation.  Channels (j, j + rot / 2), j < rot / 2, of a query or key at position
p become (a c - b s, a s + b c) with (c, s) = rope[p, j]; every product, sum and
difference is rounded to fp32, and keys are quantised from that.  Channels from
`rot` on stay.

Kinds of a case:

* "append"  new tokens' queries and keys are rotated, keys and values written;
* "sinks"   one new token of every sequence sees its last `window` positions
            and the first `sinks`;
* "prompt"  every sequence's last few tokens, a chunk of its prompt, each see
            what is not behind them, in the window or among the sinks;
* "tree"    up to 64 drafted tokens of a sequence, each of which sees the tokens
            before the drafts and its own ancestors; distances go by depth.
"""

import math
import random

import torch

own = False

WIDTH = {"bf16": 2, "f32": 4}
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 64                                  # channels of an int4 group
TINY = 2.0 ** -100                          # smaller ranges are kept as zeros
ROWS = 1 << 16                              # cache rows that prepare() fills at a time
WORKSPACE = 64 << 20                        # bytes of scratch that a serving program keeps for its attention calls
DRAFTS = 64                                 # tokens of a tree at most
PAIRS = 1 << 31                             # scores that a prompt or a tree has at most


def _append(name, tokens, fmt, dtype, heads, kv, hd, page, rot, far, padded):
    return dict(name=name, kind="append", tokens=tokens, fmt=fmt, dtype=dtype, heads=heads, kv=kv, hd=hd, page=page,
                rot=rot, far=far, padded=padded)


def _attend(name, kind, batch, new, length, fmt, dtype, heads, kv, hd, page, ragged, window, sinks):
    return dict(name=name, kind=kind, batch=batch, new=new, length=length, fmt=fmt, dtype=dtype, heads=heads, kv=kv,
                hd=hd, page=page, ragged=ragged, window=window, sinks=sinks)


def listed():
    return [
        # one user's next token on the 8B block (32 heads, 8 key/value heads of 128): latency counts
        _append("append_1_bf16", 1, "bf16", "bf16", 32, 8, 128, 16, 128, 9000, False),
        # a decode step of 64 users at different positions, fp32 as the deployment product writes them
        _append("append_64_int4_f32", 64, "int4", "f32", 32, 8, 128, 32, 128, 131072, False),
        # one sample of the reconstruction's length
        _append("append_2048_int8", 2048, "int8", "bf16", 32, 8, 128, 16, 128, 2048, False),
        # several prompts packed and padded, half of the channels rotated
        _append("append_20011_int4", 20011, "int4", "bf16", 32, 8, 128, 64, 64, 32768, True),
        # chats that have run for very long, on a cache in 8 bits: 4 sinks and a window
        _attend("sinks_16x120000_int8", "sinks", 16, 1, 120000, "int8", "bf16", 32, 8, 128, 64, False, 4096, 4),
        # a full server of the 70B shape, some sequences shorter than the window
        _attend("sinks_128_ragged_int4_f32", "sinks", 128, 1, 9000, "int4", "f32", 64, 8, 128, 32, True, 2047, 64),
        # one long prompt in one go
        _attend("prompt_1x8192_bf16", "prompt", 1, 8192, 8192, "bf16", "bf16", 32, 8, 128, 16, False, 4096, 4),
        # chunks of several prompts on top of what is cached of them
        _attend("prompt_8x512_ragged_int8", "prompt", 8, 512, 6000, "int8", "bf16", 32, 8, 128, 64, True, 2048, 16),
        # the deployed block's prompt in fp32, everything visible
        _attend("prompt_3x700_f32", "prompt", 3, 700, 700, "bf16", "f32", 32, 8, 128, 16, True, 0, 0),
        # one user's drafts in a short chat: latency counts
        _attend("tree_1x16_bf16", "tree", 1, 16, 2000, "bf16", "bf16", 32, 8, 128, 16, False, 0, 0),
        # a server's batch, trees and lengths of different sizes
        _attend("tree_32x60_ragged_int8", "tree", 32, 60, 8192, "int8", "bf16", 32, 8, 128, 16, True, 0, 0),
        # small trees of the 70B shape over long sequences on the smallest cache, windowed
        _attend("tree_16x8_int4_f32", "tree", 16, 8, 30001, "int4", "f32", 64, 8, 128, 32, False, 16384, 4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Kinds as listed: 1 to 20000 tokens appended; 1 to 128 sequences of 1 to 120000 tokens, prompts' chunks of 1 to
    8192 tokens, trees of 1 to 64; any number of heads from 1 to 16 per key/value head, pages of 16 to 128 tokens."""
    kind = rng.choice(["append", "append", "sinks", "sinks", "prompt", "prompt", "tree", "tree"])
    fmt, dtype = rng.choice(["bf16", "int8", "int4"]), rng.choice(["bf16", "bf16", "f32"])
    hd = rng.choice([64, 128, 128, 128, 256])
    kv = rng.choice([1, 2, 4, 5, 8, 8]) if hd < 256 else rng.choice([1, 2, 4])
    page = rng.choice([16, 16, 32, 64, 128])
    heads = kv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 16] if kv <= 4 else [1, 2, 4, 4, 7, 8])
    if kind == "append":
        most = 20000 * 48 * 128 // ((heads + 2 * kv) * hd * (2 if dtype == "f32" else 1))
        c = _append("", min(_log(rng, 1, 20000), most), fmt, dtype, heads, kv, hd, page,
                    rng.choice([hd, hd, hd, hd // 2, hd // 4]), _log(rng, 20000, 131072), rng.random() < 0.3)
    else:
        sinks, ragged = rng.choice([0, 1, 4, 4, 16, 64, 100]), rng.random() < 0.6
        values = 2 ** 29 // (kv * hd * (4 if fmt == "bf16" else 2 if fmt == "int8" else 1))
        if kind == "sinks":
            batch, new = _log(rng, 1, 128), 1
            length = min(_log(rng, 1, 120000), max(1, values // batch))
            window = _log(rng, 1, min(8192, 2 ** 19 // batch))
        else:
            batch = _log(rng, 1, 8 if kind == "prompt" else 32)
            new = _log(rng, 1, 8192 // batch) if kind == "prompt" else _log(rng, 1, DRAFTS)
            length = min(_log(rng, 1, 30000), max(1, values // batch), max(1, PAIRS // 2 // (batch * new * heads))) + new
            new = min(new, length)
            window = rng.choice([0, _log(rng, 1, 8192)])
        c = _attend("", kind, batch, new, length, fmt, dtype, heads, kv, hd, page, ragged, window, sinks)
    del c["name"]
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _lengths(case):
    """Every sequence's number of tokens and how many of them are new: `length` and `new`, or spread over 1..length and
    1..new by logarithm, with one empty sequence (an idle place of the server's batch) where there are at least four."""
    B, n, new = case["batch"], case["length"], case["new"]
    if not case["ragged"]:
        return [n] * B, [new] * B
    r = random.Random(B * 1000003 + n * 101 + new)
    lens = [_log(r, 1, n) for _ in range(B)]
    lens[r.randrange(B)] = n
    if B >= 4:
        lens[r.randrange(B)] = 0
    return lens, [min(k, _log(r, 1, new)) if case["kind"] != "sinks" else min(k, 1) for k in lens]


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _empty_cache(pages, case):
    """Buffers as a server takes them: what was never written is no number."""
    kv, hd, page, fmt = case["kv"], case["hd"], case["page"], case["fmt"]
    shape = (pages, kv, page)
    if fmt == "bf16":
        mk = lambda: torch.full((*shape, hd), float("nan"), dtype=torch.bfloat16, device="cuda")
        return {"k": mk(), "v": mk()}
    c = {}
    for n in ("k", "v"):
        if fmt == "int8":
            c[n] = torch.full((*shape, hd), -1, dtype=torch.int8, device="cuda")
            c[n + "_scale"] = torch.full(shape, float("nan"), dtype=torch.float32, device="cuda")
        else:
            c[n] = torch.full((*shape, hd // 2), 255, dtype=torch.uint8, device="cuda")
            c[n + "_scale"] = torch.full((*shape, hd // GROUP, 2), float("nan"), dtype=torch.bfloat16, device="cuda")
    return c


def _rows(gen, n, case):
    """n tokens' keys and values: normal, a few channels of the keys several times larger (as rotated keys have)."""
    kv, hd = case["kv"], case["hd"]
    k = torch.randn(n, kv, hd, generator=gen, device="cuda")
    k[:, :, :: hd // 4] *= 4.0
    v = torch.randn(n, kv, hd, generator=gen, device="cuda") * 0.5
    return k.to(DTYPE[case["dtype"]]), v.to(DTYPE[case["dtype"]])


def _trees(B, T, seed):
    """[B, T] ancestor masks: the first token is the root, every other one a child of one of the four before it."""
    r = random.Random(B * 7919 + T * 31 + seed)
    rows = []
    for _ in range(B):
        masks = []
        for i in range(T):
            masks.append((masks[r.randrange(max(0, i - 4), i)] if i else 0) | 1 << i)
        rows.append([m - (1 << 64) if m >> 63 else m for m in masks])
    return torch.tensor(rows, dtype=torch.int64)


def _prepare_append(case, gen):
    n, kv, hd, H, page = case["tokens"], case["kv"], case["hd"], case["heads"], case["page"]
    dt, rot = DTYPE[case["dtype"]], case["rot"]
    pages = -(-n // page) + 2                                   # one page is free, the last one takes nothing
    order = torch.randperm(pages - 1, generator=gen, device="cuda")
    at = torch.arange(n, device="cuda")
    slots = order[at // page] * page + at % page
    if case["padded"]:                                           # a thirteenth of the rows pads
        slots = torch.where(at % 13 == 5, -1, slots)
    inv = 500000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device="cuda") * 2.0 / rot)
    angle = torch.arange(case["far"], dtype=torch.float64, device="cuda")[:, None] * inv
    rope = torch.stack([torch.cos(angle), torch.sin(angle)], -1).float()
    first = torch.randint(0, max(1, case["far"] - n), (1,), generator=gen, device="cuda")
    positions = (first + at) % case["far"]
    if n <= 256:                                                 # a decode step: every token at a place of its own
        positions = torch.randint(0, case["far"], (n,), generator=gen, device="cuda")
    # queries, keys and values of a fused projection, side by side in a token's row
    qkv = torch.randn(n, H + 2 * kv, hd, generator=gen, device="cuda")
    qkv[:, H:H + kv, :: hd // 4] *= 4.0
    qkv[:, H + kv:] *= 0.5
    qkv = qkv.to(dt)
    s = {"case": dict(case), "cache": _empty_cache(pages, case), "slots": slots.contiguous(),
         "positions": positions.contiguous(), "rope": rope.contiguous(), "qkv": qkv,
         "q_out": torch.empty(n, H, hd, dtype=dt, device="cuda")}
    if case["fmt"] != "bf16":
        s["k_out"], s["v_out"] = (torch.empty(n, kv, hd, dtype=dt, device="cuda") for _ in range(2))
    return s


def _split_qkv(s):
    H, kv = s["case"]["heads"], s["case"]["kv"]
    return s["qkv"][:, :H], s["qkv"][:, H:H + kv], s["qkv"][:, H + kv:]


def prepare(case, seed):
    gen = _gen(seed)
    if case["kind"] == "append":
        return _prepare_append(case, gen)
    page, dt, B, H, hd = case["page"], DTYPE[case["dtype"]], case["batch"], case["heads"], case["hd"]
    lens, new = _lengths(case)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 2
    order = torch.randperm(pages - 1, generator=gen, device="cuda")     # pages as they were handed out
    width = max(1, max(need))
    take = torch.zeros(B, width, dtype=torch.int64)
    first = 0
    for b, n in enumerate(need):
        take[b, :n] = torch.arange(first, first + n)
        take[b, n:] = -1
        first += n
    take = take.cuda()
    table = torch.where(take >= 0, order[take.clamp(min=0)], -1).to(torch.int32)
    starts = [0]
    for k in new:
        starts.append(starts[-1] + k)
    lens_d = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pos = torch.arange(width * page, device="cuda")
    at = table.long()[:, pos // page] * page + pos % page       # [batch, width * page]
    every = at[pos < lens_d[:, None]]                            # slots of all tokens, sequence after sequence
    cache = _empty_cache(pages, case)
    for lo in range(0, every.numel(), ROWS):
        some = every[lo:lo + ROWS]
        k, v = _rows(gen, some.numel(), case)
        _plain_write(cache, case["fmt"], k, v, some)
    shape = {"sinks": (B,), "prompt": (starts[-1],), "tree": (B, case["new"])}[case["kind"]]
    s = {"case": dict(case), "cache": cache, "table": table, "lens": lens_d, "scale": 1.0 / math.sqrt(hd),
         "q": torch.randn(*shape, H, hd, generator=gen, device="cuda").to(dt),
         "out": torch.zeros(*shape, H, hd, dtype=dt, device="cuda"),
         "lse": torch.zeros(*shape, H, dtype=torch.float32, device="cuda"),
         "starts": torch.tensor(starts, dtype=torch.int32, device="cuda"),
         "counts": torch.tensor(new, dtype=torch.int32, device="cuda"), "most": max(new),
         "workspace": torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda")}
    if case["kind"] == "tree":
        s["tree"] = _trees(B, case["new"], seed).cuda()
    return s


# --------------------------------------------------------------------------
# the plain forms
# --------------------------------------------------------------------------

def _over(a, b):
    """a / b with b as a tensor on the device (a Python number would become a product with its reciprocal)."""
    return a / torch.full((), b, dtype=torch.float32, device=a.device)


def _plain_quantise(x, fmt):
    """x [n, kv, hd] -> (what the cache holds of its rows, their scales)."""
    x = x.float()
    if fmt == "bf16":
        return x.to(torch.bfloat16), None
    if fmt == "int8":
        amax = x.abs().amax(-1)
        amax = torch.where(amax < TINY, 0.0, amax)
        inv = torch.where(amax > 0, torch.full_like(amax, 127.0) / amax, 0.0)
        c = torch.round(x * inv[..., None])
        fine = torch.isfinite(amax)
        return (torch.where(fine[..., None], c, 0.0).to(torch.int8),
                torch.where(fine, _over(amax, 127.0), float("nan")))
    n, kv, hd = x.shape
    x = x.view(n, kv, hd // GROUP, GROUP)
    lo, hi = x.amin(-1), x.amax(-1)
    scale, low = _over(hi - lo, 15.0).to(torch.bfloat16), lo.to(torch.bfloat16)
    scale = torch.where(scale.float() < TINY, 0.0, scale)
    s, m = scale.float(), low.float()
    fine = torch.isfinite(s) & torch.isfinite(m)
    inv = torch.where(s > 0, torch.ones_like(s) / s, 0.0)
    c = torch.round((x - m[..., None]) * inv[..., None]).clamp(0, 15)
    c = torch.where(fine[..., None], c, 0.0).to(torch.uint8).view(n, kv, hd // 2, 2)
    pair = torch.where(fine[..., None], torch.stack([scale, low], -1), float("nan"))
    return c[..., 0] | c[..., 1] << 4, pair


def _plain_write(cache, fmt, k, v, slots):
    page = cache["k"].shape[2]
    slots = torch.where(slots < 0, cache["k"].shape[0] * page - 1, slots)      # the last page takes nothing else
    at, off = slots // page, slots % page
    k, v = _plain_quantise(k, fmt), _plain_quantise(v, fmt)
    cache["k"][at, :, off], cache["v"][at, :, off] = k[0], v[0]
    if fmt != "bf16":
        cache["k_scale"][at, :, off], cache["v_scale"][at, :, off] = k[1], v[1]


def _plain_rows(cache, name, fmt, slots):
    """fp32 values of the rows at `slots` (any shape, none negative) -> [*slots, kv, hd]."""
    page = cache[name].shape[2]
    at, off = slots // page, slots % page
    rows = cache[name][at, :, off]
    if fmt == "bf16":
        return rows.float()
    scale = cache[name + "_scale"][at, :, off].float()
    if fmt == "int8":
        return rows.float() * scale[..., None]
    c = torch.stack([rows & 15, rows >> 4], -1).float()
    c = c.view(*rows.shape[:-1], scale.shape[-2], GROUP)
    return (c * scale[..., :1] + scale[..., 1:]).flatten(-2)


def _plain_rotate(x, rope, rot):
    """x [n, heads, hd] -> fp32, the first `rot` channels rotated by rope [n, rot / 2, 2]."""
    x = x.float()
    a, b = x[..., :rot // 2], x[..., rot // 2:rot]
    c, s = rope[:, None, :, 0], rope[:, None, :, 1]
    return torch.cat([a * c - b * s, a * s + b * c, x[..., rot:]], -1)


def _plain_append(s):
    c = s["case"]
    q, k, v = _split_qkv(s)
    rope = s["rope"][s["positions"]]
    s["q_out"].copy_(_plain_rotate(q, rope, c["rot"]))
    _plain_write(s["cache"], c["fmt"], _plain_rotate(k, rope, c["rot"]), v, s["slots"])
    if c["fmt"] == "bf16":
        s["cache"]["k"][-1], s["cache"]["v"][-1] = float("nan"), float("nan")
        return
    there = (s["slots"] >= 0)[:, None, None]
    at = s["slots"].clamp(min=0)
    s["k_out"].copy_(torch.where(there, _plain_rows(s["cache"], "k", c["fmt"], at), 0.0))
    s["v_out"].copy_(torch.where(there, _plain_rows(s["cache"], "v", c["fmt"], at), 0.0))


def _plain_attend(s, q, at, there):
    """q [B, T, H, hd] over the rows at `at` [B, L] that are `there` [B, T, L] -> out [B, T, H, hd], lse [B, T, H], fp32."""
    c = s["case"]
    B, T, H, hd = q.shape
    kv, L = c["kv"], at.shape[1]
    seen = there.any(1)
    at = torch.where(seen, at, 0)
    k = torch.where(seen[..., None, None], _plain_rows(s["cache"], "k", c["fmt"], at), 0.0)    # [B, L, kv, hd]
    x = torch.matmul(q.float().view(B, T, kv, H // kv, hd).permute(0, 2, 3, 1, 4).reshape(B, kv, H // kv * T, hd),
                     k.permute(0, 2, 3, 1)).view(B, kv, H // kv, T, L)
    del k
    x = torch.where(there[:, None, None], x.mul_(s["scale"]), float("-inf"))
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    p = torch.exp_(x.sub_(m))
    total = p.sum(-1, keepdim=True)
    v = torch.where(seen[..., None, None], _plain_rows(s["cache"], "v", c["fmt"], at), 0.0)
    o = torch.matmul(p.view(B, kv, H // kv * T, L), v.permute(0, 2, 1, 3)).view(B, kv, H // kv, T, hd)
    o = torch.where(total == 0, 0.0, o / total)
    lse = torch.log(total) + m
    return o.permute(0, 3, 1, 2, 4).reshape(B, T, H, hd), lse[..., 0].permute(0, 3, 1, 2).reshape(B, T, H)


def _all_slots(s):
    """[B, L] positions' slots (0 where the table has none), and the positions [L]."""
    page, table = s["case"]["page"], s["table"].long()
    pos = torch.arange(table.shape[1] * page, device=table.device)
    return (table[:, pos // page] * page + pos % page).clamp(min=0), pos


def _plain_sinks(s):
    c, n = s["case"], s["lens"].long()[:, None]
    page, table = c["page"], s["table"].long()
    first = (n - c["window"]).clamp(min=0)                       # of the window
    i = torch.arange(c["sinks"] + c["window"], device=n.device)
    pos = torch.where(i < c["sinks"], i, first + i - c["sinks"])
    there = (pos < n) & ((i < c["sinks"]) | (pos >= c["sinks"]))
    pos = torch.where(there, pos, 0)
    at = table.gather(1, pos // page) * page + pos % page
    o, lse = _plain_attend(s, s["q"][:, None], at, there[:, None])
    s["out"].copy_(o[:, 0])
    s["lse"].copy_(lse[:, 0])


def _near(p, t, c):
    """Whether position t is in p's window or a sink."""
    return (t > p - c["window"]) | (t < c["sinks"]) if c["window"] else torch.ones_like(t > p)


def _plain_prompt(s):
    c, n, k = s["case"], s["lens"].long(), s["counts"].long()
    at, t = _all_slots(s)
    i = torch.arange(s["most"], device=n.device)
    p = (n - k)[:, None] + i                                     # [B, T]
    there = (t <= p[..., None]) & (i < k[:, None])[..., None] & _near(p[..., None], t, c)
    row = (s["starts"][:-1].long()[:, None] + i).clamp(max=s["q"].shape[0] - 1)
    o, lse = _plain_attend(s, s["q"][row], at, there)
    real = i < k[:, None]
    s["out"].copy_(o[real])
    s["lse"].copy_(lse[real])


def _plain_tree(s):
    c, n, k = s["case"], s["lens"].long(), s["counts"].long()
    at, t = _all_slots(s)
    T = s["q"].shape[1]
    j = torch.arange(T, device=n.device)
    bit = (s["tree"][..., None] >> j & 1).bool() & (j < k[:, None])[:, None]       # [B, T, T]: j is an ancestor of i, or i
    depth = bit.sum(-1) - 1
    ctx = (n - k)[:, None]
    p = ctx + depth                                              # [B, T]
    draft = t - ctx                                              # [B, L]
    is_draft = (draft >= 0) & (draft < k[:, None])
    d = draft.clamp(0, T - 1)
    pos = torch.where(is_draft, p.gather(1, d), t)
    sees = torch.where(is_draft[:, None], bit.gather(2, d[:, None].expand(-1, T, -1)), (draft < 0)[:, None])
    there = sees & _near(p[..., None], pos[:, None], c)
    real = (j < k[:, None])[..., None]
    o, lse = _plain_attend(s, s["q"], at, there & real)
    s["out"].copy_(torch.where(real[..., None], o, s["out"].float()))
    s["lse"].copy_(torch.where(real, lse, s["lse"]))


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        from paper_2506_03781_gb300 import api
        if kind == "append":
            q, k, v = _split_qkv(s)
            api.uq_kv_append(s["cache"], k, v, s["slots"], s["positions"], s["rope"], q=q, q_out=s["q_out"])
            if c["fmt"] != "bf16":
                api.uq_kv_read(s["cache"], s["slots"], s["k_out"], s["v_out"])
        else:
            more = dict(lse=s["lse"], scale=s["scale"], window=c["window"], sinks=c["sinks"], workspace=s["workspace"])
            if kind == "sinks":
                api.uq_paged_attn_sinks(s["cache"], s["q"], s["table"], s["lens"], s["out"], **more)
            elif kind == "prompt":
                api.uq_paged_prompt_attn(s["cache"], s["q"], s["starts"], s["table"], s["lens"], s["out"], **more)
            else:
                api.uq_paged_tree_attn(s["cache"], s["q"], s["tree"], s["table"], s["lens"], s["out"],
                                       counts=s["counts"], **more)
    else:
        {"append": _plain_append, "sinks": _plain_sinks, "prompt": _plain_prompt, "tree": _plain_tree}[kind](s)
    if kind != "append":
        return {"out": s["out"], "lse": s["lse"]}
    if c["fmt"] == "bf16":
        return {"q": s["q_out"], "k": s["cache"]["k"], "v": s["cache"]["v"]}
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


# --------------------------------------------------------------------------
# the work
# --------------------------------------------------------------------------

def _row_bytes(case):
    hd = case["hd"]
    return {"bf16": 2 * hd, "int8": hd + 4, "int4": hd // 2 + 4 * (hd // GROUP)}[case["fmt"]]


def _seen(case, n, k):
    """(cache rows that any of the k new of n tokens sees, sum over them of how many each sees)."""
    w, s = case["window"] or n, case["sinks"]
    one = lambda p: min(p + 1, w) + min(s, max(0, p + 1 - w))    # what position p sees of a causal sequence
    if k <= 0:
        return 0, 0
    if case["kind"] == "tree":                                   # a draft sees about what a token at its depth would
        ctx = n - k
        return one(ctx - 1) + k, k * one(ctx - 1) + k * (1 + math.log2(k))
    first = max(0, n - k + 1 - w)                                # start of the first new token's window
    return n - first + min(s, first), sum(one(p) for p in range(n - k, n))


def work(case):
    kv, hd, w, row, H = case["kv"], case["hd"], WIDTH[case["dtype"]], _row_bytes(case), case["heads"]
    if case["kind"] == "append":
        n = case["tokens"]
        used = n - len(range(5, n, 13)) if case["padded"] else n
        moved = n * (2 * H * hd * w + 16) + used * 2 * kv * (hd * w + row) + min(n, case["far"]) * case["rot"] * 4
        if case["fmt"] != "bf16":                                # read back
            moved += n * (2 * kv * hd * w + 8)
        return {"bytes": moved, "flops": n * (H + kv) * case["rot"] * 3}
    lens, new = _lengths(case)
    seen = [_seen(case, n, k) for n, k in zip(lens, new)]
    rows, pairs = sum(r for r, _ in seen), sum(p for _, p in seen)
    moved = rows * 2 * kv * row + sum(new) * H * (2 * hd * w + 4) + 4 * rows // case["page"]
    return {"bytes": moved, "flops": int(4 * pairs * H * hd)}


# --------------------------------------------------------------------------
# in 64 bits
# --------------------------------------------------------------------------

def _exact_new(x, fmt):
    """The values that a row of new tokens stands for once it is stored. A 64-bit quotient, product or difference is
    rounded to fp32 where the definition has it so: that rounding decides codes (48 bits of a product are exact here)."""
    f32 = lambda t: t.float().double()
    d = x.double()
    if fmt == "bf16":
        return x.to(torch.bfloat16).double()
    if fmt == "int8":
        top = d.abs().max(-1, keepdim=True).values
        step, per = f32(top / 127), f32(127 / top)
        return torch.where(top < TINY, 0.0, f32(d * per).round() * step)
    g = d.unflatten(-1, (-1, GROUP))
    low, high = g.min(-1, keepdim=True).values, g.max(-1, keepdim=True).values
    step = f32(f32(high - low) / 15).to(torch.bfloat16).double()
    base = low.to(torch.bfloat16).double()
    code = torch.where(step < TINY, 0.0, f32(f32(g - base) * f32(1 / step)).round().clamp(0, 15))
    return (code * step + base).flatten(-2)


def _exact_kept(cache, name, fmt, slots):
    """The values of the rows at `slots` [n], in 64 bits -> [kv, n, hd]."""
    page = cache[name].shape[2]
    pick = lambda t: t[torch.div(slots, page, rounding_mode="floor"), :, slots % page].transpose(0, 1)
    rows = pick(cache[name])
    if fmt == "bf16":
        return rows.double()
    scales = pick(cache[name + "_scale"]).double()
    if fmt == "int8":
        return rows.double() * scales.unsqueeze(-1)
    codes = torch.empty(*rows.shape[:2], 2 * rows.shape[2], dtype=torch.float64, device=rows.device)
    codes[..., 0::2] = (rows % 16).double()
    codes[..., 1::2] = (rows // 16).double()
    codes = codes.unflatten(-1, (-1, GROUP))
    return (codes * scales[..., 0:1] + scales[..., 1:2]).flatten(-2)


def _exact_append(s, case):
    f32 = lambda t: t.float().double()
    H, kv, hd, rot = case["heads"], case["kv"], case["hd"], case["rot"]
    x = s["qkv"][:, :H + kv].double()
    at = s["rope"].double().index_select(0, s["positions"])
    cos, sin = at[:, None, :, 0], at[:, None, :, 1]
    turned = x.clone()
    lo, hi = x[:, :, :rot // 2], x[:, :, rot // 2:rot]
    turned[:, :, :rot // 2] = f32(f32(lo * cos) - f32(hi * sin))
    turned[:, :, rot // 2:rot] = f32(f32(lo * sin) + f32(hi * cos))
    k = _exact_new(turned[:, H:].float(), case["fmt"])
    v = _exact_new(s["qkv"][:, H + kv:], case["fmt"])
    if case["fmt"] != "bf16":
        k[s["slots"] < 0], v[s["slots"] < 0] = 0, 0
        return {"q": turned[:, :H], "k": k, "v": v}
    whole = []
    keep = s["slots"] >= 0
    for rows in (k, v):
        pool = torch.full(s["cache"]["k"].shape, float("nan"), dtype=torch.float64, device="cuda")
        flat = pool.transpose(1, 2).reshape(-1, kv, hd)
        flat[s["slots"][keep]] = rows[keep]
        whole.append(flat.view(pool.shape[0], case["page"], kv, hd).transpose(1, 2).contiguous())
    return {"q": turned[:, :H], "k": whole[0], "v": whole[1]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "append":
        return _exact_append(s, case)
    page, H, hd, kv, kind = case["page"], case["heads"], case["hd"], case["kv"], case["kind"]
    lens, new = _lengths(case)
    out, lse = s["out"].double(), s["lse"].double()
    w, sinks = case["window"], case["sinks"]
    first = 0
    for b, (n, k) in enumerate(zip(lens, new)):
        into = (out[b:b + 1], lse[b:b + 1]) if kind == "sinks" else (
            (out[first:first + k], lse[first:first + k]) if kind == "prompt" else (out[b, :k], lse[b, :k]))
        queries = (s["q"][b:b + 1] if kind == "sinks" else s["q"][first:first + k] if kind == "prompt" else s["q"][b, :k])
        first += k
        if k == 0:
            if kind == "sinks":
                into[1].fill_(float("-inf"))
            continue
        ctx = n - k
        place = torch.arange(n, device="cuda")                   # a cached token's distance from the start
        mine = place[ctx:].clone()                               # a new token's
        sees = place[None, :] <= mine[:, None]                   # [k, n]
        if kind == "tree":
            sees[:, ctx:] = False
            for i, m in enumerate(s["tree"][b, :k].tolist()):
                kin = [j for j in range(k) if m >> j & 1]
                sees[i, [ctx + j for j in kin]] = True
                mine[i] = ctx + len(kin) - 1
            place = torch.cat([place[:ctx], mine])
        if w:
            sees &= (mine[:, None] - place[None, :] < w) | (place[None, :] < sinks)
        used = sees.any(0).nonzero()[:, 0]
        sees = sees[:, used]
        slots = s["table"][b].long()[torch.div(used, page, rounding_mode="floor")] * page + used % page
        K, V = (_exact_kept(s["cache"], name, case["fmt"], slots) for name in ("k", "v"))      # [kv, n, hd]
        r = H // kv
        for h in range(kv):
            for lo in range(0, k, 1024):
                q = queries[lo:lo + 1024, h * r:(h + 1) * r].double()                           # [t, r, hd]
                x = (q.reshape(-1, hd) @ K[h].T * s["scale"]).view(-1, r, used.numel())
                x = torch.where(sees[lo:lo + 1024, None], x, float("-inf"))
                into[1][lo:lo + 1024, h * r:(h + 1) * r] = torch.logsumexp(x, -1)
                p = torch.softmax(x, -1).nan_to_num(0.0)
                into[0][lo:lo + 1024, h * r:(h + 1) * r] = (p.flatten(0, 1) @ V[h]).view(-1, r, hd)
    return {"out": out, "lse": lse}
