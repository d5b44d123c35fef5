"""What the serving operators of this framework are timed on: a paged key-value
cache that is quantised as it is written, read back, and attended over by one
new token per sequence.

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

Kinds of a case:

* "attend"  one new token of every sequence attends over its cached tokens
            (grouped queries, optionally only the last `window` tokens);
* "step"    a decode step's cache work: the new tokens' keys and values are
            written, then attended over together with the older ones;
* "prompt"  prompts' keys and values are written and read back, as the
            prompts' own attention sees them;
* "read"    a cached prefix is read back.
"""

import math
import random

import torch

own = False

WIDTH = {"bf16": 2, "f32": 4}
DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 64                                  # channels of an int4 group
TINY = 2.0 ** -100                          # smaller ranges are kept as zeros
WORKSPACE = 32 << 20                        # bytes of scratch that a serving program keeps for its attention calls
ROWS = 1 << 16                              # cache rows that prepare() fills at a time


def _attend(name, kind, batch, length, fmt, dtype, heads, kv, hd, page, ragged, window=0):
    return dict(name=name, kind=kind, batch=batch, length=length, fmt=fmt, dtype=dtype, heads=heads, kv=kv, hd=hd,
                page=page, ragged=ragged, window=window)


def _tokens(name, kind, tokens, fmt, dtype, kv, hd, page, padded=False):
    return dict(name=name, kind=kind, tokens=tokens, fmt=fmt, dtype=dtype, kv=kv, hd=hd, page=page, padded=padded)


def listed():
    return [
        # one user's short chat on the 8B block (32 heads, 8 key/value heads of 128): latency counts
        _attend("attend_1x300_bf16", "attend", 1, 300, "bf16", "bf16", 32, 8, 128, 16, False),
        # one user's long document, fp32 queries as the deployment product writes them
        _attend("attend_1x131000_int8_f32", "attend", 1, 131000, "int8", "f32", 32, 8, 128, 64, False),
        # a server's batch of requests of very different lengths, unquantised cache in small pages
        _attend("attend_64_ragged_bf16", "attend", 64, 8192, "bf16", "bf16", 32, 8, 128, 16, True),
        # a full server of the 70B shape (64 heads, 8 key/value heads) on the smallest cache
        _attend("attend_128x4096_int4", "attend", 128, 4096, "int4", "bf16", 64, 8, 128, 32, False),
        # as many key/value heads as heads, of 64 channels
        _attend("attend_48_mha64_int8", "attend", 48, 2047, "int8", "bf16", 16, 16, 64, 16, True),
        # 16 heads share one key/value head of 256 channels; the last 4096 tokens only
        _attend("attend_16_window_hd256", "attend", 16, 9000, "bf16", "bf16", 16, 1, 256, 64, False, window=4096),
        # a decode step of a small batch
        _attend("step_16_int8", "step", 16, 1000, "int8", "bf16", 32, 8, 128, 16, True),
        # a decode step of a large batch, fp32 activations
        _attend("step_256_int4_f32", "step", 256, 2048, "int4", "f32", 32, 8, 128, 64, True),
        # a chunk of a prompt between decode steps
        _tokens("prompt_33_int8", "prompt", 33, "int8", "bf16", 8, 128, 16),
        # one sample of the reconstruction's length
        _tokens("prompt_2048_bf16_int8", "prompt", 2048, "int8", "bf16", 8, 128, 16),
        # several prompts packed and padded, fp32
        _tokens("prompt_20011_f32_int4", "prompt", 20011, "int4", "f32", 8, 128, 64, padded=True),
        # a long shared prefix is read back for the attention of the prompt that follows it
        _tokens("read_60000_int4", "read", 60000, "int4", "bf16", 8, 128, 32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Kinds as listed: 1 to 256 sequences of 1 to 131072 tokens (2^18 in all at most, of 8 heads of 128 in int4), any
    number of heads from 1 to 16 per key/value head, pages of 16 to 128 tokens; 1 to 32768 tokens written or read."""
    kind = rng.choice(["attend", "attend", "attend", "step", "step", "prompt", "prompt", "read"])
    fmt, dtype = rng.choice(["bf16", "int8", "int4"]), rng.choice(["bf16", "bf16", "f32"])
    hd = rng.choice([64, 128, 128, 128, 256])
    kv = rng.choice([1, 2, 4, 5, 8, 8, 16]) if hd < 256 else rng.choice([1, 2, 4])
    page = rng.choice([16, 16, 32, 64, 128])
    if kind in ("attend", "step"):
        batch = _log(rng, 1, 256)
        # half of the largest case's cached values: bf16 takes over three times the bytes of int4
        most = 2 ** 28 // (kv * hd * (4 if fmt == "bf16" else 2 if fmt == "int8" else 1))
        length = min(_log(rng, 1, 131072), max(1, most // batch))
        heads = kv * rng.choice([1, 2, 3, 4, 4, 6, 7, 8, 8, 12, 16])
        window = _log(rng, 1, length) if rng.random() < 0.2 else 0
        c = _attend("", kind, batch, length, fmt, dtype, heads, kv, hd, page, rng.random() < 0.6, window)
    else:
        tokens = min(_log(rng, 1, 32768), 2 ** 25 // (kv * hd))
        c = _tokens("", kind, tokens, fmt, dtype, kv, hd, page, rng.random() < 0.3)
    del c["name"]
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _lengths(case):
    """Every sequence's number of tokens: `length`, or spread over 1..length by logarithm, with one empty sequence
    (an idle place of the server's batch) where there are at least four and nothing is written."""
    B, n = case["batch"], case["length"]
    if not case["ragged"]:
        return [n] * B
    r = random.Random(B * 1000003 + n)
    lens = [_log(r, 1, n) for _ in range(B)]
    lens[r.randrange(B)] = n
    if B >= 4 and case["kind"] == "attend":
        lens[r.randrange(B)] = 0
    return lens


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


def prepare(case, seed):
    gen = _gen(seed)
    page, dt = case["page"], DTYPE[case["dtype"]]
    kv, hd = case["kv"], case["hd"]
    lens = _lengths(case) if case["kind"] in ("attend", "step") else [case["tokens"]]
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 2                                        # one page is free, the last one takes nothing
    order = torch.randperm(pages - 1, generator=gen, device="cuda")     # pages as they were handed out
    width = max(1, max(need))
    take = torch.zeros(len(lens), width, dtype=torch.int64)
    first = 0
    for b, n in enumerate(need):
        take[b, :n] = torch.arange(first, first + n)
        take[b, n:] = -1
        first += n
    take = take.cuda()
    table = torch.where(take >= 0, order[take.clamp(min=0)], -1).to(torch.int32)
    lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pos = torch.arange(width * page, device="cuda")
    at = table.long()[:, pos // page] * page + pos % page       # [batch, width * page]
    every = at[pos < lens[:, None]]                              # slots of all tokens, sequence after sequence
    cache = _empty_cache(pages, case)
    s = {"case": dict(case), "cache": cache}
    if case["kind"] != "prompt":                                 # what is in the cache already
        for lo in range(0, every.numel(), ROWS):
            some = every[lo:lo + ROWS]
            k, v = _rows(gen, some.numel(), case)
            _plain_write(cache, case["fmt"], k, v, some)
    if case["kind"] in ("attend", "step"):
        B, H = case["batch"], case["heads"]
        s.update(table=table, lens=lens, scale=1.0 / math.sqrt(hd),
                 q=torch.randn(B, H, hd, generator=gen, device="cuda").to(dt),
                 out=torch.empty(B, H, hd, dtype=dt, device="cuda"),
                 lse=torch.empty(B, H, dtype=torch.float32, device="cuda"),
                 workspace=torch.empty(WORKSPACE, dtype=torch.uint8, device="cuda"))
    if case["kind"] == "step":
        last = (lens.long() - 1)[:, None]
        s["slots"] = at.gather(1, last)[:, 0].contiguous()
        s["k"], s["v"] = _rows(gen, case["batch"], case)
    if case["kind"] in ("prompt", "read"):
        n = case["tokens"]
        if case["padded"]:                                       # a thirteenth of the rows pads
            every = torch.where(torch.arange(n, device="cuda") % 13 == 5, -1, every)
        s["slots"] = every.contiguous()
        s["k_out"], s["v_out"] = (torch.empty(n, kv, hd, dtype=dt, device="cuda") for _ in range(2))
        if case["kind"] == "prompt":
            s["k"], s["v"] = _rows(gen, n, case)
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
    for name, x in (("k", k), ("v", v)):
        rows, scales = _plain_quantise(x, fmt)
        cache[name][at, :, off] = rows
        if scales is not None:
            cache[name + "_scale"][at, :, off] = scales


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


def _plain_read(s):
    slots, fmt = s["slots"], s["case"]["fmt"]
    there = (slots >= 0)[:, None, None]
    for name in ("k", "v"):
        s[name + "_out"].copy_(torch.where(there, _plain_rows(s["cache"], name, fmt, slots.clamp(min=0)), 0.0))


def _plain_attend(s):
    c, cache, q, table, lens = s["case"], s["cache"], s["q"], s["table"].long(), s["lens"]
    B, H, hd = q.shape
    kv, page = c["kv"], c["page"]
    pos = torch.arange(table.shape[1] * page, device=q.device)
    at = table[:, pos // page] * page + pos % page
    first = lens - c["window"] if c["window"] else torch.zeros_like(lens)
    there = (pos < lens[:, None]) & (pos >= first[:, None]) & (at >= 0)
    at = at.clamp(min=0)
    k = _plain_rows(cache, "k", c["fmt"], at)                                  # [B, L, kv, hd]
    x = torch.einsum("bgrd,blgd->bgrl", q.float().view(B, kv, H // kv, hd), k) * s["scale"]
    del k
    x = torch.where(there[:, None, None], x, float("-inf"))
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), 0.0, m)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    v = torch.where(there[:, :, None, None], _plain_rows(cache, "v", c["fmt"], at), 0.0)
    o = torch.einsum("bgrl,blgd->bgrd", p, v)
    o = torch.where(total == 0, 0.0, o / total)
    s["out"].copy_(o.reshape(B, H, hd))
    s["lse"].copy_((torch.log(total) + m).reshape(B, H))


def run(s):
    kind = s["case"]["kind"]
    if own:
        from paper_2506_03781_gb300 import api
        if kind in ("prompt", "step"):
            api.uq_kv_write(s["cache"], s["k"], s["v"], s["slots"])
        if kind in ("prompt", "read"):
            api.uq_kv_read(s["cache"], s["slots"], s["k_out"], s["v_out"])
        else:
            api.uq_paged_attn(s["cache"], s["q"], s["table"], s["lens"], s["out"], lse=s["lse"], scale=s["scale"],
                              window=s["case"]["window"], workspace=s["workspace"])
    else:
        if kind in ("prompt", "step"):
            _plain_write(s["cache"], s["case"]["fmt"], s["k"], s["v"], s["slots"])
        _plain_read(s) if kind in ("prompt", "read") else _plain_attend(s)
    return {"k": s["k_out"], "v": s["v_out"]} if kind in ("prompt", "read") else {"out": s["out"], "lse": s["lse"]}


def _row_bytes(case):
    hd = case["hd"]
    return {"bf16": 2 * hd, "int8": hd + 4, "int4": hd // 2 + 4 * (hd // GROUP)}[case["fmt"]]


def work(case):
    kv, hd, w, row = case["kv"], case["hd"], WIDTH[case["dtype"]], _row_bytes(case)
    if case["kind"] in ("prompt", "read"):
        n = case["tokens"]
        used = n - len(range(5, n, 13)) if case["padded"] else n
        dense = 2 * kv * hd * w
        ins = used * dense if case["kind"] == "prompt" else 0
        return {"bytes": ins + used * 2 * kv * row + n * dense + 8 * n, "flops": used * 2 * kv * hd * 2}
    lens = _lengths(case)
    seen = sum(min(n, case["window"]) if case["window"] else n for n in lens)
    B, H = case["batch"], case["heads"]
    moved = seen * 2 * kv * row + B * H * (2 * hd * w + 4) + 4 * B + 4 * sum(-(-n // case["page"]) for n in lens)
    if case["kind"] == "step":
        moved += B * 2 * kv * hd * w
    return {"bytes": moved, "flops": 4 * seen * H * hd}


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
    """The values of the rows at `slots` [n], in 64 bits -> [n, kv, hd]."""
    page = cache[name].shape[2]
    pick = lambda t: t.transpose(1, 2).flatten(0, 1)[slots]
    rows = pick(cache[name])
    assert cache[name].shape[2] == page
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


def exact(case, seed):
    s = prepare(case, seed)
    cache, fmt, page = s["cache"], case["fmt"], case["page"]
    if case["kind"] in ("prompt", "read"):
        answer = {}
        for name in ("k", "v"):
            if case["kind"] == "prompt":
                val = _exact_new(s[name], fmt)
            else:
                val = _exact_kept(cache, name, fmt, s["slots"].clamp(min=0))
            val[s["slots"] < 0] = 0
            answer[name] = val
        return answer
    B, H, hd, kv = case["batch"], case["heads"], case["hd"], case["kv"]
    out = torch.zeros(B, H, hd, dtype=torch.float64, device="cuda")
    lse = torch.full((B, H), float("-inf"), dtype=torch.float64, device="cuda")
    fresh = {n: _exact_new(s[n], fmt) for n in ("k", "v")} if case["kind"] == "step" else None
    for b, n in enumerate(s["lens"].tolist()):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n <= first:
            continue
        pos = torch.arange(first, n, device="cuda")
        slots = s["table"][b].long()[torch.div(pos, page, rounding_mode="floor")] * page + pos % page
        K, V = (_exact_kept(cache, name, fmt, slots).transpose(0, 1) for name in ("k", "v"))     # [kv, n, hd]
        if fresh is not None:
            K, V = K.clone(), V.clone()
            K[:, -1], V[:, -1] = fresh["k"][b], fresh["v"][b]
        x = s["q"][b].double().unflatten(0, (kv, -1)) @ K.transpose(1, 2) * s["scale"]          # [kv, r, n]
        lse[b] = torch.logsumexp(x, -1).flatten()
        out[b] = (torch.softmax(x, -1) @ V).flatten(0, 1)
    return {"out": out, "lse": lse}
