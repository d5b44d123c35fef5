"""uq_kv_write and uq_kv_read on the GPU against the oracle's rows: codes,
scales and values are equal bit for bit (both sides take the same fp32
roundings)."""

import numpy as np
import pytest
import torch

from oracle import kv as OK
from paper_2506_03781_gb300 import api
from tests import kv_cases as C

pytestmark = pytest.mark.gpu
F32 = np.float32
FORMATS, HEADS = ("bf16", "int8", "int4"), (64, 128, 256)


def same(a, b):
    return all((x is None and y is None) or np.array_equal(x, y, equal_nan=True) for x, y in zip(a, b))


def write(fmt, dtype, k, v, slots, kv, page, pages, hd):
    cache = api.empty_kv_cache(pages, kv, page, hd, C.FMT[fmt], C.dev())
    C.poison(cache)
    kt, kx = C.typed(k, dtype)
    vt, vx = C.typed(v, dtype)
    api.uq_kv_write(cache, kt, vt, torch.from_numpy(slots).to(C.dev()))
    torch.cuda.synchronize()
    return cache, kx, vx


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hd", HEADS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("n,kv,page", [(1, 1, 16), (1, 8, 64), (7, 3, 16), (33, 8, 32), (130, 5, 256), (1000, 2, 128)])
def test_write_and_read_back(fmt, hd, dtype, n, kv, page):
    rng = np.random.default_rng(n + hd)
    pages = -(-n // page) + 2
    slots = rng.permutation(pages * page)[:n].astype(np.int64)
    k, v = (rng.standard_t(4, (n, kv, hd)).astype(F32) for _ in range(2))
    cache, kx, vx = write(fmt, dtype, k, v, slots, kv, page, pages, hd)
    rest = np.setdiff1d(np.arange(pages * page), slots)
    for name, x in (("k", kx), ("v", vx)):
        ref = OK.quantise_rows(x, fmt)
        assert same(C.cache_rows(cache, fmt, name, slots), ref), name
        # what no slot names keeps its bits
        codes, scales, minima = C.cache_rows(cache, fmt, name, rest)
        for part in (codes if fmt == "bf16" else None, scales, minima):
            assert part is None or np.isnan(part).all()
        if fmt != "bf16":
            assert (codes == (-1 if fmt == "int8" else 15)).all()
        for out in ("f32", "bf16"):
            ko, vo = (torch.full((n, kv, hd), 7.0, dtype=C.DT[out], device=C.dev()) for _ in range(2))
            api.uq_kv_read(cache, torch.from_numpy(slots).to(C.dev()), ko, vo)
            got = (ko if name == "k" else vo).float().cpu().numpy()
            val = OK.row_values(ref, fmt).astype(F32)            # one rounding of the exact value
            assert np.array_equal(got, OK.to_bf16(val) if out == "bf16" else val)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_slots_that_are_not_in_the_pool(fmt, dtype):
    n, kv, page, pages, hd = 40, 4, 16, 3, 128
    rng = np.random.default_rng(3)
    k, v = (rng.standard_normal((n, kv, hd)).astype(F32) for _ in range(2))
    slots = rng.permutation(pages * page)[:n].astype(np.int64)
    bad = np.arange(n) % 3 == 1
    slots[bad] = rng.choice([-1, -2 ** 63, pages * page, pages * page + 5, 2 ** 62, 2 ** 63 - 1], bad.sum())
    cache, kx, vx = write(fmt, dtype, k, v, slots, kv, page, pages, hd)
    for name, x in (("k", kx), ("v", vx)):
        assert same(C.cache_rows(cache, fmt, name, slots[~bad]), OK.quantise_rows(x[~bad], fmt))
    ko, vo = (torch.full((n, kv, hd), float("nan"), device=C.dev()) for _ in range(2))
    api.uq_kv_read(cache, torch.from_numpy(slots).to(C.dev()), ko, vo)
    for got, x in ((ko, kx), (vo, vx)):
        got = got.cpu().numpy()
        assert (got[bad] == 0).all()
        assert np.array_equal(got[~bad], OK.row_values(OK.quantise_rows(x[~bad], fmt), fmt).astype(F32))


SPECIAL = {
    "zeros": lambda x: x * 0, "negative zeros": lambda x: -(x * 0), "constant": lambda x: x * 0 + F32(0.37),
    "one nan": lambda x: _set(x, 17, np.nan), "one inf": lambda x: _set(x, 40, np.inf), "-inf": lambda x: _set(x, 5, -np.inf),
    "both infinities": lambda x: _set(_set(x, 5, -np.inf), 6, np.inf), "all inf": lambda x: x * 0 + F32(np.inf),
    "tiny": lambda x: x * F32(1e-32), "just not tiny": lambda x: x * F32(1e-29), "subnormal": lambda x: x * F32(1e-40),
    "huge": lambda x: x / np.abs(x).max() * F32(3.0e38), "largest": lambda x: np.sign(x) * F32(3.3895e38),
    "positive only": lambda x: np.abs(x) + F32(3), "one outlier": lambda x: _set(x, 3, 1e4),
    "ties": lambda x: np.round(x * 8) / 8,
}


def _set(x, i, v):
    x = x.copy()
    x[..., i] = v
    return x


@pytest.mark.parametrize("what", sorted(SPECIAL))
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_special_rows(what, fmt, dtype):
    n, kv, page, hd = 5, 2, 16, 128
    rng = np.random.default_rng(11)
    base = rng.standard_normal((n, kv, hd)).astype(F32)
    with np.errstate(all="ignore"):
        x = SPECIAL[what](base).astype(F32)
    x[1] = base[1]                                    # its neighbours are ordinary rows
    slots = np.arange(n, dtype=np.int64) + 3
    cache, kx, vx = write(fmt, dtype, x, -x, slots, kv, page, 2, hd)
    ko, vo = (torch.empty(n, kv, hd, device=C.dev()) for _ in range(2))
    api.uq_kv_read(cache, torch.from_numpy(slots).to(C.dev()), ko, vo)
    for name, xx, got in (("k", kx, ko), ("v", vx, vo)):
        ref = OK.quantise_rows(xx, fmt)
        assert same(C.cache_rows(cache, fmt, name, slots), ref)
        with np.errstate(all="ignore"):
            assert np.array_equal(got.cpu().numpy(), OK.row_values(ref, fmt).astype(F32), equal_nan=True)


@pytest.mark.parametrize("fmt", FORMATS)
def test_strided_rows(fmt):
    """Slices of a fused projection in, heads-first tensors out."""
    n, kv, hd, page = 19, 3, 64, 16
    rng = np.random.default_rng(5)
    fused, x = C.typed(rng.standard_normal((n, 4 * kv, hd)), "bf16")
    k, v = fused[:, kv:2 * kv], fused[:, 3 * kv:]
    cache = api.empty_kv_cache(3, kv, page, hd, C.FMT[fmt], C.dev())
    slots = rng.permutation(3 * page)[:n].astype(np.int64)
    every = torch.from_numpy(np.concatenate([[9], slots])).to(C.dev())
    api.uq_kv_write(cache, k, v, every[1:])           # 8-byte aligned slots
    ko, vo = (torch.full((kv, n + 2, hd), 5.0, device=C.dev()) for _ in range(2))
    api.uq_kv_read(cache, every[1:], ko[:, 1:-1].transpose(0, 1), vo[:, 1:-1].transpose(0, 1))
    for got, lo in ((ko, kv), (vo, 3 * kv)):
        val = OK.row_values(OK.quantise_rows(x[:, lo:lo + kv], fmt), fmt).astype(F32).transpose(1, 0, 2)
        assert np.array_equal(got[:, 1:-1].cpu().numpy(), val)
        assert (got[:, 0] == 5).all() and (got[:, -1] == 5).all()
    # one key row for every head (a broadcast input): read, never written
    one = fused[:, :1].expand(n, kv, hd)
    api.uq_kv_write(cache, one, one, every[1:])
    assert same(C.cache_rows(cache, fmt, "k", slots),
                OK.quantise_rows(np.broadcast_to(x[:, :1], (n, kv, hd)), fmt))


def test_no_tokens_is_no_work():
    cache = api.empty_kv_cache(1, 2, 16, 64, api.KV_INT8, C.dev())
    C.poison(cache)
    none = torch.empty(0, 2, 64, device=C.dev())
    slots = torch.empty(0, dtype=torch.int64, device=C.dev())
    api.uq_kv_write(cache, none, none, slots)
    api.uq_kv_read(cache, slots, none, none)
    torch.cuda.synchronize()
    assert (cache["k"] == -1).all() and torch.isnan(cache["k_scale"]).all()


def test_rows_beyond_32_bit_offsets():
    """A pool of 2^32 bytes and more per tensor: the last page is written, read and nothing else changes."""
    kv, page, hd = 8, 256, 256
    pages = 2 ** 32 // (kv * page * hd * 2) + 3
    cache = api.empty_kv_cache(pages, kv, page, hd, api.KV_BF16, C.dev())
    for t in cache.values():
        t.zero_()
    n = 3
    k, kx = C.typed(np.random.default_rng(0).standard_normal((n, kv, hd)) + 10, "f32")
    slots = torch.tensor([pages * page - 1, pages * page - 2, 2 ** 32 // (kv * hd * 2) + 7], device=C.dev())
    api.uq_kv_write(cache, k, k, slots)
    ko, vo = torch.empty_like(k), torch.empty_like(k)
    api.uq_kv_read(cache, slots, ko, vo)
    assert np.array_equal(ko.cpu().numpy(), OK.to_bf16(kx)) and torch.equal(ko, vo)
    assert int((cache["k"] != 0).sum()) == n * kv * hd
    del cache


def test_refusals():
    d = C.dev()
    cache = api.empty_kv_cache(2, 2, 16, 64, api.KV_INT8, d)
    k = torch.zeros(3, 2, 64, device=d)
    slots = torch.zeros(3, dtype=torch.int64, device=d)
    with pytest.raises(ValueError, match="slots"):
        api.uq_kv_write(cache, k, k, slots.int())
    with pytest.raises(ValueError, match="slots"):
        api.uq_kv_write(cache, k, k, slots[:2])
    with pytest.raises(ValueError, match="v has"):
        api.uq_kv_write(cache, k, k.bfloat16(), slots)
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        api.uq_kv_write(cache, k.half(), k.half(), slots)
    with pytest.raises(ValueError, match="k has shape"):
        api.uq_kv_write(cache, k[:, :1], k, slots)
    with pytest.raises(ValueError, match="contiguous rows"):
        t = torch.zeros(3, 64, 2, device=d).transpose(1, 2)
        api.uq_kv_write(cache, t, t, slots)
    with pytest.raises(ValueError, match="k_scale"):
        api.uq_kv_write({**cache, "k_scale": cache["k_scale"].half()}, k, k, slots)
    with pytest.raises(ValueError, match="must be on"):
        api.uq_kv_write(cache, k.cpu(), k, slots)
    with pytest.raises(api.UQError) as e:                          # rows that are no multiple of 16 bytes apart
        t = torch.zeros(3, 2, 66, device=d)[..., :64]
        api.uq_kv_write(cache, t, t, slots)
    assert e.value.status == api.UQ_ERR_ALIGN
    with pytest.raises(api.UQError) as e:                          # outputs that overlap
        t = torch.zeros(1, 2, 64, device=d).expand(3, 2, 64)
        api.uq_kv_read(cache, slots, t, k)
    assert e.value.status == api.UQ_ERR_ARG and "overlap" in str(e.value)
    for shape, status in (((2, 2, 24, 64), api.UQ_ERR_UNSUPPORTED), ((2, 2, 8, 64), api.UQ_ERR_UNSUPPORTED),
                          ((2, 2, 16, 96), api.UQ_ERR_UNSUPPORTED)):
        c = api.empty_kv_cache(*shape, api.KV_BF16, d)
        t = torch.zeros(3, 2, shape[3], device=d)
        with pytest.raises(api.UQError) as e:
            api.uq_kv_write(c, t, t, slots)
        assert e.value.status == status
