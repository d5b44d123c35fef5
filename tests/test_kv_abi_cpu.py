"""Refusals of the key-value cache's C entry points, before anything is
launched (fake pointers: only where there is no GPU)."""

import pytest
import torch

from paper_2506_03781_gb300 import api

cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation tests run only without a GPU")
FAKE = 0x7f0000000000


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2506_03781_gb300 import build
    build.build()
    yield
    _copy(True, n=0)                                   # a good call, after which uq_last_error is empty again


def _cache(**over):
    d = dict(k=FAKE, v=FAKE + 0x1000, k_scale=FAKE + 0x2000, v_scale=FAKE + 0x3000, pages=4, kv_heads=2, page_size=16,
             head_dim=128, format=api.KV_INT8)
    d.update(over)
    return api.uq_kv_cache(*[d[n] for n, _ in api.uq_kv_cache._fields_])


CACHE_CASES = [
    (dict(k=0), "ARG"), (dict(v=0), "ARG"), (dict(k_scale=0), "ARG"), (dict(v_scale=0), "ARG"), (dict(k=FAKE + 8), "ALIGN"),
    (dict(v_scale=FAKE + 4), "ALIGN"), (dict(pages=0), "ARG"), (dict(pages=1 << 31), "ARG"), (dict(kv_heads=0), "ARG"),
    (dict(kv_heads=4097), "ARG"), (dict(page_size=8), "UNSUPPORTED"), (dict(page_size=48), "UNSUPPORTED"),
    (dict(page_size=512), "UNSUPPORTED"), (dict(page_size=0), "UNSUPPORTED"), (dict(head_dim=96), "UNSUPPORTED"),
    (dict(head_dim=0), "UNSUPPORTED"), (dict(format=3), "ARG"), (dict(format=-1), "ARG"),
]


def _copy(write, **over):
    d = dict(cache=_cache(), k=FAKE + 0x4000, v=FAKE + 0x5000, dtype=api.W_BF16, n=5, s=(256, 128, 256, 128),
             slots=FAKE + 0x6000)
    d.update(over)
    L = api.lib()
    if write:
        return L.uq_kv_write(d["cache"], d["k"], d["v"], d["dtype"], d["n"], *d["s"], d["slots"], None)
    return L.uq_kv_read(d["cache"], d["slots"], d["n"], d["k"], d["v"], d["dtype"], *d["s"], None)


def _attn(**over):
    d = dict(cache=_cache(), q=FAKE + 0x4000, dtype=api.W_F32, batch=3, heads=8, qs=(1024, 128), table=FAKE + 0x5000,
             ts=7, mp=7, lens=FAKE + 0x6000, scale=0.1, window=0, out=FAKE + 0x7000, os=(1024, 128), lse=FAKE + 0x8000,
             ws=FAKE + 0x9000, wb=32 << 20)
    d.update(over)
    return api.lib().uq_paged_attn(d["cache"], d["q"], d["dtype"], d["batch"], d["heads"], *d["qs"], d["table"], d["ts"],
                                   d["mp"], d["lens"], d["scale"], d["window"], d["out"], *d["os"], d["lse"], d["ws"],
                                   d["wb"], None)


@cpu_only
@pytest.mark.parametrize("over,expect", CACHE_CASES)
def test_caches(over, expect):
    for st in (_copy(True, cache=_cache(**over)), _copy(False, cache=_cache(**over)), _attn(cache=_cache(**over))):
        assert st == getattr(api, "UQ_ERR_" + expect), api.uq_last_error()
        assert "cache" in api.uq_last_error()


@cpu_only
def test_scales_of_a_bf16_cache_may_be_null():
    c = _cache(format=api.KV_BF16, k_scale=0, v_scale=0)
    for st in (_copy(True, cache=c), _copy(False, cache=c), _attn(cache=c)):
        assert st == api.UQ_ERR_CUDA                   # validated; there is no GPU to launch on


@cpu_only
@pytest.mark.parametrize("over,expect", [
    (dict(k=0), "ARG"), (dict(v=0), "ARG"), (dict(slots=0), "ARG"), (dict(k=FAKE + 8), "ALIGN"),
    (dict(slots=FAKE + 4), "ALIGN"), (dict(dtype=2), "ARG"), (dict(n=-1), "ARG"), (dict(n=1 << 30), "ARG"),
    (dict(s=(-256, 128, 256, 128)), "ARG"), (dict(s=(256, 128, 1 << 60, 128)), "ARG"), (dict(s=(260, 128, 256, 128)), "ALIGN"),
    (dict(s=(256, 132, 256, 128)), "ALIGN"),
])
def test_copies(over, expect):
    for write in (True, False):
        assert _copy(write, **over) == getattr(api, "UQ_ERR_" + expect), api.uq_last_error()


@cpu_only
def test_overlapping_rows_are_read_but_not_written():
    for s in ((0, 128, 256, 128), (256, 0, 256, 128), (256, 128, 128, 128), (256, 128, 256, 64), (128, 512, 256, 128)):
        assert _copy(True, s=s) == api.UQ_ERR_CUDA
        assert _copy(False, s=s) == api.UQ_ERR_ARG and "overlap" in api.uq_last_error()
    assert _copy(False, s=(128, 640, 256, 128)) == api.UQ_ERR_CUDA           # heads first
    assert _attn(os=(512, 128)) == api.UQ_ERR_ARG and _attn(qs=(0, 0)) == api.UQ_ERR_CUDA


@cpu_only
@pytest.mark.parametrize("over,expect", [
    (dict(q=0), "ARG"), (dict(out=0), "ARG"), (dict(table=0), "ARG"), (dict(lens=0), "ARG"), (dict(ws=0), "ARG"),
    (dict(q=FAKE + 8), "ALIGN"), (dict(out=FAKE + 4), "ALIGN"), (dict(table=FAKE + 2), "ALIGN"), (dict(lens=FAKE + 1), "ALIGN"),
    (dict(lse=FAKE + 2), "ALIGN"), (dict(ws=FAKE + 8), "ALIGN"), (dict(wb=8), "ARG"), (dict(dtype=5), "ARG"),
    (dict(batch=-1), "ARG"), (dict(batch=65536), "ARG"), (dict(heads=7), "ARG"), (dict(heads=0), "ARG"),
    (dict(heads=1 << 20), "ARG"), (dict(mp=0), "ARG"), (dict(mp=1 << 28), "ARG"), (dict(ts=6), "ARG"), (dict(window=-1), "ARG"),
    (dict(scale=float("nan")), "ARG"), (dict(scale=float("inf")), "ARG"), (dict(qs=(1026, 128)), "ALIGN"),
    (dict(os=(1024, -128)), "ARG"),
])
def test_attention(over, expect):
    assert _attn(**over) == getattr(api, "UQ_ERR_" + expect), api.uq_last_error()


@cpu_only
def test_nothing_to_do_is_ok():
    assert _copy(True, n=0, k=0, v=0, slots=0) == _copy(False, n=0, k=0, v=0, slots=0) == api.UQ_OK
    assert _attn(batch=0, q=0, out=0, table=0, lens=0) == api.UQ_OK
    assert _attn(lse=0) == api.UQ_ERR_CUDA


def test_workspace_of_heads_it_does_not_take():
    f = api.uq_paged_attn_workspace_bytes
    assert [f(3, 2, 128), f(0, 1, 128), f(4, 0, 128), f(4, 4, 96), f(1 << 20, 1, 64)] == [-1] * 5


def test_caches_and_slots_of_the_binding():
    for fmt, row, scales in ((api.KV_BF16, 128, None), (api.KV_INT8, 128, (5, 2, 16)), (api.KV_INT4, 64, (5, 2, 16, 2, 2))):
        c = api.empty_kv_cache(5, 2, 16, 128, fmt, "cpu")
        assert c["k"].shape == c["v"].shape == (5, 2, 16, row)
        assert ("k_scale" in c) == (scales is not None)
        if scales:
            assert c["k_scale"].shape == c["v_scale"].shape == scales
    with pytest.raises(ValueError):
        api.empty_kv_cache(5, 2, 16, 128, 7, "cpu")
    table = torch.tensor([[4, 0], [2, -1]], dtype=torch.int32)
    seq, pos = torch.tensor([0, 0, 1, 1]), torch.tensor([3, 17, 15, 16])
    assert api.kv_slots(table, seq, pos, 16).tolist() == [4 * 16 + 3, 1, 2 * 16 + 15, -1]
    with pytest.raises(ValueError):
        api.uq_kv_write(api.empty_kv_cache(5, 2, 16, 128, device="cpu"), *[torch.zeros(1, 2, 128)] * 2, torch.zeros(1).long())
