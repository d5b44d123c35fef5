"""uq_kv_append on the GPU against the oracle: what it decides is exact in fp32, so rows, scales and queries are equal."""

import numpy as np
import pytest
import torch

from oracle import kv as OK
from paper_2506_03781_gb300 import api
from tests import kv_cases as C

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "int8", "int4")


def rope_table(rows, rot):
    angle = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(rot // 2) * 2.0 / rot)
    return np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


class Append:
    def __init__(self, fmt, dtype, n, H, kv, hd, page, rot, seed=0, rows=300):
        rng = np.random.default_rng(seed)
        self.fmt, self.rot, self.kv, self.H, self.hd = fmt, rot, kv, H, hd
        pages = -(-n // page) + 2
        self.cache = api.empty_kv_cache(pages, kv, page, hd, C.FMT[fmt], C.dev())
        C.poison(self.cache)
        self.slots = rng.permutation(pages * page)[:n].astype(np.int64)
        self.positions = rng.integers(0, rows, n)
        self.rope = rope_table(rows, rot)
        self.fused, self.x = C.typed(rng.standard_normal((n, H + 2 * kv, hd)), dtype)
        self.q_out = torch.full((n, H, hd), 7.0, dtype=C.DT[dtype], device=C.dev())
        self.dtype = dtype

    def parts(self, x):
        return x[:, :self.H], x[:, self.H:self.H + self.kv], x[:, self.H + self.kv:]

    def run(self, **more):
        q, k, v = self.parts(self.fused)
        d = lambda a: torch.from_numpy(a).to(C.dev())
        args = dict(q=q, q_out=self.q_out)
        args.update(more)
        api.uq_kv_append(self.cache, k, v, d(self.slots), d(self.positions), d(self.rope), **args)
        torch.cuda.synchronize()

    def check(self, **more):
        before = {n: t.clone() for n, t in self.cache.items()}
        self.run(**more)
        q, k, v = self.parts(self.x)
        page = self.cache["k"].shape[2]
        there = (self.slots >= 0) & (self.slots < self.cache["k"].shape[0] * page)
        with np.errstate(all="ignore"):
            turned = OK.rotate(k, self.rope, self.positions, self.rot)
            want_q = OK.rotate(q, self.rope, self.positions, self.rot)
        if self.dtype == "bf16":
            want_q = torch.from_numpy(want_q).to(torch.bfloat16).float().numpy()
        assert same(self.q_out.float().cpu().numpy(), want_q)
        for name, x in (("k", turned), ("v", v)):
            kept = OK.quantise_rows(x[there], self.fmt)
            got = C.cache_rows(self.cache, self.fmt, name, self.slots[there])
            for a, b in zip(got, kept):
                assert a is None and b is None or same(np.asarray(a, np.float64), np.asarray(b, np.float64)), name
        used = torch.zeros(self.cache["k"].shape[0] * page, dtype=torch.bool, device=C.dev())
        used[torch.from_numpy(self.slots[there]).to(C.dev())] = True
        for name, t in self.cache.items():            # nothing else is written
            rows = lambda a: a.transpose(1, 2).reshape(used.numel(), -1).clone(memory_format=torch.contiguous_format).view(torch.uint8)
            assert torch.equal(rows(t)[~used], rows(before[name])[~used]), name


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("hd,rots", [(64, (64, 32, 16)), (128, (128, 64, 48)), (256, (256, 128, 80, 16))])
@pytest.mark.parametrize("n,H,kv,page", [(1, 4, 2, 16), (33, 6, 3, 32), (130, 7, 7, 256), (5, 1, 1, 64), (70, 16, 1, 16)])
def test_rows_and_queries(fmt, dtype, hd, rots, n, H, kv, page):
    for rot in rots:
        Append(fmt, dtype, n, H, kv, hd, page, rot, seed=n + rot).check()


@pytest.mark.parametrize("fmt", FORMATS)
def test_padding_and_positions_that_the_table_has_not(fmt):
    a = Append(fmt, "f32", 64, 4, 2, 64, 16, 32, seed=3)
    a.slots[5::7] = -1
    a.slots[3] = 10 ** 12
    a.positions[::9] = -1
    a.positions[1::9] = 300
    a.positions[2] = 2 ** 62
    a.check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_numbers_of_all_sizes(fmt, dtype):
    a = Append(fmt, dtype, 40, 4, 2, 128, 16, 128, seed=4)
    a.fused[:8] *= 1e30
    a.fused[8:16] *= 1e-30
    a.fused[16:20] *= 1e-38
    a.fused[20, 5, 3] = float("inf")
    a.fused[21, 4, 100] = float("nan")
    a.fused[22, 6, 7] = -float("inf")
    a.fused[23] = 0
    a.x = a.fused.float().cpu().numpy()
    a.check()


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
def test_queries_in_place_none_and_strided(dtype):
    a = Append("int8", dtype, 50, 6, 2, 64, 16, 64, seed=5)
    a.check()
    want, rows = a.q_out.clone(), {n: t.clone() for n, t in a.cache.items()}
    C.poison(a.cache)
    a.run(q=None, q_out=None)
    assert all(torch.equal(t.view(torch.uint8), a.cache[n].view(torch.uint8)) for n, t in rows.items())
    room = torch.full((6, 50, 3, 64), 7.0, dtype=C.DT[dtype], device=C.dev())
    a.run(q_out=room[:, :, 1].transpose(0, 1))
    assert torch.equal(room[:, :, 1].transpose(0, 1), want) and (room[:, :, 0] == 7).all() and (room[:, :, 2] == 7).all()
    q = a.parts(a.fused)[0]
    a.run(q=q, q_out=q)
    assert torch.equal(q, want)


def test_no_tokens_and_a_stream():
    a = Append("int4", "bf16", 20, 4, 2, 64, 16, 64, seed=6)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a.check(stream=s)
    e = torch.zeros(0, 2, 64, device=C.dev())
    z = torch.zeros(0, dtype=torch.int64, device=C.dev())
    api.uq_kv_append(a.cache, e, e, z, z, torch.zeros(3, 32, 2, device=C.dev()), q=e, q_out=e)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_then_attend(fmt):
    """A chat as it is served: a prompt in two chunks, one token, then a tree of drafts, one sequence's cache; the last
    rows against the oracle on the cache's values."""
    rng = np.random.default_rng(9)
    H, kv, hd, page, n = 8, 2, 64, 16, 90
    cache = api.empty_kv_cache(8, kv, page, hd, C.FMT[fmt], C.dev())
    C.poison(cache)
    table = torch.from_numpy(rng.permutation(8).astype(np.int32)[None, :6]).to(C.dev())
    rope = torch.from_numpy(rope_table(128, hd)).to(C.dev())
    fused, _ = C.typed(rng.standard_normal((n, H + 2 * kv, hd)), "f32")
    masks = [1, 3, 5, 11]
    depth = [bin(m).count("1") - 1 for m in masks]
    place = torch.arange(n, device=C.dev())
    pos = torch.cat([place[:86], 86 + torch.tensor(depth, device=C.dev())])
    out = torch.empty(n, H, hd, device=C.dev())
    q = torch.empty_like(out)
    slots = api.kv_slots(table, torch.zeros_like(place), place, page)
    for lo, hi in ((0, 50), (50, 85), (85, 86), (86, 90)):
        f = fused[lo:hi]
        api.uq_kv_append(cache, f[:, H:H + kv], f[:, H + kv:], slots[lo:hi], pos[lo:hi].contiguous(), rope, q=f[:, :H], q_out=q[lo:hi])
        lens = torch.tensor([hi], dtype=torch.int32, device=C.dev())
        more = dict(window=30, sinks=4)
        if hi - lo == 1:
            api.uq_paged_attn_sinks(cache, q[lo:hi], table, lens, out[lo:hi], **more)
        elif lo < 86:
            api.uq_paged_prompt_attn(cache, q[lo:hi], torch.tensor([0, hi - lo], dtype=torch.int32, device=C.dev()), table, lens, out[lo:hi], **more)
        else:
            api.uq_paged_tree_attn(cache, q[None, lo:hi], torch.tensor([masks], device=C.dev()), table, lens, out[None, lo:hi], **more)
    torch.cuda.synchronize()
    K, V = (OK.row_values(C.cache_rows(cache, fmt, name, slots.cpu().numpy()), fmt).transpose(1, 0, 2) for name in ("k", "v"))
    sees = np.zeros((n, n), bool)
    sees[:86, :86] = OK.prompt_sees(86, 86, 30, 4)
    sees[86:] = OK.tree_sees(90, masks, 30, 4)
    for i in range(n):
        at = np.nonzero(sees[i])[0]
        ref, _ = OK.attend(q[i].cpu().numpy(), K[:, at], V[:, at], hd ** -0.5)
        assert np.abs(out[i].cpu().numpy() - ref).max() < 2e-5, i
