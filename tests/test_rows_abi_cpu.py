"""Refusals of uq_kv_append, uq_paged_attn_sinks, uq_paged_prompt_attn and uq_paged_tree_attn before anything is
launched (fake pointers: only where there is no GPU), and the oracle's masks."""

import numpy as np
import pytest
import torch

from oracle import kv as OK
from paper_2506_03781_gb300 import api

cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation tests run only without a GPU")
FAKE = 0x7f0000000000


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2506_03781_gb300 import build
    build.build()
    yield
    _append(n=0)                                       # a good call, after which uq_last_error is empty again


def _cache(**over):
    d = dict(k=FAKE, v=FAKE + 0x1000, k_scale=FAKE + 0x2000, v_scale=FAKE + 0x3000, pages=4, kv_heads=2, page_size=16,
             head_dim=128, format=api.KV_INT8)
    d.update(over)
    return api.uq_kv_cache(*[d[n] for n, _ in api.uq_kv_cache._fields_])


def _append(**over):
    d = dict(cache=_cache(), k=FAKE + 0x4000, v=FAKE + 0x5000, dtype=api.W_BF16, n=5, s=(256, 128, 256, 128),
             slots=FAKE + 0x6000, pos=FAKE + 0x7000, rope=FAKE + 0x8000, rows=100, rot=64, q=FAKE + 0x9000, heads=8,
             qs=(1024, 128), out=FAKE + 0xa000, os=(1024, 128))
    d.update(over)
    return api.lib().uq_kv_append(d["cache"], d["k"], d["v"], d["dtype"], d["n"], *d["s"], d["slots"], d["pos"], d["rope"],
                                  d["rows"], d["rot"], d["q"], d["heads"], *d["qs"], d["out"], *d["os"], None)


COMMON = dict(cache=_cache(), q=FAKE + 0x4000, dtype=api.W_F32, batch=3, heads=8, table=FAKE + 0x5000, ts=7, mp=7,
              lens=FAKE + 0x6000, scale=0.1, window=9, sinks=4, out=FAKE + 0x7000, lse=FAKE + 0x8000, ws=FAKE + 0x9000,
              wb=64 << 20)


def _sinks(**over):
    d = dict(COMMON, qs=(1024, 128), os=(1024, 128))
    d.update(over)
    return api.lib().uq_paged_attn_sinks(d["cache"], d["q"], d["dtype"], d["batch"], d["heads"], *d["qs"], d["table"], d["ts"],
                                         d["mp"], d["lens"], d["scale"], d["window"], d["sinks"], d["out"], *d["os"], d["lse"],
                                         d["ws"], d["wb"], None)


def _prompt(**over):
    d = dict(COMMON, qs=(1024, 128), os=(1024, 128), tokens=20, starts=FAKE + 0xa000)
    d.update(over)
    return api.lib().uq_paged_prompt_attn(d["cache"], d["q"], d["dtype"], d["tokens"], d["heads"], *d["qs"], d["starts"],
                                          d["batch"], d["table"], d["ts"], d["mp"], d["lens"], d["scale"], d["window"],
                                          d["sinks"], d["out"], *d["os"], d["lse"], d["ws"], d["wb"], None)


def _tree(**over):
    d = dict(COMMON, drafts=5, qs=(5120, 1024, 128), os=(5120, 1024, 128), tree=FAKE + 0xb000, rs=5, counts=FAKE + 0xc000)
    d.update(over)
    if len(d["qs"]) == 2:
        d["qs"] = (5 * d["qs"][0], *d["qs"])
    if len(d["os"]) == 2:
        d["os"] = (5 * d["os"][0], *d["os"])
    return api.lib().uq_paged_tree_attn(d["cache"], d["q"], d["dtype"], d["batch"], d["drafts"], d["heads"], *d["qs"],
                                        d["tree"], d["rs"], d["counts"], d["table"], d["ts"], d["mp"], d["lens"], d["scale"],
                                        d["window"], d["sinks"], d["out"], *d["os"], d["lse"], d["ws"], d["wb"], None)


@cpu_only
@pytest.mark.parametrize("over", [dict(k=0), dict(v_scale=FAKE + 4), dict(pages=0), dict(kv_heads=0), dict(page_size=48),
                                  dict(head_dim=96), dict(format=3)])
def test_caches(over):
    for call in (_append, _sinks, _prompt, _tree):
        assert call(cache=_cache(**over)) != api.UQ_OK and "cache" in api.uq_last_error()


@cpu_only
def test_good_calls_pass_the_checks():
    for call in (_append, _sinks, _prompt, _tree):
        assert call() == api.UQ_ERR_CUDA               # validated; there is no GPU to launch on
    assert _append(q=0, out=0, heads=0) == _tree(counts=0) == _tree(lse=0) == _prompt(lse=0) == api.UQ_ERR_CUDA


@cpu_only
@pytest.mark.parametrize("over,expect", [
    (dict(k=0), "ARG"), (dict(v=0), "ARG"), (dict(slots=0), "ARG"), (dict(pos=0), "ARG"), (dict(rope=0), "ARG"),
    (dict(q=0), "ARG"), (dict(out=0), "ARG"), (dict(k=FAKE + 8), "ALIGN"), (dict(slots=FAKE + 4), "ALIGN"),
    (dict(pos=FAKE + 4), "ALIGN"), (dict(rope=FAKE + 8), "ALIGN"), (dict(q=FAKE + 2), "ALIGN"), (dict(out=FAKE + 8), "ALIGN"),
    (dict(dtype=2), "ARG"), (dict(n=-1), "ARG"), (dict(n=1 << 30), "ARG"), (dict(heads=0), "ARG"), (dict(heads=1 << 17), "ARG"),
    (dict(n=1 << 29, heads=8), "ARG"), (dict(rot=0), "UNSUPPORTED"), (dict(rot=24), "UNSUPPORTED"), (dict(rot=144), "UNSUPPORTED"),
    (dict(rows=0), "ARG"), (dict(s=(-256, 128, 256, 128)), "ARG"), (dict(s=(260, 128, 256, 128)), "ALIGN"),
    (dict(os=(1024, 64)), "ARG"), (dict(os=(0, 128)), "ARG"), (dict(qs=(1026, 128)), "ALIGN"),
])
def test_append(over, expect):
    assert _append(**over) == getattr(api, "UQ_ERR_" + expect), api.uq_last_error()


@cpu_only
@pytest.mark.parametrize("over,expect", [
    (dict(q=0), "ARG"), (dict(out=0), "ARG"), (dict(table=0), "ARG"), (dict(lens=0), "ARG"), (dict(ws=0), "ARG"),
    (dict(q=FAKE + 8), "ALIGN"), (dict(out=FAKE + 4), "ALIGN"), (dict(table=FAKE + 2), "ALIGN"), (dict(lens=FAKE + 1), "ALIGN"),
    (dict(lse=FAKE + 2), "ALIGN"), (dict(ws=FAKE + 8), "ALIGN"), (dict(wb=8), "ARG"), (dict(dtype=5), "ARG"),
    (dict(batch=-1), "ARG"), (dict(batch=65536), "ARG"), (dict(heads=7), "ARG"), (dict(heads=0), "ARG"),
    (dict(mp=0), "ARG"), (dict(mp=1 << 28), "ARG"), (dict(ts=6), "ARG"), (dict(window=-1), "ARG"), (dict(sinks=-1), "ARG"),
    (dict(scale=float("nan")), "ARG"), (dict(scale=2.4e38), "ARG"), (dict(qs=(1026, 128)), "ALIGN"),
    (dict(os=(512, 128)), "ARG"),
])
def test_attention(over, expect):
    for call in (_sinks, _prompt, _tree):
        assert call(**over) == getattr(api, "UQ_ERR_" + expect), (call.__name__, api.uq_last_error())


@cpu_only
def test_prompts_and_trees():
    for over, expect in ((dict(starts=0), "ARG"), (dict(starts=FAKE + 2), "ALIGN"), (dict(tokens=-1), "ARG"), (dict(tokens=1 << 28), "ARG")):
        assert _prompt(**over) == getattr(api, "UQ_ERR_" + expect), api.uq_last_error()
    for over, expect in ((dict(tree=0), "ARG"), (dict(tree=FAKE + 4), "ALIGN"), (dict(counts=FAKE + 2), "ALIGN"), (dict(rs=4), "ARG"),
                         (dict(drafts=65), "ARG"), (dict(drafts=-1), "ARG"), (dict(batch=65535, drafts=64, heads=65536, rs=64), "ARG"),
                         (dict(os=(5120, 512, 128)), "ARG"), (dict(os=(1024, 1024, 128)), "ARG"), (dict(qs=(5121, 1024, 128)), "ALIGN")):
        assert _tree(**over) == getattr(api, "UQ_ERR_" + expect), (over, api.uq_last_error())
    assert _tree(os=(128, 384, 1920)) == _tree(qs=(0, 0, 0)) == api.UQ_ERR_CUDA          # heads first; broadcast queries


@cpu_only
def test_nothing_to_do_is_ok():
    assert _append(n=0, k=0, v=0, slots=0, pos=0, rope=0) == api.UQ_OK
    assert _sinks(batch=0, q=0) == _prompt(batch=0, q=0) == _prompt(tokens=0, q=0) == _tree(batch=0, q=0) == _tree(drafts=0, q=0) == api.UQ_OK


def test_workspace_of_heads_it_does_not_take():
    f = api.uq_paged_rows_workspace_bytes
    assert [f(3, 2, 128), f(0, 1, 128), f(4, 0, 128), f(4, 4, 96), f(1 << 20, 1, 64)] == [-1] * 5


def test_masks_of_the_oracle():
    assert OK.prompt_sees(5, 2).tolist() == [[1, 1, 1, 1, 0], [1] * 5]
    assert OK.prompt_sees(6, 2, 2, 1).tolist() == [[1, 0, 0, 1, 1, 0], [1, 0, 0, 0, 1, 1]]
    # root, two children, a grandchild of the second: a path is what a prompt of it would see
    masks = [1, 3, 5, 13]
    assert OK.tree_sees(6, masks).tolist() == [[1, 1, 1, 0, 0, 0], [1, 1, 1, 1, 0, 0], [1, 1, 1, 0, 1, 0], [1, 1, 1, 0, 1, 1]]
    path = OK.tree_sees(6, masks, 2, 1)[3][[0, 1, 2, 4, 5]]
    assert path.tolist() == OK.prompt_sees(5, 1, 2, 1)[0].tolist()


def test_rotation_of_the_oracle():
    x = np.arange(8, dtype=np.float32).reshape(1, 1, 8)
    rope = np.array([[[0, 1], [1, 0]]], np.float32)      # a quarter turn of the first pair, none of the second
    assert OK.rotate(x, rope, np.array([0]), 4).ravel().tolist() == [-2, 1, 0, 3, 4, 5, 6, 7]
    assert np.isnan(OK.rotate(x, rope, np.array([1]), 4).ravel()[:4]).all()
