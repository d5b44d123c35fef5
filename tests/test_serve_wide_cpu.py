"""Prompts of a block with heads of 256 channels: long ones attend over rows that are read back, because the attention over
the cache takes such fp32 heads row by row (no GPU: the library's calls are stood in for)."""

import dataclasses

import numpy as np
import pytest
import torch

from oracle import kv as OK
from paper_2506_03781_gb300 import api, serve, synth


@pytest.mark.parametrize("n,head_dim,window,back", [(255, 256, 0, False), (256, 256, 0, True), (300, 256, 0, True),
                                                    (300, 256, 9, False), (300, 128, 0, False), (0, 256, 0, False)])
def test_which_way_a_prompt_goes(monkeypatch, n, head_dim, window, back):
    shape = dataclasses.replace(synth.BLOCKS["tiny"], head_dim=head_dim)
    pool = serve.PagePool(40, shape.kv_heads, head_dim, page_size=16, sequences=2, device="cpu")
    d, s = serve.BlockDecoder.__new__(serve.BlockDecoder), pool.open()
    d.shape, d.pool, d.window, d.sinks, d.workspace = shape, pool, window, 0, None
    rng = np.random.default_rng(n)
    Q, K, V = (rng.standard_normal((n, h, head_dim)).astype(np.float32) for h in (shape.heads, shape.kv_heads, shape.kv_heads))
    calls = []
    d._append = lambda X, slots, positions: torch.from_numpy(Q)
    d._rest = lambda X, o: o

    def read(cache, slots, k, v):
        calls.append("read")
        k.copy_(torch.from_numpy(K))
        v.copy_(torch.from_numpy(V))

    monkeypatch.setattr(api, "uq_kv_read", read)
    monkeypatch.setattr(api, "uq_paged_prompt_attn", lambda *a, **more: calls.append("attention"))
    o = d.prefill(s, torch.zeros(n, shape.d))
    assert calls == (["read"] if back else ["attention"] if n else []) and pool.length[s] == n
    if back:
        for t in range(0, n, 37):
            ref, _ = OK.attend(Q[t], K[:t + 1].transpose(1, 0, 2), V[:t + 1].transpose(1, 0, 2), head_dim ** -0.5)
            # a score's sum of 256 terms reaches about 4 and is off by some sqrt(256) half steps of that, 4e-6; times |v| <= 4
            assert np.abs(o[t].numpy() - ref).max() < 2e-5, t
