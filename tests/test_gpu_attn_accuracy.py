"""fp32 results of uq_paged_attn to a bound that a dropped term exceeds
(attn_emulation.FP32_BOUND; kv_cases.tolerance bounds the worst case and cannot
see one)."""

import numpy as np
import pytest
import torch

from oracle import kv as OK
from paper_2506_03781_gb300 import api
from tests import attn_emulation as E
from tests import kv_cases as C

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "int8", "int4")


def check(c):
    scale = c.hd ** -0.5
    out, _ = c.run(scale=scale)
    out = out.cpu().numpy()
    for b, n in enumerate(c.lens):
        ref, _ = OK.attend(c.qv[b], c.K[b], c.V[b], scale)
        mass, _ = OK.attend_mass(c.qv[b], c.K[b], c.V[b], scale)
        off = (np.abs(out[b] - ref) / np.maximum(mass, 1e-30)).max()
        assert off <= E.FP32_BOUND, f"sequence {b} of {n} tokens: {off:.3g} of the mass"


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("hd", (64, 128, 256))
@pytest.mark.parametrize("r", (4, 16))
def test_few_tokens(fmt, hd, r):
    """The weights of two and three positions are not averaged over many: a lost term shows most."""
    check(C.Case(fmt, "f32", hd, 2, r, 16, [1, 2, 3, 2, 3, 2, 3, 5, 17, 40], seed=hd))


@pytest.mark.parametrize("fmt", FORMATS)
def test_many_tokens(fmt):
    check(C.Case(fmt, "f32", 128, 2, 4, 64, [1000, 70001], seed=11))


@pytest.mark.parametrize("fmt", FORMATS)
def test_long_parts_of_a_warp(fmt):
    """1024 sequences share the pages of one of 4000 tokens, so that a warp adds up thousands of positions of one sign."""
    n, hd, B = 4000, 64, 1024
    c = C.Case(fmt, "f32", hd, 1, 1, 16, [n], seed=12)
    v = np.abs(np.random.default_rng(13).standard_normal((n, 1, hd))).astype(np.float32) / 2
    slots = c.table[0, np.arange(n) // 16].astype(np.int64) * 16 + np.arange(n) % 16
    kept = OK.quantise_rows(v, fmt)
    C.rows_to_cache(c.cache, fmt, "v", kept, slots)
    V = OK.row_values(kept, fmt).transpose(1, 0, 2)
    q, qv = C.typed(np.random.default_rng(14).standard_normal((B, 1, hd)), "f32")
    out = torch.full_like(q, float("nan"))
    api.uq_paged_attn(c.cache, q, c.tab.expand(B, -1).contiguous(), c.len.expand(B).contiguous(), out)
    torch.cuda.synchronize()
    ref, _ = OK.attend(qv[:, 0], c.K[0], V, hd ** -0.5)
    mass, _ = OK.attend_mass(qv[:, 0], c.K[0], V, hd ** -0.5)
    off = (np.abs(out[:, 0].cpu().numpy() - ref) / mass).max()
    assert off <= E.FP32_BOUND, f"{off:.3g} of the mass"
