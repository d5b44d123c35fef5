"""Infinities in rows of a bf16 cache: uq_paged_attn gives what the sums of its
definition give, although weights and fp32 queries enter them in several terms."""

import numpy as np
import pytest
import torch

from oracle import kv as OK
from tests import kv_cases as C

pytestmark = pytest.mark.gpu


def with_rows(dtype, seed=31):
    c = C.Case("bf16", dtype, 64, 2, 4, 16, [1, 2, 30, 400], seed=seed)
    c.spot = lambda b, t: (int(c.table[b, t // 16]), t % 16)
    return c


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("channel", (5, 63))
def test_infinite_keys_of_score_minus_infinity_have_the_weight_zero(dtype, channel):
    """Queries of few and of many significant bits; the position counts as if it were hidden."""
    c = with_rows(dtype)
    few = torch.tensor([1.0, 0.75, 1.5, 0.296875], device=C.dev()).repeat(2)
    c.q[:2, :, channel] = few.to(c.q.dtype)
    c.q[2:, :, channel] = c.q[2:, :, channel].abs() + 0.1
    c.qv = c.q.float().cpu().numpy()
    hidden = {}
    for b, at in ((1, [0]), (2, [0, 17, 29]), (3, [15, 16, 399])):
        for t in at:
            page, off = c.spot(b, t)
            c.cache["k"][page, :, off, channel] = float("-inf")
        hidden[b] = np.array(at)
    c.check(hidden=hidden)


@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("value", (float("inf"), float("-inf")))
def test_infinite_values_give_infinities_in_their_channel(dtype, value):
    """In the heaviest position, whose weight is exactly 1, and in any other: an infinity there, and nothing elsewhere."""
    for heavy in (True, False):
        c = with_rows(dtype, seed=32 + heavy)
        for b, n in enumerate(c.lens):
            for h in range(c.kv):
                x = np.einsum("rd,nd->rn", c.qv[b].reshape(c.kv, c.r, c.hd)[h], c.K[b][h])
                t = int(x.max(0).argmax() if heavy else n // 2)
                page, off = c.spot(b, t)
                c.cache["v"][page, h, off, 7] = value
                c.V[b][h, t, 7] = 0
        out, lse = c.run()
        assert (out[..., 7].float() == value).all()
        out[..., 7] = 0                                            # the rest is as without the infinity
        got = out.float().cpu().numpy()
        for b in range(len(c.lens)):
            ref, ref_lse = OK.attend(c.qv[b], c.K[b], c.V[b], c.hd ** -0.5)
            tol, _ = C.tolerance(c.qv[b], c.K[b], c.V[b], c.hd ** -0.5, ref, ref_lse, dtype)
            keep = np.arange(c.hd) != 7
            assert (np.abs(got[b] - ref) <= tol)[:, keep].all()
