"""The bound on fp32 results of the attention (attn_emulation.FP32_BOUND): the
arithmetic as it is stays within half of it, and each of its parts that is left
out exceeds it."""

import numpy as np
import pytest

from oracle import kv as OK
from tests import attn_emulation as E


def off(fmt, n, rows, hd, positive=False, **what):
    """The largest error, in units of sum_t p_t |v_t|, of `rows` queries over n positions."""
    rng = np.random.default_rng(n + hd)
    worst = 0.0
    for _ in range(4):
        k, v = rng.standard_normal((n, hd)).astype(np.float32), rng.standard_normal((n, hd)).astype(np.float32) / 2
        kept_k, kept_v = OK.quantise_rows(k, fmt), OK.quantise_rows(np.abs(v) if positive else v, fmt)
        q = rng.standard_normal((rows, hd)).astype(np.float32)
        K, V = (OK.row_values(t, fmt)[None] for t in (kept_k, kept_v))
        ref, _ = OK.attend(q, K, V, hd ** -0.5)
        mass, _ = OK.attend_mass(q, K, V, hd ** -0.5)
        err = np.abs(E.attend_fp32(q, kept_k, kept_v, fmt, hd ** -0.5, **what) - ref)
        worst = max(worst, (err / np.maximum(mass, 1e-30)).max())       # a channel of zeros has to be exact
    return worst


@pytest.mark.parametrize("fmt", ("bf16", "int8"))
@pytest.mark.parametrize("hd", (64, 128, 256))
def test_the_whole_arithmetic_is_within_half_of_it(fmt, hd):
    for n, rows in ((1, 8), (2, 64), (17, 64), (1000, 8)):
        assert off(fmt, n, rows, hd) <= E.FP32_BOUND / 2
    assert off(fmt, 2500, 2, hd, positive=True) <= E.FP32_BOUND / 2


@pytest.mark.parametrize("fmt", ("bf16", "int8"))
@pytest.mark.parametrize("hd", (64, 128))
@pytest.mark.parametrize("what", (dict(weight_terms=2), dict(weight_terms=1), dict(query_terms=1)))
def test_a_dropped_term_exceeds_it(fmt, hd, what):
    for n in (2, 3, 5):
        assert off(fmt, n, 64, hd, **what) > 1.5 * E.FP32_BOUND


def test_two_terms_of_a_query_over_bf16_rows_exceed_it():
    for n in (2, 3, 5):
        assert off("bf16", n, 64, 128, query_terms=2) > 1.5 * E.FP32_BOUND


@pytest.mark.parametrize("fmt", ("bf16", "int8"))
def test_sums_that_are_cut_off_over_a_long_part_exceed_it(fmt):
    assert off(fmt, 2500, 2, 64, positive=True, fp32_sums=False) > 1.5 * E.FP32_BOUND
