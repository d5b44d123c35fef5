"""What pins the oracle of the key-value cache (oracle/kv.py): brute force over
the codes, error bounds, closed forms and torch in fp64."""

import numpy as np
import pytest
import torch

from oracle import kv as OK

F32, F64 = np.float32, np.float64


def test_bf16_rounding_is_torchs():
    x = np.random.default_rng(0).standard_normal(4000).astype(F32) * F32(3)
    x[:6] = [0.0, -0.0, np.inf, -np.inf, 1e-40, 3.3e38]
    assert np.array_equal(OK.to_bf16(x), torch.from_numpy(x).bfloat16().float().numpy())


@pytest.mark.parametrize("fmt,codes", [("int8", np.arange(-127, 128)), ("int4", np.arange(16))])
def test_codes_are_the_nearest_of_the_grid(fmt, codes):
    """No other code stands for a value nearer to x (by more than the rounding of the quotient can explain)."""
    x = np.random.default_rng(1).standard_t(4, (50, 128)).astype(F32)
    c, s, m = OK.quantise_rows(x, fmt)
    val = OK.row_values((c, s, m), fmt)
    per = np.repeat(s, 128 if fmt == "int8" else 64, -1).reshape(50, 128).astype(F64)
    low = 0.0 if m is None else np.repeat(m, 64, -1).astype(F64)
    best = np.abs(codes[:, None, None] * per + low - x).min(0)
    assert (np.abs(val - x) <= best + 2e-5 * per).all()
    # at most half a step (int4: and what the minimum's and the scale's rounding to bf16 put beyond the ends)
    slack = 0 if m is None else 2.0 ** -8 * (np.abs(low) + 15 * per)
    assert (np.abs(val - x) <= 0.5001 * per + slack).all()


def test_rows_that_are_not_numbers_read_as_nan():
    x = np.random.default_rng(2).standard_normal((6, 128)).astype(F32)
    x[0, 3], x[1, 70], x[2, 100], x[3] = np.nan, np.inf, -np.inf, np.inf
    x[4] = 0
    for fmt in ("int8", "int4"):
        val = OK.row_values(OK.quantise_rows(x, fmt), fmt)
        hit = {"int8": [slice(0, 128)] * 3, "int4": [slice(0, 64), slice(64, 128), slice(64, 128)]}[fmt]
        for i in range(3):
            assert np.isnan(val[i, hit[i]]).all()
        if fmt == "int4":
            assert np.isfinite(val[0, 64:]).all() and np.isfinite(val[1, :64]).all()
        assert np.isnan(val[3]).all() and (val[4] == 0).all() and np.isfinite(val[5]).all()


def test_constant_and_tiny_rows():
    x = np.full((1, 64), 0.375, F32)
    assert np.array_equal(OK.row_values(OK.quantise_rows(x, "int4"), "int4"), x)
    assert np.abs(OK.row_values(OK.quantise_rows(x, "int8"), "int8") - x).max() < 1e-7
    tiny = np.linspace(-1e-31, 1e-31, 64, dtype=F32)[None]
    assert (OK.row_values(OK.quantise_rows(tiny, "int8"), "int8") == 0).all()


@pytest.mark.parametrize("kv,r,n", [(1, 1, 1), (2, 4, 33), (8, 1, 100)])
def test_attention_is_torchs_in_64_bits(kv, r, n):
    rng = np.random.default_rng(n)
    q, k, v = rng.standard_normal((kv * r, 64)), rng.standard_normal((kv, n, 64)), rng.standard_normal((kv, n, 64))
    out, lse = OK.attend(q, k, v, 0.3)
    tq, tk, tv = (torch.from_numpy(t) for t in (q, np.repeat(k, r, 0), np.repeat(v, r, 0)))
    x = (tk @ tq[..., None])[..., 0] * 0.3
    assert np.allclose(lse, torch.logsumexp(x, -1).numpy(), rtol=1e-13, atol=1e-13)
    assert np.allclose(out, (torch.softmax(x, -1)[:, None] @ tv)[:, 0].numpy(), rtol=1e-12, atol=1e-13)


def test_attention_over_nothing_and_over_equal_rows():
    out, lse = OK.attend(np.ones((4, 64)), np.zeros((2, 0, 64)), np.zeros((2, 0, 64)), 1.0)
    assert (out == 0).all() and np.isneginf(lse).all()
    k = np.ones((1, 10, 64))
    v = np.arange(10.0)[None, :, None] * np.ones((1, 10, 64))
    out, lse = OK.attend(np.ones((1, 64)), k, v, 0.5)
    assert np.allclose(out, 4.5) and np.allclose(lse, 32 + np.log(10))
