"""Numbers of bf16 rows of V that are not finite, in batches whose units (a sequence's rows of one key/value head) lie whole in
a block, several to a block, and cut over blocks: who sees them has them in their channels, and nobody else and no other
channel has.  Against the oracle in 64 bits; tolerances as rows_cases has them, of the finite channels."""

import numpy as np
import pytest
import torch

from oracle import kv as OK
from tests.rows_cases import Rows, tolerance

pytestmark = pytest.mark.gpu
BAD = (float("nan"), float("inf"), -float("inf"))


def batch(rng, count, longest, most):
    """Ragged lengths and new tokens: empty sequences, sequences without new tokens, some long ones."""
    lens = rng.integers(1, longest, count)
    lens[5::17] = 0
    lens[3::23] = rng.integers(1500, 2500, len(lens[3::23]))
    new = np.minimum(lens, rng.integers(1, most + 1, count))
    new[7::11] = 0
    return lens.tolist(), new.tolist()


def spoil(r, rng, sequences):
    """Puts what is not finite into rows of V of the new tokens of some sequences, into r.c.V too; {sequence: V without}."""
    clean = {}
    for i, b in enumerate(sequences):
        clean[b] = r.c.V[b].copy()
        for j in range(3):
            t = r.lens[b] - 1 - int(rng.integers(0, r.new[b])) if j else r.lens[b] - 1
            head, channels = int(rng.integers(0, r.kv)), rng.choice(r.hd, 1 + j, replace=False)
            page, off = int(r.c.table[b, t // r.c.page]), t % r.c.page
            value = BAD[(i + j) % 3]
            r.c.cache["v"][page, head, off, torch.from_numpy(channels).to(r.c.cache["v"].device)] = value
            r.c.V[b][head, t, channels] = value
    return clean


def check(r, clean, window, sinks):
    scale = r.hd ** -0.5
    out, lse = r.run(scale=scale, window=window, sinks=sinks)
    out, lse = out.float().cpu().numpy(), lse.cpu().numpy()
    left, seen, spared = np.ones(out.shape[:-2], bool), 0, 0
    for b, k in enumerate(r.new):
        sees = r.sees(b, window, sinks)
        for i in range(k):
            where = r.at(b, i)
            left[where] = False
            if i % (4 if b in clean else 9) and i < k - 1:            # (the oracle takes half a minute for all)
                continue
            pos = np.nonzero(sees[i])[0]
            K, V, fine, q = r.c.K[b][:, pos], r.c.V[b][:, pos], clean.get(b, r.c.V[b])[:, pos], r.qv[where]
            with np.errstate(invalid="ignore"):
                ref, ref_lse = OK.attend(q, K, V, scale)
            ok = np.isfinite(ref)
            finite_ref, _ = OK.attend(q, K, fine, scale)
            tol, tol_lse = tolerance(q, K, fine, scale, finite_ref, ref_lse, r.dtype, fine)
            got = out[where]
            assert np.array_equal(got[~ok], ref[~ok].astype(np.float32), equal_nan=True), (b, i)
            assert np.isfinite(got[ok]).all(), f"sequence {b}, new token {i} of {k}: {np.argwhere(~np.isfinite(got) & ok)[:3]}"
            assert (np.abs(got - finite_ref)[ok] <= tol[ok]).all(), (b, i)
            assert (np.abs(lse[where] - ref_lse) <= tol_lse).all(), (b, i)
            if b in clean:
                seen += not ok.all()
                spared += ok.all()
    assert (out[left] == 7).all() and (lse[left] == 7).all()          # rows of no token
    return seen, spared


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 128), ("bf16", 256), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("trees,window,sinks", [(False, 0, 0), (False, 40, 3), (True, 0, 0), (True, 33, 4)])
def test_batches(dtype, hd, trees, window, sinks):
    rng = np.random.default_rng(hd + window + trees)
    lens, new = batch(rng, 110, 330, 60 if trees else 150)
    r = Rows("bf16", dtype, hd, 4, 3, 16, lens, new, trees=trees, seed=hd + 1)
    some = [b for b in range(110) if new[b] > 1 and (b % 5 == 0 or lens[b] > 1000 or b > 105)]
    clean = spoil(r, rng, some)
    seen, spared = check(r, clean, window, sinks)
    assert seen > 30 and spared > 20


@pytest.mark.parametrize("trees", (False, True))
def test_every_sequence_has_some(trees):
    """No unit of a block is clean; rows of 37 heads over one of K and V, which tokens of two units share."""
    rng = np.random.default_rng(3)
    lens, new = batch(rng, 60, 200, 40)
    r = Rows("bf16", "bf16", 64, 1, 37, 32, lens, new, trees=trees, seed=5)
    clean = spoil(r, rng, [b for b in range(60) if new[b]])
    seen, spared = check(r, clean, 0, 0)
    assert seen > 30 and spared > 20


def test_one_long_prompt_and_many_single_tokens():
    rng = np.random.default_rng(8)
    lens, new = [700] + [90 + i for i in range(40)], [500] + [1] * 40
    r = Rows("bf16", "f32", 128, 2, 4, 64, lens, new, seed=6)
    clean = spoil(r, rng, [0, 1, 20, 40])
    seen, spared = check(r, clean, 0, 0)
    assert seen > 3 and spared > 5
