"""uq_paged_attn at the ends of the range: keys, queries and scales whose scores
are ordinary numbers although their factors are not."""

import numpy as np
import pytest

from oracle import kv as OK
from tests import kv_cases as C

pytestmark = pytest.mark.gpu
FORMATS = ("bf16", "int8", "int4")
F32 = np.float32


def case(fmt, dtype, k_size, q_size, lens=(1, 50, 700), hd=128, r=4, seed=21):
    """A case whose keys and queries are normal, times k_size and q_size."""
    c = C.Case(fmt, dtype, hd, 2, r, 16, list(lens), seed=seed)
    rng = np.random.default_rng(seed + 1)
    for b, n in enumerate(c.lens):
        k = (rng.standard_normal((n, c.kv, hd)) * k_size).astype(F32)
        kept = OK.quantise_rows(k, fmt)
        C.rows_to_cache(c.cache, fmt, "k", kept, c.table[b].astype(np.int64)[np.arange(n) // 16] * 16 + np.arange(n) % 16)
        c.K[b] = OK.row_values(kept, fmt).transpose(1, 0, 2)
    c.q, c.qv = C.typed(rng.standard_normal((len(c.lens), c.kv * r, hd)) * q_size, dtype)
    return c


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("size", (1e-28, 1e-20, 1e20, 1e32, 1e34, 1e35, 1e36))
def test_keys_of_all_sizes(fmt, dtype, size):
    """Scores of order 1: queries are as small as keys are large."""
    case(fmt, dtype, size, 1 / size).check()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ("bf16", "f32"))
@pytest.mark.parametrize("k,q,scale", [(1e36, 1.0, 1e-37), (1e35, 1e-12, -1e-24), (1e-28, 1.0, 1e27), (1e-28, 1e33, 1e-6),
                                       (1e-28, 1e-7, 1e34), (1.0, 1e36, 1e-37), (1.0, 1e-36, 1e35)])
def test_scales_that_belong_to_such_sizes(fmt, dtype, k, q, scale):
    case(fmt, dtype, k, q).check(scale=scale)
