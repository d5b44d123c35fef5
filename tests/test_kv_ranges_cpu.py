"""Ends of the range of the key-value cache's arguments (no GPU: fake pointers, nothing is launched)."""

import pytest
import torch

from paper_2506_03781_gb300 import api, build

cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="fake pointers: only without a GPU")


@pytest.mark.parametrize("sequence,position", [(0, -1), (0, -17), (1, 32), (0, 10 ** 12), (2, 0), (-1, 3), (-3, 3)])
def test_slots_of_what_the_table_has_no_place_for(sequence, position):
    """-1, as where the table's entry is negative: the table is not read at all, nor from its other end."""
    table = torch.tensor([[4, 0], [2, 7]], dtype=torch.int32)
    got = api.kv_slots(table, torch.tensor([0, sequence, 1]), torch.tensor([3, position, 17]), 16)
    assert got.tolist() == [4 * 16 + 3, -1, 7 * 16 + 1]


def test_slots_of_an_empty_table_and_of_one_sequence():
    assert api.kv_slots(torch.zeros(2, 0, dtype=torch.int32), torch.tensor([0, 1]), torch.tensor([0, 5]), 16).tolist() == [-1, -1]
    table = torch.tensor([[4, 0], [2, 7]], dtype=torch.int32)
    assert api.kv_slots(table, 1, torch.tensor([0, 16, 40]), 16).tolist() == [32, 112, -1]


@cpu_only
@pytest.mark.parametrize("scale,ok", [(1.7e38, True), (-1.7e38, True), (2.4e38, False), (-3.4e38, False), (0.0, True)])
def test_scales_beyond_the_exponentials_base(scale, ok):
    """Scores are taken to base 2: a scale whose product with log2(e) is no fp32 number would make every score NaN."""
    build.build()
    fake = 0x7f0000000000
    c = api.uq_kv_cache(fake, fake + 0x1000, None, None, 4, 2, 16, 128, api.KV_BF16)
    L = api.lib()
    st = L.uq_paged_attn(c, fake + 0x4000, api.W_F32, 3, 8, 1024, 128, fake + 0x5000, 7, 7, fake + 0x6000, scale, 0,
                         fake + 0x7000, 1024, 128, None, fake + 0x9000, 32 << 20, None)
    assert st == (api.UQ_ERR_CUDA if ok else api.UQ_ERR_ARG)          # validated; there is no GPU to launch on
    if not ok:
        assert "scale" in api.uq_last_error()
    assert L.uq_kv_write(c, 0, 0, api.W_F32, 0, 0, 0, 0, 0, 0, None) == api.UQ_OK      # uq_last_error is empty again
