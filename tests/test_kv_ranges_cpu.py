"""Ends of the range of the key-value cache's arguments."""

import pytest
import torch

from paper_2506_03781_gb300 import api


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
