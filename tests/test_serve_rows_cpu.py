"""Truncating sequences, keeping a path of drafts, and the checks of extend and verify (no GPU: nothing is launched)."""

import pytest
import torch

from paper_2506_03781_gb300 import api, serve
from tests.test_serve_cpu import decoder, pool, state


@pytest.mark.parametrize("fmt", (api.KV_BF16, api.KV_INT8, api.KV_INT4))
def test_a_path_moves_up(fmt):
    p = pool(pages=8, fmt=fmt)
    s, t = p.open(), p.open()
    p.append([t], [3])
    p.append([s], [30])
    for i, rows in enumerate(p.cache.values()):
        rows.copy_(torch.arange(rows.numel()).reshape(rows.shape) % 100 + i)
    slots, _ = p.append([s], [9])
    want = {n: r[slots // 16, :, slots % 16].clone() for n, r in p.cache.items()}
    other = {n: r[p.owned[t][0]].clone() for n, r in p.cache.items()}
    p.keep(s, 9, [1, 2, 5, 8])
    assert p.length[s] == 34 and len(p.owned[s]) == 3
    at = api.kv_slots(p.table, torch.full((4,), s), torch.arange(30, 34), 16)
    for n, r in p.cache.items():
        assert torch.equal(r[at // 16, :, at % 16], want[n][[1, 2, 5, 8]])
        assert torch.equal(r[p.owned[t][0]], other[n])


def test_pages_behind_come_back():
    p = pool()
    s = p.open()
    p.append([s], [50])
    free = len(p.free)
    p.truncate(s, 17)
    assert p.length[s] == 17 and len(p.free) == free + 2 and p.table[s].tolist()[2:] == [-1] * (p.table.shape[1] - 2)
    p.keep(s, 17, [])
    assert p.length[s] == 0 and p.owned[s] == []
    p.append([s], [96])


def test_refusals_take_nothing():
    p = pool()
    d, s = decoder(p), p.open()
    p.append([s], [5])
    before = state(p)
    for drafts, path in ((6, []), (-1, []), (3, [0, 0]), (3, [2, 1]), (3, [3]), (3, [-1])):
        with pytest.raises(ValueError):
            p.keep(s, drafts, path)
    for n in (-1, 6):
        with pytest.raises(ValueError):
            p.truncate(s, n)
    for X, counts in ((torch.zeros(3, d.shape.d), [2]), (torch.zeros(3, d.shape.d), [3, 0]), (torch.zeros(3, d.shape.d + 1), [3]),
                      (torch.zeros(0, d.shape.d), [-1])):
        with pytest.raises(ValueError):
            d.extend([s], X, counts)
    for shape, parents in (((1, 2), [[-1]]), ((1, 2), [[-1, 1]]), ((1, 2), [[-1, -2]]), ((2, 1), [[-1]]), ((1, 65), [[-1] * 65])):
        with pytest.raises(ValueError):
            d.verify([s], torch.zeros(*shape, d.shape.d), parents)
    assert d.extend([s], torch.zeros(0, d.shape.d), [0]).shape == (0, d.shape.d)
    assert d.verify([s], torch.zeros(1, 0, d.shape.d), [[]]).shape == (1, 0, d.shape.d)
    assert d.verify([], torch.zeros(0, 0, d.shape.d), []).shape == (0, 0, d.shape.d)
    assert state(p) == before


def test_ancestors():
    masks, depths = serve.ancestors([[-1, 0, 0, 2], [-1, -1, 1, -1]])
    assert masks == [[1, 3, 5, 13], [1, 2, 6, 8]] and depths == [[0, 1, 1, 2], [0, 0, 1, 0]]
    assert serve.ancestors([list(range(-1, 63))])[0][0][63] == -1
