"""The page pool and the decoder's checks (no GPU: nothing is launched)."""

import pytest
import torch

from paper_2506_03781_gb300 import api, serve, synth


def pool(pages=6, page_size=16, sequences=3, **more):
    return serve.PagePool(pages, 2, 64, page_size=page_size, sequences=sequences, device="cpu", **more)


def state(p):
    return dict(p.length), {s: list(o) for s, o in p.owned.items()}, list(p.free), p.table.tolist()


def test_slots_of_all_tokens_are_apart():
    p = pool()
    a, b = p.open(), p.open()
    seen = []
    for sequences, counts in (([a], [15]), ([b, a], [1, 1]), ([a, b], [20, 30])):
        first = [p.length[s] for s in sequences]
        slots, pos = p.append(sequences, counts)
        want = [t for n0, n in zip(first, counts) for t in range(n0, n0 + n)]
        assert pos.tolist() == want and slots.dtype == pos.dtype == torch.int64
        of = [s for s, n in zip(sequences, counts) for _ in range(n)]
        assert slots.tolist() == api.kv_slots(p.table, torch.tensor(of), pos, 16).tolist()
        seen += slots.tolist()
    assert len(set(seen)) == len(seen) == 67 and min(seen) >= 0


def test_a_sequence_named_twice_is_refused():
    p = pool()
    s = p.open()
    p.append([s], [15])
    before = state(p)
    with pytest.raises(ValueError, match="twice"):
        p.append([s, s], [1, 1])
    assert state(p) == before


def decoder(p):
    """One whose weights are never reached."""
    d = serve.BlockDecoder.__new__(serve.BlockDecoder)
    d.shape, d.pool = synth.BLOCKS["tiny"], p
    return d


def test_a_prefill_begins_a_sequence():
    p = pool()
    d, s = decoder(p), p.open()
    p.append([s], [5])
    before = state(p)
    with pytest.raises(ValueError, match="has 5 tokens"):
        d.prefill(s, torch.zeros(3, d.shape.d))
    assert state(p) == before


def test_no_tokens():
    p = pool()
    d, s = decoder(p), p.open()
    for sequences, counts in (([], []), ([s], [0])):
        slots, pos = p.append(sequences, counts)
        assert slots.tolist() == pos.tolist() == [] and slots.dtype == pos.dtype == torch.int64
    assert d.prefill(s, torch.zeros(0, d.shape.d)).shape == (0, d.shape.d)
    assert d.decode([], torch.zeros(0, d.shape.d)).shape == (0, d.shape.d)
    assert p.length[s] == 0 and p.owned[s] == []


def test_what_is_refused_takes_nothing():
    p = pool()
    d, s, t = decoder(p), p.open(), p.open()
    before = state(p)
    for sequences, counts in (([s], [-1]), ([s, t], [1]), ([s], [1, 2])):
        with pytest.raises(ValueError, match="count"):
            p.append(sequences, counts)
    for X in (torch.zeros(3, d.shape.d + 1), torch.zeros(d.shape.d), torch.zeros(1, 3, d.shape.d)):
        with pytest.raises(ValueError, match="X"):
            d.prefill(s, X)
    for X in (torch.zeros(3, d.shape.d), torch.zeros(2, d.shape.d - 1), torch.zeros(d.shape.d)):
        with pytest.raises(ValueError, match="X"):
            d.decode([s, t], X)
    assert state(p) == before
