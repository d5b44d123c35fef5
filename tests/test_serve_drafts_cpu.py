"""Which drafts may stay behind a verification, and what may follow them (no GPU: the library's calls are stood in for)."""

import itertools

import pytest
import torch

from paper_2506_03781_gb300 import api, serve
from tests.test_serve_cpu import decoder, pool, state

TREE = [-1, 0, 0, 2, 1, 3]                       # 0 - (1 - 4, 2 - 3 - 5)
CHAINS = [[], [0], [0, 1], [0, 2], [0, 1, 4], [0, 2, 3], [0, 2, 3, 5]]


@pytest.fixture
def drafted(monkeypatch):
    """(pool, a sequence of 20 tokens and the 6 drafts of TREE, decoder)."""
    monkeypatch.setattr(api, "uq_paged_tree_attn", lambda *a, **more: None)
    p = pool(pages=12)
    d, s = decoder(p), p.open()
    d.window = d.sinks = 0
    d._append = lambda X, slots, pos: X.new_zeros(X.shape[0], d.shape.heads, d.shape.head_dim)
    d._rest = lambda X, o: X
    p.append([s], [20])
    d.verify([s], torch.zeros(1, 6, d.shape.d), [TREE])
    return p, s, d


def test_only_chains_stay(drafted):
    p, s, _ = drafted
    before = state(p)
    for n in range(7):
        for path in itertools.combinations(range(6), n):
            if list(path) not in CHAINS:
                with pytest.raises(ValueError, match="chain"):
                    p.keep(s, 6, path)
    assert state(p) == before
    p.keep(s, 6, [0, 2, 3, 5])
    assert p.length[s] == 24
    p.append([s], [1])


def test_every_chain_may_stay(monkeypatch, drafted):
    p, s, d = drafted
    for path in CHAINS:
        p.keep(s, 6, path)
        assert p.length[s] == 20 + len(path)
        p.truncate(s, 20)
        d.verify([s], torch.zeros(1, 6, d.shape.d), [TREE])


def test_parts_of_the_drafts_and_tokens_before_them(drafted):
    p, s, d = drafted
    before = state(p)
    for drafts, path in ((4, [0, 1]), (3, []), (2, [0]), (8, [0, 2]), (8, [0, 1, 3]), (8, [1, 2])):
        with pytest.raises(ValueError, match="chain"):
            p.keep(s, drafts, path)
    assert state(p) == before
    p.keep(s, 8, [0, 1, 2, 4, 5])                # two tokens before, then drafts 0, 2 and 3
    assert p.length[s] == 23
    d.verify([s], torch.zeros(1, 6, d.shape.d), [TREE])
    p.keep(s, 5, [1, 2, 4])                      # draft 0 is before these
    assert p.length[s] == 27
    d.verify([s], torch.zeros(1, 6, d.shape.d), [TREE])
    p.keep(s, 9, [1])                            # no draft stays
    assert p.length[s] == 25


def test_nothing_follows_a_tree(drafted):
    p, s, d = drafted
    before = state(p)
    for call in (lambda: p.append([s], [1]), lambda: d.decode([s], torch.zeros(1, d.shape.d)),
                 lambda: d.extend([s], torch.zeros(2, d.shape.d), [2]),
                 lambda: d.verify([s], torch.zeros(1, 1, d.shape.d), [[-1]])):
        with pytest.raises(ValueError, match="tree of drafts"):
            call()
    p.append([s], [0])
    assert state(p) == before
    p.truncate(s, 22)                            # drafts 0 and 1 are a chain
    p.append([s], [1])
    p.keep(s, 3, [0, 2])                         # and tokens like others from then on
    assert p.length[s] == 22


def test_chains_may_be_followed_and_drafts_end_with_their_sequence(drafted):
    p, s, d = drafted
    p.keep(s, 6, [])
    d.verify([s], torch.zeros(1, 3, d.shape.d), [[-1, 0, 1]])
    with pytest.raises(ValueError, match="chain"):
        p.keep(s, 3, [0, 2])
    d.verify([s], torch.zeros(1, 2, d.shape.d), [[-1, -1]])
    p.truncate(s, 10)
    p.append([s], [1])
    d.verify([s], torch.zeros(1, 2, d.shape.d), [[-1, -1]])
    p.close(s)
    assert p.drafted == {}
