"""How the attention cuts its work, restated on the CPU: every tile is worked on
once, the warps of a run are neighbours, and the blocks that hold a (sequence,
key/value head) are the ones that its join looks for.

The kernel's own expressions (uq_attn.cuh: Split, Walk, the bounds of a block, the
runs, the flags), with its constants read from the source.  Places are intervals
here, so that totals beyond 2^31 cost no more than small ones."""

import bisect
import itertools
import os
import random
import re

import pytest

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_03781_gb300", "csrc",
                      "uq_attn.cuh")
TEXT = open(SOURCE).read()


def constant(name):
    return int(re.search(rf"\b{name} = (\d+)[,;]", TEXT).group(1))


MIN_WARPS, SNAP_PLACES, SNAP_TILES = (constant(n) for n in ("kMinWarps", "kSnapPlaces", "kSnapTiles"))


class Split:
    def __init__(self, total, blocks, most):
        if total <= 0x7FFFFFFF:
            self.warps = min(most, max(MIN_WARPS, (total + blocks - 1) // blocks))
            self.n = min(self.warps * blocks, total)
        else:
            self.warps, self.n = most, most * blocks
        self.per = total // self.n
        self.more = total - self.per * self.n
        self.snaps = self.per <= SNAP_PLACES

    def start(self, i):
        return self.per * i + min(i, self.more)

    def block_of(self, t):
        big = self.more * (self.per + 1)
        x, d = (t, self.per + 1) if t < big else (t - big, self.per)
        i = x // d
        return (i if t < big else self.more + i) // self.warps


def share_of(many, i, n):
    if many <= 0xFFFFFF:
        assert many * i < 2 ** 32                      # the kernel's 32-bit product
    return many * i // n


def grid_of(batch, max_tiles, head, units, full):
    most = ((max_tiles + head) * units + MIN_WARPS - 1) // MIN_WARPS
    return full if most > full // batch else most * batch


def tiles_of(n, window, tok):
    first = max(n - window, 0) if window > 0 else 0
    return max(1, (n - (first & ~15) + tok - 1) // tok)


def check(tiles, units, grid, nw, head):
    """tiles: of every sequence; units: key/value heads (and chunks of their query heads) of each."""
    starts, place = [], 0
    for t in tiles:
        for _ in range(units):
            starts.append(place)
            place += t + head
    total = place
    tiles_in = lambda i: tiles[i // units]

    def locate(p):
        i = bisect.bisect_right(starts, p) - 1
        return i, p - starts[i]

    split = Split(total, grid, nw)
    covered, partial, raised, whole = {}, {}, {}, set()
    for block in range(grid):
        if block * split.warps >= split.n:
            continue

        def bound(b):
            p = split.start(min(b * split.warps, split.n))
            if not split.snaps or p == 0 or p >= total:
                return p
            i, at = locate(p)
            unit = tiles_in(i) + head
            return p if tiles_in(i) > SNAP_TILES * nw else starts[i] + (0 if 2 * at < unit else unit)

        begin = bound(block)
        many = bound(block + 1) - begin
        if many <= 0:
            continue
        active = min(nw if split.snaps else split.warps, many)
        pieces = {}                                    # (warp, begun here) -> (unit, it has the last tile)
        for warp in range(active):
            mine = share_of(many, warp, active)
            rem = share_of(many, warp + 1, active) - mine
            assert rem > 0
            i, at = locate(begin + mine)
            parts = []
            while rem > 0:
                take = min(rem, tiles_in(i) + head - at)
                lo, hi = max(at - head, 0), max(at + take - head, 0)
                rem -= take
                if hi > lo:
                    parts.append((i, lo, hi))
                i, at = i + 1, 0
            for k, (i, lo, hi) in enumerate(parts):
                covered.setdefault(i, []).append((lo, hi))
                from_start, to_end = lo == 0, hi == tiles_in(i)
                if from_start and to_end:
                    whole.add(i)
                    continue
                assert from_start or k == 0, "only a share's first part was begun before"
                assert to_end or k + 1 == len(parts), "only its last part goes on"
                assert (warp, from_start) not in pieces
                pieces[warp, from_start] = (i, to_end)
        # runs of neighbours, as warp 0 builds them
        on = [w for w in range(nw) if (w, False) in pieces]
        here = [w for w in range(nw) if (w, True) in pieces]
        done = [w for w in on if pieces[w, False][1]]
        runs = []                                      # unit, first and last warp, has the first tile, has the last
        if on and not any(w < on[0] for w in here):
            runs.append((pieces[on[0], False][0], on[0], done[0] if done else on[-1], False, bool(done)))
        for w in here:
            rest, ends = [x for x in on if x > w], [x for x in done if x > w]
            runs.append((pieces[w, True][0], w, ends[0] if ends else rest[-1] if rest else w, True, bool(ends)))
        used = set()
        for i, w0, w1, from_start, to_end in runs:
            for w in range(w0, w1 + 1):
                key = w, from_start and w == w0
                assert key in pieces and pieces[key][0] == i
                used.add(key)
            if from_start and to_end:
                whole.add(i)
            else:
                assert (block, from_start) not in raised
                raised[block, from_start] = i
                partial.setdefault(i, []).append(block)
        assert used == set(pieces) and len(runs) <= nw + 1
        assert [k for k, r in enumerate(runs) if r[3] and not r[4]] in ([], [len(runs) - 1])
        assert [k for k, r in enumerate(runs) if not r[3]] in ([], [0])
    assert len(covered) == len(starts)
    for i, parts in covered.items():
        at = 0
        for lo, hi in sorted(parts):
            assert lo == at
            at = hi
        assert at == tiles_in(i)
        assert (i in whole) != (i in partial)
        if i in partial:
            own0, own1 = split.block_of(starts[i] + head), split.block_of(starts[i] + head + tiles_in(i) - 1)
            assert partial[i] == list(range(own0, own1 + 1)) and own1 > own0
            for block in partial[i]:                   # the flag that the join looks at, and so the partial
                assert raised[block, block == own0] == i
    return total


@pytest.mark.parametrize("nw", (8, 12))
@pytest.mark.parametrize("head", sorted({int(x) for x in re.search(r"kHead = FMT == UQ_KV_INT4 \? (\d) : (\d);", TEXT).groups()}))
def test_random_batches(nw, head):
    r = random.Random(nw + head)
    for _ in range(250):
        batch, units, tok = r.choice([1, 1, 2, 3, 5, 12, 40, 130, 400]), r.choice([1, 2, 3, 8]), r.choice([16, 32, 64])
        longest, window = r.choice([1, 40, 200, 1000, 9000]), r.choice([0, 0, 1, 100])
        lens = [r.randint(0, longest) if r.random() < 0.8 else r.randint(0, 1) for _ in range(batch)]
        room = -(-(max(lens) + r.choice([1, 16, 2000])) // tok)
        check([tiles_of(n, window, tok) for n in lens], units, grid_of(batch, room, head, units, r.choice([152, 152, 7, 1])),
              nw, head)


@pytest.mark.parametrize("nw", (8, 12))
@pytest.mark.parametrize("batch", (1000, 4000, 16000, 64000))
def test_large_batches_of_short_sequences(nw, batch):
    r = random.Random(batch)
    check([1] * batch, 8 if batch < 64000 else 2, 152, nw, 3)
    if batch <= 16000:
        check([r.randint(1, 9) for _ in range(batch)], 2, 152, nw, 2)


@pytest.mark.parametrize("nw", (8, 12))
def test_long_sequences_among_short_ones(nw):
    """Blocks begin with whole heads but within the long ones, whose joins take the bounds that were not moved."""
    r = random.Random(nw)
    for _ in range(150):
        batch = r.choice([5, 30, 120, 300])
        tiles = [r.choice([SNAP_TILES * nw - 1, SNAP_TILES * nw, SNAP_TILES * nw + 1, 60, 200, 700]) if r.random() < 0.1
                 else r.randint(1, 6) for _ in range(batch)]
        check(tiles, r.choice([1, 2, 4]), 152, nw, r.choice([2, 3]))


@pytest.mark.parametrize("nw", (8, 12))
def test_more_places_than_32_bits(nw):
    r = random.Random(nw)
    for batch, units, longest in ((70, 4, 2 ** 26), (300, 8, 2 ** 26), (65000, 1, 2 ** 18), (1, 64, 2 ** 26)):
        total = check([r.randint(longest // 2, longest) for _ in range(batch)], units, 152, nw, 3)
        assert total > 2 ** 31
    check([2 ** 26] + [1] * 40 + [2 ** 26] * 40 + [1], 2, 152, nw, 2)


@pytest.mark.parametrize("blocks", (2, 3, 4))
def test_some_block_sees_every_flag(blocks):
    """A block raises its flag, then each lane that looks at another block's flag has a fence of its own and looks.
    A look is sure to see a flag if some fence of that flag's block (all are behind the raising) comes before the
    looking lane's.  Whatever the order of the fences, the looks of at least one block see all flags: if every block
    missed one, each missed block's fences would all come later, in a circle."""
    lanes = [(b, o) for b in range(blocks) for o in range(blocks) if o != b]        # block b's lane that looks at o's flag
    if len(lanes) <= 6:
        orders = itertools.permutations(lanes)
    else:
        r = random.Random(0)
        orders = (r.sample(lanes, len(lanes)) for _ in range(20000))
    for order in orders:
        at = {lane: k for k, lane in enumerate(order)}
        first = [min(at[b, o] for o in range(blocks) if o != b) for b in range(blocks)]
        assert any(all(first[o] < at[b, o] for o in range(blocks) if o != b) for b in range(blocks))
