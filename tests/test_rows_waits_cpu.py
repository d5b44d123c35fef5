"""Waits of the kernel of attention over several rows that a test cannot reach on a GPU, read from its source: how long who
passes over a unit waits for the next, and what is waited for when a wait has run out."""

import os
import re

import pytest

from tests.test_kernel_order_cpu import ROOT

PATH = os.path.join(ROOT, "paper_2506_03781_gb300", "csrc", "uq_rows.cuh")
SOURCE = re.sub(r"//[^\n]*", "", open(PATH).read())


def constant(name):
    return eval(re.search(rf"constexpr long long {name} = (.*?);", SOURCE).group(1).replace("ll", ""))


def test_who_passes_over_a_unit_waits_as_long_as_the_others_need_for_it():
    """A tile of rows that has no part in a unit waits for the next one through all of its tiles: 2^30 positions, 64 a tile,
    of 5000 clocks (4-bit rows, fp32) at most, are far more than the second that other waits last."""
    walk = SOURCE[SOURCE.index("auto next_unit = [&]"):]
    walk = walk[:walk.index("auto load_queries")]
    assert re.search(r"for \(long long limit = kWaitClocks;;\) \{\s*const Item\* const it = next_item\(limit\);", walk)
    limit = re.search(r"limit = (kWaitClocks \+ .*?);", walk[walk.index("return it;"):]).group(1)
    for tiles in (1, 100, 10 ** 6, (1 << 30) // 64 + 2):
        clocks = eval(limit.replace("it->end - it->tile", "tiles"), {}, dict(tiles=tiles, kWaitClocks=constant("kWaitClocks"), kTileClocks=constant("kTileClocks")))
        assert 4 * 5000 * tiles + (1 << 31) <= clocks < 1 << 62
    assert "tma::bar_wait(tma::smem_addr(&bar), parity, limit)" in SOURCE
    assert "wait(item_full[item_no % kItems], (item_no / kItems) & 1, limit)" in SOURCE


def test_loops_without_a_count_end():
    """Each of them goes through a bounded wait, or takes something from a finite rest."""
    loops = re.findall(r"while \((.*)\) \{\n|for \(([^;]*;;)\)", SOURCE)
    kinds = {a or b for a, b in loops}
    assert kinds == {"rem > 0", "j >= u.groups", "hi - b > 1", "const Item* const it = alive ? next_item() : nullptr", "alive && it",
                     "long long limit = kWaitClocks;;"}
    assert "bar_try_wait" not in SOURCE and "mbarrier" not in SOURCE


@pytest.mark.parametrize("ring", range(3, 17))
@pytest.mark.parametrize("v", (0, 1))
def test_after_a_timeout_the_copies_that_may_be_on_their_way_are_waited_for(ring, v):
    """A copier has started halves v, v + 2, ... and each but the first ones only when the half before it in its place was
    used up, and halves are used up in their order: those from then on may still be on their way, and no other."""
    first = re.search(r"for \(uint32_t h = (.*?); h < half; h \+= 2\)", SOURCE).group(1)
    cond, a, b = re.match(r"(.*) \? (.*) : (.*)$", first.replace("(uint32_t)", "").replace("kRing", "ring")).groups()
    for n in range(40):
        half = v + 2 * n
        started = list(range(v, half, 2))
        used_up = half - 2 - ring                    # what the last one's start waited for, if it waited
        drained = list(range(eval(a if eval(cond) else b), half, 2))
        assert drained == [h for h in started if h > used_up]


def test_products_on_their_way_end_before_tensor_memory_is_given_back():
    tail = SOURCE[SOURCE.index("tma::smem_addr(&drain), 0)") - 300:]
    marks = ["if (!alive) {", "tc::commit(tma::smem_addr(&drain))", "tma::bar_wait(tma::smem_addr(&drain), 0)", "__syncthreads();", "tc::dealloc("]
    at = [tail.index(m) for m in marks]
    assert at == sorted(at)
