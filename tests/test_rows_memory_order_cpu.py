"""The order of tensor memory's reads and writes in the kernel of attention over several rows, read from its source: a
race there could not be seen in a result."""

import os
import re

from tests.test_kernel_order_cpu import ROOT, kernels

PATH = os.path.join(ROOT, "paper_2506_03781_gb300", "csrc", "uq_rows.cuh")


def test_scores_are_read_before_the_other_half_writes_weights_over_them():
    """Two warpgroups share a tile of rows, and where scores were weights go: what one has read is known to the other
    (a fence, the barrier, a fence) before that one's first store."""
    body, = (b for b in kernels(PATH) if "take_tensor_memory(" in b)
    step = body[body.index("auto in_order = [&](auto MIXED)"):]
    step = step[:step.index("if (mixed) in_order(")]
    marks = [m.group() for m in re.finditer(r"tc::load32\(|tc::wait_load\(|tc::fence_before\(\)|exchange\(\)|tc::fence_after\(\)|lift_to\(|\bweigh\(", step)]
    assert marks == ["tc::load32(", "tc::wait_load(", "tc::fence_before()", "exchange()", "tc::fence_after()", "lift_to(", "weigh("]
