"""The order of steps in the kernel of attention over several rows that would hang a GPU in another order, read from its
source (as tests/test_kernel_order_cpu.py does for kernels that allocate in their own body)."""

import os

from tests.test_kernel_order_cpu import ROOT, kernels

PATH = os.path.join(ROOT, "paper_2506_03781_gb300", "csrc", "uq_rows.cuh")


def test_tensor_memory_is_taken_between_the_grid_wait_and_the_start_of_dependents():
    bodies = [b for b in kernels(PATH) if "take_tensor_memory(" in b]
    assert len(bodies) == 1
    body = bodies[0]
    wait, alloc, start, free = (body.index(s) for s in ("inputs_ready();", "take_tensor_memory(", "dependents_may_start();", "tc::dealloc("))
    assert wait < alloc < start < free
    assert "__syncthreads();" in body[alloc:start]         # one thread's signal counts for its block


def test_every_wait_is_bounded():
    """Waits on barriers go through bar_wait, which gives up; none spins by itself."""
    for body in kernels(PATH):
        assert "bar_try_wait" not in body and "mbarrier" not in body and "while (true)" not in body
