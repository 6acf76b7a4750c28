"""Tensor memory is allocated before a kernel lets its successor start.

griddepcontrol.launch_dependents takes effect when one thread of every CTA has issued it.  A successor's CTA on the same
SM could then take the tensor memory that this CTA's allocating warp has yet to ask for, and wait for this kernel to end
while it waits for the memory.  So a barrier of the whole CTA stands between the two.  Read from the sources: the order
is not something that a run shows.
"""
import os
import re

import pytest

from _util import ROOT

CSRC = os.path.join(ROOT, "paper_2606_15682_gb300", "csrc")


def kernels():
    """(file, line, text from a call of tmem_alloc to the next griddep_wait_and_release)."""
    found = []
    for name in sorted(os.listdir(CSRC)):
        text = open(os.path.join(CSRC, name)).read()
        for m in re.finditer(r"^\s+(?:if \([^\n]*\) )?tmem_alloc(?:_pair)?\(", text, flags=re.M):
            release = text.find("griddep_wait_and_release();", m.end())
            assert release >= 0
            found.append((name, text.count("\n", 0, m.end()) + 1, text[m.end():release]))
    return found


def test_every_kernel_with_tensor_memory_is_found():
    assert {name for name, _, _ in kernels()} == {"gemm.cu", "extend_rows.cu", "extend_tiles.cu"}


@pytest.mark.parametrize("name,line,between", kernels(), ids=lambda v: str(v)[:20])
def test_a_barrier_stands_between_allocation_and_release(name, line, between):
    assert re.search(r"__syncthreads\(\);|cluster_sync_all\(\);", between), f"{name}:{line}"
