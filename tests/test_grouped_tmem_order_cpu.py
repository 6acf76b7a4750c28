"""The experts' linears allocate tensor memory before they let their successor start, as the other kernels with tensor
memory do: a successor's CTA on the same SM could otherwise take the memory that this one has yet to ask for.  Read from
the source: the order is not something that a run shows."""
import os
import re

from _util import ROOT

SOURCE = os.path.join(ROOT, "paper_2606_15682_gb300", "csrc", "gemm_grouped.cu")


def test_a_barrier_stands_between_allocation_and_release():
    text = open(SOURCE).read()
    calls = list(re.finditer(r"^\s+if \([^\n]*\) pair_tmem_alloc\(", text, flags=re.M))
    assert len(calls) == 1
    between = text[calls[0].end():text.index("griddep_wait_and_release();", calls[0].end())]
    assert "cluster_sync_all();" in between
