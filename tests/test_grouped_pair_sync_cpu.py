"""How the two CTAs of a pair in the experts' linears hear of each other.  A wait for what the other CTA's threads arrive with
has to acquire at the scope of the cluster; and a place of the queue of units is handed back, for the peer to overwrite, only
after one load has brought all of it into registers that are used.  Read from the source: a run does not show what the
hardware may not order."""
import os
import re

import pytest

from _util import ROOT

TEXT = open(os.path.join(ROOT, "paper_2606_15682_gb300", "csrc", "gemm_grouped.cu")).read()
KERNEL = TEXT[TEXT.index("grouped_kernel(const __grid_constant__"):TEXT.index("host ---")]


@pytest.mark.parametrize("bar", ["unit_full", "unit_empty", "unit_begun", "acc_empty"])
def test_waits_for_the_other_cta_acquire_at_cluster_scope(bar):
    waits = re.findall(rf"(\w+)\(&?{bar}\b(?!\[i\])[^;]*;", KERNEL)
    waits = [w for w in waits if "wait" in w]
    assert waits and set(waits) == {"wait_pair"}
    body = KERNEL[KERNEL.index("const auto wait_pair"):]
    assert "mbar_wait_bounded_cluster(" in body[:body.index("};")]


def test_a_place_of_the_queue_is_read_by_one_load_before_it_is_handed_back():
    reads = [m for m in re.finditer(r"queue\[slot\]", KERNEL) if "send_16" not in KERNEL[m.start() - 30:m.start()]]
    assert len(reads) == 1 and KERNEL[:reads[0].start()].endswith("load_unit(&")
    after = KERNEL[reads[0].end():]
    back = after.index("arrive_relaxed(pair_address(&unit_empty[slot], 1))")
    assert "__all_sync(0xffffffffu, t->tokens != 0)" in after[:back]
    load = TEXT[TEXT.index("Unit load_unit("):]
    load = load[:load.index("\n}")]
    assert load.count("asm volatile") == 1 and "ld.shared.v4.b32" in load
