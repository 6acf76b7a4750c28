"""Failure detection of extend_attention_nvfp4 without a GPU fault: a stage that never fills.

The test-only knob makes one barrier of CTA 0 wait for an arrival that never comes.  The bounded waits run out after
some 2 s, every role of the CTA stops, the call reports TIMEOUT, and the next call is right again.
"""
import time

import pytest
import torch

import _paged as P
from _util import lib
from test_gpu_extend_attention import check as check_short
from test_gpu_extend_attention import queries, run
from test_gpu_extend_attention_long import check as check_long

pytestmark = pytest.mark.gpu

# (new tokens, lengths, options): decode with one part and with several, 8 rows by the rows kernel, 16, 24 and 32 rows,
# tiles of one and of two halves, each kind of context and of score.
FORMS = [
    ([1, 1], [600, 130], {}), ([1, 1], [9000, 700], dict(logit_cap=20.0)), ([1, 1], [300, 40], {}),
    ([2, 2], [1500, 800], {}), ([4, 4], [1500, 800], {}), ([4, 4], [5000, 800], dict(logit_cap=20.0)),
    ([6, 6], [1500, 800], {}), ([6, 6], [300, 100], {}),
    ([20, 20], [1500, 800], {}), ([150, 60], [1500, 800], {}), ([150, 60], [1500, 800], dict(logit_cap=20.0, window=700)),
    ([60, 60], [300, 200], {}),
]


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


@pytest.mark.parametrize("which", range(len(FORMS)))
def test_a_lost_stage_times_out_and_the_next_call_is_right(N, which):
    news, lens, opt = FORMS[which]
    page, fmt = ((0, 0), (64, 1))[which % 2]
    case = P.Case(N, lens, 2, page, fmt, seed=900 + which)
    q = queries(sum(news), 10, 70)
    check = check_long if max(lens) > 512 else check_short
    check(N, case, q, news, **opt)
    assert N.nvfp4_get_device_status() == 0
    N.nvfp4_debug_inject_fault(N.FAULT_ATTN_SKIP_STAGE)
    try:
        t0 = time.time()
        run(N, case, q, news, **opt)
        torch.cuda.synchronize()
        waited = time.time() - t0
    finally:
        N.nvfp4_debug_inject_fault(N.FAULT_NONE)
    assert N.nvfp4_get_device_status() == 6
    assert 1.0 < waited < 8.0, "the lost stage is waited for, and not for ever"
    check(N, case, q, news, **opt)
    assert N.nvfp4_get_device_status() == 0
