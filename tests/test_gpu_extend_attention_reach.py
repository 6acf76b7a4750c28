"""extend_attention_nvfp4 at the ends of its arguments' ranges: windows, positions, and tables far wider than the sequences.

Tolerances are those of the files that the references come from.
"""
import numpy as np
import pytest
import torch

import _paged as P
from _util import lib
from test_gpu_extend_attention import queries, run
from test_gpu_extend_attention_long import check as check_long

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


@pytest.mark.parametrize("news,lens", [([6, 8], [2, 3]), ([12, 5], [7, 1]), ([3, 3], [900, 0]), ([90, 40], [60, 700])])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 4, 2 ** 30])
@pytest.mark.parametrize("hq,hkv,capacity", [(2, 2, 1000), (6, 2, 1000), (5, 1, 100)])
def test_windows_past_every_key(N, news, lens, window, hq, hkv, capacity):
    """A window wider than any context is no window, also for sequences that bring more queries than they hold tokens."""
    lens = [min(n, capacity) for n in lens]
    case = P.Case(N, lens, hkv, 0, 0, seed=600, capacity=capacity)
    q = queries(sum(news), hq, 40)
    out = check_long(N, case, q, news, window=window)
    assert torch.equal(out, run(N, case, q, news))
    assert N.nvfp4_get_device_status() == 0
