"""extend_attention_nvfp4 with caps far above the scores, and with rows far apart under one cap, by each kernel.

c tanh(s / c) is s itself where c is large.  The result is held to the tolerances of the two files that the references
come from: nothing is added for the cap, since its relative error (2^-20 of a score of a few units) is far below the
2^-10 of the weights.
"""
import numpy as np
import pytest
import torch

import _paged as P
from _util import lib
from test_gpu_extend_attention import check as check_short
from test_gpu_extend_attention import queries, run
from test_gpu_extend_attention_long import check as check_long
from test_gpu_extend_attention_long import reference

pytestmark = pytest.mark.gpu

CAPS = [1e3, 1e4, 1e5, 1e6, 1e8, 1e12, 1e30, 3.4e38]
# Rows of a sequence and KV head: 5, 20 and 30 (few rows), then tiles.
NEWS = [[1, 1], [4, 4], [6, 6], [150, 20]]


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("news", NEWS)
@pytest.mark.parametrize("page,fmt", [(0, 0), (48, 1)])
def test_caps_far_above_the_scores(N, news, cap, page, fmt):
    for lens, check in (([1500, 800], check_long), ([400, 333], check_short)):
        case = P.Case(N, lens, 2, page, fmt, seed=400)
        q = queries(sum(news), 10, 20, spread=2.0)
        check(N, case, q, news, logit_cap=cap)
        check(N, case, q * 16, news, logit_cap=cap)
        check(N, case, q, news, logit_cap=cap, slopes=np.linspace(0.0, 0.1, 10).astype(np.float32))
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("news", NEWS)
@pytest.mark.parametrize("cap", [1e4, 1e6])
def test_a_row_at_the_cap_leaves_the_others_exact(N, news, cap):
    """Head 2 of each group of five has scores of the cap's size, its neighbours in the warp scores of a few units."""
    case = P.Case(N, [1500, 800], 2, 0, 0, seed=410)
    q = queries(sum(news), 10, 21)
    q[:, 2::5] *= 2.0 ** int(np.log2(cap) + 4)
    out = run(N, case, q, news, logit_cap=cap)
    torch.cuda.synchronize()
    ref, bound, _ = reference(case, q, news, logit_cap=cap)
    keep = [h for h in range(10) if h % 5 != 2]
    y = out.double().cpu().numpy()
    assert np.isfinite(y).all()
    over = (np.abs(y - ref) - (P.half_ulp(ref) * (1 + 2.0 ** -6) + bound))[:, keep]
    assert over.max() <= 0, f"worst excess {over.max():.3e}"


@pytest.mark.parametrize("news", NEWS)
@pytest.mark.parametrize("cap", [1e-30, 1e-3, 0.5, 2.0])
def test_caps_below_the_scores(N, news, cap):
    case = P.Case(N, [1500, 800], 2, 32, 0, seed=420)
    q = queries(sum(news), 10, 22, spread=4.0)
    check_long(N, case, q, news, logit_cap=cap)
    q[:, 0] = 0  # scores of 0 beside them
    check_long(N, case, q, news, logit_cap=cap)
