"""extend_attention_nvfp4 with queries that are not finite: NaN for those that see a key, zeros for those that see none."""
import numpy as np
import pytest
import torch

import _paged as P
from _util import lib
from test_gpu_extend_attention import queries, run
from test_gpu_extend_attention_long import check, reference

pytestmark = pytest.mark.gpu

BAD = [float("nan"), float("inf"), -float("inf")]
# Rows of a sequence and KV head: decode, few rows, tiles with both halves and with one; long and short contexts.
FORMS = [([1, 1], [1500, 800]), ([1, 1], [9000, 5]), ([4, 4], [1500, 800]), ([6, 6], [5000, 800]), ([20, 20], [1500, 800]),
         ([150, 20], [1500, 800]), ([1, 1], [300, 40]), ([4, 4], [300, 40]), ([60, 40], [300, 40])]


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("which", range(len(FORMS)))
@pytest.mark.parametrize("opt", [{}, dict(logit_cap=20.0), dict(slopes="s"), dict(logit_cap=5.0, slopes="s")])
@pytest.mark.parametrize("page,fmt", [(0, 0), (64, 1)])
def test_such_a_row_is_nan_and_no_other(N, which, bad, opt, page, fmt):
    news, lens = FORMS[which]
    opt = dict(opt)
    if "slopes" in opt:
        opt["slopes"] = np.linspace(0, 0.1, 10).astype(np.float32)
    case = P.Case(N, lens, 2, page, fmt, seed=700)
    q = queries(sum(news), 10, 50).contiguous()
    q[0, 3, 5] = bad                       # one head of the first token
    q[sum(news) - 1, 7, 127] = bad         # and of the last
    rows = [(0, 3), (sum(news) - 1, 7)]
    dev = {k: (torch.from_numpy(v).cuda() if k == "slopes" else v) for k, v in opt.items()}
    out = run(N, case, q, news, **dev)
    torch.cuda.synchronize()
    hit = torch.zeros(q.shape[:2], dtype=torch.bool)
    for i, h in rows:
        hit[i, h] = True
    nan = out.isnan().cpu()
    assert nan[hit].all(), "every channel of the row"
    assert not nan[~hit].any()
    # The other rows are what they are without it, within the tolerance of the longer contexts' file.
    clean = q.clone()
    for i, h in rows:
        clean[i, h] = 0
    ref, bound, _ = reference(case, clean, news, **opt)
    over = np.abs(out.double().cpu().numpy() - ref) - (P.half_ulp(ref) * (1 + 2.0 ** -6) + bound)
    assert over[~hit.numpy()].max() <= 0
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("news,capacity", [([3, 3], 2000), ([60, 40], 2000), ([3, 3], 100), ([60, 40], 100)])
def test_such_a_row_that_sees_nothing_is_zero(N, news, capacity, bad):
    case = P.Case(N, [90, 0], 2, 0, 0, seed=710, capacity=capacity)
    q = queries(sum(news), 10, 51).contiguous()
    q[news[0]:, :, 9] = bad                      # the whole empty sequence
    doc = np.zeros(sum(news), np.int32)
    q[1, :, 9], doc[1] = bad, 95                 # and a document that starts after its query
    check(N, case, q, news, doc_start=doc)
    assert N.nvfp4_get_device_status() == 0
