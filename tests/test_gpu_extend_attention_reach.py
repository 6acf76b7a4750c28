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
from test_gpu_extend_attention_long import reference

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


@pytest.mark.parametrize("tokens", [1, 3, 5, 6, 60])
@pytest.mark.parametrize("length", [2 ** 24 + 41, 2 ** 25 + 1])
def test_distance_bias_at_positions_past_24_bits(N, tokens, length):
    """Only the last pages are there.  |p - t| is a small number also where p and t themselves need more bits than fp32 has."""
    page, hq, present = 4096, 5, 2
    per = -(-length // page)
    case = P.Case(N, [page * present], 1, page, 0, seed=610)
    shown = case.table[0].copy()
    table = np.full((1, per), -1, np.int32)
    table[0, per - present:] = shown
    case.lens, case.per = [length], per
    case.lens_dev.copy_(torch.tensor([length], dtype=torch.int32))
    case.set_table(table)
    q = queries(tokens, hq, 41)
    slopes = np.array([0.5, 0.25, 0.1, 1.0, 2.0], np.float32)
    got = run(N, case, q, [tokens], slopes=torch.from_numpy(slopes).cuda())
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 0
    # The same keys and distances in a sequence that starts at the first page that is there.
    first = (per - present) * page
    case.lens, case.per = [length - first], present
    case.lens_dev.copy_(torch.tensor(case.lens, dtype=torch.int32))
    case.set_table(shown[None, :])
    check_long(N, case, q, [tokens], slopes=slopes)
    want, bound, _ = reference(case, q, [tokens], slopes=slopes)
    over = np.abs(got.double().cpu().numpy() - want) - (P.half_ulp(want) * (1 + 2.0 ** -6) + bound)
    assert over.max() <= 0, f"worst excess {over.max():.3e}"


@pytest.mark.parametrize("news", [[1, 1], [4, 4], [150, 20], [40, 40]])
@pytest.mark.parametrize("scale", [1e-9, 1e-30, 1e-38])
@pytest.mark.parametrize("capacity", [0, 400])
@pytest.mark.parametrize("opt", [{}, dict(window=70), dict(logit_cap=5.0)])
def test_scales_and_queries_whose_product_underflows(N, news, scale, capacity, opt):
    """Scores of zero: a plain mean of the visible V, with keys hidden from some of a tile's rows."""
    lens = [390, 200] if capacity else [1500, 800]
    case = P.Case(N, lens, 2, 0, 0, seed=620, capacity=capacity or None)
    for spread in (0.0, 2.0 ** -100, 1.0):
        check_long(N, case, queries(sum(news), 10, 42, spread=spread), news, scale=scale, **opt)
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("news", [[1, 1], [4, 4], [150, 20]])
@pytest.mark.parametrize("capacity", [0, 400])
def test_zero_keys_under_scales_and_queries_whose_product_overflows(N, news, capacity):
    """Every product of Q and K is 0, and so is every score."""
    lens = [390, 200] if capacity else [1500, 800]
    case = P.Case(N, lens, 2, 0, 0, seed=630, capacity=capacity or None)
    codes, scales = case.data["k"]
    case.data["k"] = (np.zeros_like(codes), scales)
    case.cache.k_codes.zero_()
    q = queries(sum(news), 10, 43, spread=2.0 ** 125)
    check_long(N, case, q, news, scale=1e4)
    check_long(N, case, q, news, scale=3e38, window=70)
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("lens", [[1, 2, 3, 5, 9], [20, 40, 16, 17, 64], [129, 300, 512, 90, 250]])
@pytest.mark.parametrize("new", [1, 2, 4, 6, 60])
@pytest.mark.parametrize("capacity", [513, 8192])
def test_short_sequences_in_a_wide_table(N, lens, new, capacity):
    """The buffers' context chooses the weights' precision: f16's stated bound, 2^-29 of the largest weight, at any length."""
    hq, hkv = 10, 2
    news = [min(new, n) for n in lens]
    case = P.Case(N, lens, hkv, 64, 0, seed=640, capacity=capacity)
    for spread in (1.0, 60.0):  # weights that fall off slowly and fast
        q = queries(sum(news), hq, 44, spread=spread)
        check_long(N, case, q, news)
        check_long(N, case, q, news, slopes=np.linspace(0.02, 1.0, hq).astype(np.float32))
    assert N.nvfp4_get_device_status() == 0
