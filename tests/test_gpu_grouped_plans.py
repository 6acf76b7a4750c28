"""The experts' linears with plans that moe_sort did not write for them: one left from a larger step names more rows of an
expert than there are choices.  Such an expert has as many rows as there are choices, and nothing behind them is written."""
import pytest
import torch

import _moe as M
from _util import lib

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


# Choices on either side of where a launch needs boxes of more rows (32, 128), few and many an expert: both forms.
@pytest.mark.parametrize("choices,experts", [(1, 1), (1, 3), (20, 1), (20, 2), (32, 1), (33, 1), (33, 4), (100, 1), (100, 2),
                                             (127, 3), (128, 1), (129, 1), (129, 5)])
@pytest.mark.parametrize("form", ["rows", "rows mxfp4", "nvfp4", "mxfp4", "mxfp4 rotated"])
def test_a_plan_of_more_rows_than_choices_is_cut_to_them(N, choices, experts, form):
    idx = torch.full((choices, 1), experts - 1, dtype=torch.int32)
    plan, mx, k, n = M.make_plan(N, idx, experts), "mxfp4" in form, 512, 256
    a, w = M.Rows(N, plan, k, 2, mx), M.Weights(N, experts, n, k, 5, mx)
    R = plan.max_rows
    out = torch.full((R + 256, n), -7.0, dtype=BF, device="cuda")
    codes = torch.full((R + 256, n // 4), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full(((R + 256) * n // 32,), 0xA5, dtype=torch.uint8, device="cuda")
    size, g = R * n // 32, torch.tensor([0.02], device="cuda")

    def call():
        if form == "rows":
            N.nvfp4_linear_grouped(plan, a.codes, a.scales, a.g, w.codes, w.scales, w.g, out[:R], n, k)
        elif form == "rows mxfp4":
            N.mxfp4_linear_grouped(plan, a.codes, a.scales, w.codes, w.scales, out[:R], n, k)
        elif mx:
            N.mxfp4_linear_grouped_swiglu_quantize(plan, a.codes, a.scales, w.codes, w.scales, n // 2, k, codes[:R],
                                                   scales[:size], rotate=form.endswith("rotated"))
        else:
            N.nvfp4_linear_grouped_swiglu_quantize(plan, a.codes, a.scales, a.g, w.codes, w.scales, w.g, n // 2, k, g,
                                                   codes[:R], scales[:size])
        torch.cuda.synchronize()
        assert N.nvfp4_get_device_status() == 0
        return out.clone(), codes.clone(), scales.clone()
    right = call()
    for rows in (R, 1 << 30):  # to the buffers' end, and past it
        stale = torch.zeros(experts, dtype=torch.int32)
        stale[experts - 1] = rows
        plan.rows.copy_(stale)
        assert all(torch.equal(x, y) for x, y in zip(call(), right)), "the experts' rows and those behind them"
    assert (out[choices:] == -7).all() and (codes[choices:] == 0xA5).all()
