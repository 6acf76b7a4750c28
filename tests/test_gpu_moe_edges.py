"""Calls of the mixture of experts that its other tests leave out: infinities and NaN among the tokens' values, a router over
more tokens than a wave of the GPU's SMs, the gradient of rows that were weighted on their way out.

Tolerances: as in test_gpu_moe_rows.py (half a bf16 step; a sum of n products in fp32 within n 2^-24 of their magnitudes) and
test_gpu_moe_route.py (100 units of 2^-23 relative to a weight)."""
import numpy as np
import pytest
import torch

import _moe as M
from _util import lib
from test_gpu_moe_route import choice, logits, weights_of
from test_gpu_moe_rows import near, some_plan

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


@pytest.mark.parametrize("form", ["nvfp4", "mxfp4", "mxfp4 rotated"])
def test_values_that_are_not_finite_are_the_quantizers(N, form):
    tokens, cols = 40, 320
    plan, _ = some_plan(N, tokens)
    x = M.rand_bf16((tokens, cols), 3, 4.0)
    for i, v in enumerate((INF, -INF, NAN, -NAN, 3e38, -3e38, 1e-40, -0.0)):
        x[3 * i, 17 * i] = v          # one in a block
        x[3 * i + 1, 32:64] = v       # a block of nothing else
        x[3 * i + 2, 100:104] = torch.tensor([v, -v, INF, 1.0])
    R, rotate = plan.max_rows, form.endswith("rotated")
    codes = torch.empty(tokens, cols // 2, dtype=torch.uint8, device="cuda")
    rc = torch.full((R, cols // 2), 0xA5, dtype=torch.uint8, device="cuda")
    rs = torch.full((R * cols // 16,), 0xA5, dtype=torch.uint8, device="cuda")
    if form == "nvfp4":
        g = torch.tensor([0.004], device="cuda")
        scales = torch.empty(N.nvfp4_scales_bytes(tokens, cols, N.SCALES_ROWMAJOR), dtype=torch.uint8, device="cuda")
        N.nvfp4_quantize(x, g, codes, scales, N.SCALES_ROWMAJOR)
        N.moe_dispatch_nvfp4(plan, x, g, rc, rs)
    else:
        half = torch.empty(tokens, cols // 32, dtype=torch.uint8, device="cuda")
        N.mxfp4_quantize(x, codes, half, N.SCALES_ROWMAJOR, rotate=rotate)
        scales = half.repeat_interleave(2, 1)
        N.moe_dispatch_mxfp4(plan, x, rc, rs, rotate=rotate)
    back = torch.empty(R, cols // 16, dtype=torch.uint8, device="cuda")
    N.nvfp4_scales_relayout(rs, back, R, cols, N.SCALES_MMA, N.SCALES_ROWMAJOR)
    t, j = np.nonzero(plan.row_of.cpu().numpy() >= 0)
    at, t = plan.row_of[t, j].long(), torch.as_tensor(t, device="cuda")
    assert torch.equal(rc[at], codes[t]) and torch.equal(back[at], scales.view(tokens, -1)[t])
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("tokens,experts,k,bias", [(20001, 64, 8, False), (5003, 256, 8, True), (70000, 8, 2, False)])
def test_a_router_over_many_tokens(N, tokens, experts, k, bias):
    l = logits(tokens, experts, 5)
    b = torch.linspace(-0.2, 0.2, experts, device="cuda") if bias else None
    idx = torch.full((tokens, k), 99999, dtype=torch.int32, device="cuda")
    w = torch.full((tokens, k), NAN, device="cuda")
    N.moe_route(l, idx, w, score=N.MOE_SIGMOID if bias else N.MOE_SOFTMAX, bias=b)
    l64, got = l.double().cpu().numpy(), idx.cpu().numpy()
    if bias:  # by 32 bits: in 64, neighbours may lie 2^-21 of their sizes the wrong way round
        key = 1 / (1 + np.exp(-l64)) + b.double().cpu().numpy()
        chosen = np.take_along_axis(key, got.astype(np.int64), 1)
        slack = 2.0 ** -21 * (1 + np.abs(chosen))
        assert (np.diff(chosen, axis=1) <= slack[:, 1:]).all()
        rest = key.copy()
        np.put_along_axis(rest, got.astype(np.int64), -np.inf, 1)
        assert (rest.max(1) <= chosen[:, -1] + slack[:, -1]).all()
        assert (np.sort(got, 1)[:, 1:] > np.sort(got, 1)[:, :-1]).all()
    else:
        assert np.array_equal(got, choice(l64, k))
    want = weights_of(l64, got, bias, True, 1.0)
    assert (np.abs(w.double().cpu().numpy() - want) <= 100 * 2.0 ** -23 * want).all()
    d_w = torch.randn(tokens, k, device="cuda")
    d_l = torch.full((tokens, experts), NAN, device="cuda")
    N.moe_route_backward(l, idx, d_w, d_l, score=N.MOE_SIGMOID if bias else N.MOE_SOFTMAX)
    # w (D - sum D w), times 1 - p for sigmoid, and nothing for the others.  Each of the terms within 100 units of its size, and
    # the sum of k of them.
    W, D, i = torch.as_tensor(want, device="cuda"), d_w.double(), idx.long()
    grad = W * (D - (D * W).sum(1, keepdim=True))
    if bias:
        grad = grad * torch.sigmoid(-l.double().gather(1, i))
    most = D.abs().max(1, keepdim=True).values
    assert ((d_l.gather(1, i).double() - grad).abs() <= 300 * 2.0 ** -23 * 2 * W * most).all()
    assert not d_l.scatter(1, i, 0.0).any()
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("tokens,cols", [(1, 8), (33, 2048), (400, 1000)])
def test_the_gradient_of_weighted_rows(N, tokens, cols):
    """rows = w x: dx is moe_combine of the rows' gradient with the same weights, dw moe_combine_backward's with x in place of
    its d_out and without its other output."""
    plan, _ = some_plan(N, tokens)
    x, w = M.rand_bf16((tokens, cols), 3), torch.randn(tokens, 3, device="cuda")
    d_rows = M.rand_bf16((plan.max_rows, cols), 4)
    d_x, d_w = torch.empty_like(x), torch.empty_like(w)
    N.moe_combine(plan, d_rows, d_x, weights=w)
    N.moe_combine_backward(plan, x, d_rows, w, None, d_w)
    row_of = plan.row_of.long()
    x64, w64 = x.double().requires_grad_(), w.double().requires_grad_()
    has = (row_of >= 0)
    rows = torch.zeros(plan.max_rows, cols, dtype=torch.float64, device="cuda")
    t, j = has.nonzero(as_tuple=True)
    rows = rows.index_put((row_of[t, j],), w64[t, j, None] * x64[t])
    (rows * d_rows.double()).sum().backward()
    near(d_x, x64.grad.cpu().numpy(), 3 * 2.0 ** -24 * (w64.abs()[..., None] * torch.where(
        has[..., None], d_rows.double()[row_of.clamp(min=0)].abs(), 0.0)).sum(1).detach().cpu().numpy())
    mag = torch.where(has, (x64.abs()[:, None] * d_rows.double()[row_of.clamp(min=0)].abs()).sum(-1), 0.0).detach()
    assert ((d_w.double() - w64.grad).abs() <= (cols / 8 + 10) * 2.0 ** -24 * mag).all()
    assert N.nvfp4_get_device_status() == 0


def test_the_gradient_of_weighted_rows_is_that_of_differences(N):
    """Small integers: exact in bf16 and fp32."""
    tokens, cols = 6, 16
    plan, _ = some_plan(N, tokens)
    gen = torch.Generator(device="cuda").manual_seed(2)

    def ints(*shape):
        return torch.randint(-2, 3, shape, generator=gen, device="cuda").float()
    x, w, c = ints(tokens, cols).to(BF), ints(tokens, 3), ints(plan.max_rows, cols).to(BF)

    def value(x, w):
        rows = torch.zeros(plan.max_rows, cols, dtype=BF, device="cuda")
        N.moe_dispatch(plan, x, rows, weights=w)
        return (rows.double() * c.double()).sum().item()
    d_x, d_w, at = torch.empty_like(x), torch.empty_like(w), value(x, w)
    N.moe_combine(plan, c, d_x, weights=w)
    N.moe_combine_backward(plan, x, c, w, None, d_w)
    for t in range(tokens):
        for j in range(3):
            moved = w.clone()
            moved[t, j] += 1
            assert value(x, moved) - at == d_w[t, j].item()
        for i in range(0, cols, 5):
            moved = x.clone()
            moved[t, i] += 1
            assert value(moved, w) - at == d_x[t, i].item()
