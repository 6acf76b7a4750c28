"""The experts' linears against 64-bit products of the same 4-bit operands.

Tolerances: half a bf16 step (1 + 2^-6 of it), and K additions in 32 bits, each within 2^-23 of the sum of magnitudes.  The
quantized SwiGLU output must be what the quantizer's recipe gives for some h within such an error of both products
(|SiLU'| <= 1.1), and (2 + |G| / 4) 2^-21 of h: 2^x within 2^-22 and its argument, 1.44 |G|, rounded twice (1.5 |G| 2^-24),
a sum 2^-24, a reciprocal 2^-23, two products 2^-24 each.
"""
import numpy as np
import pytest
import torch

import _moe as M
from _util import assert_mxfp4_within, assert_nvfp4_within, f32, lib, rotated_tolerance
from oracle import mxfp4_oracle as X
from oracle import nvfp4_oracle as O

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


RAGGED = [0, 1, 127, 128, 129, 300, 0, 5, 256, 513, 31, 0]
COUNTS = {"one": [1], "none": [0, 0, 0], "first of many": [3] + [0] * 300, "few": [2, 0, 1, 4, 0, 3], "ragged": RAGGED,
          "large": [700, 70], "edges": [16, 17, 32, 33, 48, 64, 65, 96, 97, 160, 161, 192, 255, 257, 288],
          "thousand": [1] * 1024,
          # Few choices an expert, but some experts with more than a small tile of 64, 128 and 256 rows.
          "uneven": [300, 64, 65, 129, 1, 33, 193, 127] + [0] * 40}


def linear(N, plan, a, w, out, n, k, mx, g_a=None):
    if mx:
        N.mxfp4_linear_grouped(plan, a.codes, a.scales, w.codes, w.scales, out, n, k)
    else:
        N.nvfp4_linear_grouped(plan, a.codes, a.scales, a.g if g_a is None else g_a, w.codes, w.scales, w.g, out, n, k)


def check_linear(N, counts, n, k, mx=False, per_expert=False, pad=0, seed=0):
    E = len(counts)
    plan = M.make_plan(N, M.choices(counts, 2 if sum(counts) > 1 else 1, seed, drop=3), E)
    a, w = M.Rows(N, plan, k, 11 + seed, mx), M.Weights(N, E, n, k, 100 + seed, mx)
    g_a = torch.linspace(0.001, 0.004, E, device="cuda") if per_expert else None
    out = torch.full((plan.max_rows, n + pad), -7.0, dtype=BF, device="cuda")
    linear(N, plan, a, w, out[:, :n], n, k, mx, g_a)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 0
    sums, mag = M.products(a.values, a.expert, w.values)
    g = np.ones(E, np.float32)
    if not mx:
        ga = f32(a.g if g_a is None else g_a)
        g = (ga * f32(w.g)).astype(np.float32)
    g = g.astype(np.float64)[a.expert][:, None]
    at = torch.as_tensor(a.at, device="cuda")
    got, want = out[at][:, :n].double().cpu().numpy(), sums * g
    over = np.abs(got - want) - M.half_ulp(want) * (1 + 2.0 ** -6) - k * 2.0 ** -23 * mag * g
    assert over.max(initial=-1) <= 0, over.max()
    rest = torch.ones(plan.max_rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert (out[rest] == -7).all() and (out[:, n:] == -7).all()
    return plan, a, w, out


@pytest.mark.parametrize("counts", COUNTS, ids=lambda c: c)
@pytest.mark.parametrize("mx", [False, True])
def test_rows_of_every_kind(N, counts, mx):
    check_linear(N, COUNTS[counts], 256, 512, mx)


@pytest.mark.parametrize("n", [16, 48, 128, 144, 240, 256, 272, 384, 512, 1040])
@pytest.mark.parametrize("k", [256, 768, 1536])
def test_sizes(N, n, k):
    check_linear(N, [5, 0, 130, 290], n, k, per_expert=True, pad=8)


@pytest.mark.parametrize("n", [16, 144, 272, 1040])
@pytest.mark.parametrize("k", [256, 1536])
def test_sizes_with_few_rows_an_expert(N, n, k):
    check_linear(N, [5, 0, 130, 70] + [0] * 20, n, k, per_expert=True, pad=8)


@pytest.mark.parametrize("inner", [128, 384, 1024])
@pytest.mark.parametrize("form", ["nvfp4", "mxfp4", "mxfp4 rotated"])
def test_swiglu_sizes_with_few_rows_an_expert(N, inner, form):
    check_swiglu(N, [5, 0, 130, 70] + [0] * 20, inner, 768, form != "nvfp4", form.endswith("rotated"), per_expert=False)


@pytest.mark.parametrize("counts", ["few", "ragged", "uneven"])
def test_a_long_sum(N, counts):
    check_linear(N, COUNTS[counts], 256, 5120)


def test_many_tiles(N):
    check_linear(N, [400, 900, 3, 250, 0, 640], 2048, 1024, seed=3)


@pytest.mark.parametrize("mx", [False, True])
def test_rows_are_the_dense_linears_to_the_accumulation(N, mx):
    """Each expert's rows through nvfp4_linear / mxfp4_linear: the same products, sums perhaps in another order."""
    plan, a, w, out = check_linear(N, [40, 200], 512, 1024, mx)
    start, rows = plan.row_start.tolist(), plan.rows.tolist()
    for e in range(2):
        n_rows = rows[e]
        dense = torch.empty(n_rows, 512, dtype=BF, device="cuda")
        sc = a.scales.view(-1, 128 * 64)[start[e] // 128:].contiguous()
        codes = a.codes[start[e]:start[e] + n_rows].contiguous()
        if mx:
            N.mxfp4_linear(codes, sc, w.codes[e], w.scales[e], dense, n_rows, 512, 1024)
        else:
            N.nvfp4_linear(codes, sc, a.g, w.codes[e], w.scales[e], w.g[e:e + 1], dense, n_rows, 512, 1024)
        d = (dense.double() - out[start[e]:start[e] + n_rows].double()).abs()
        assert (d <= dense.double().abs() * 2.0 ** -7 + 1e-3 * dense.double().abs().max()).all()


def unpack(plan, codes, scales, at, cols, mx):
    sc = O.scales_from_mma(scales.cpu().numpy(), plan.max_rows, cols)[at]
    return codes.cpu().numpy()[at], sc[:, ::2] if mx else sc, sc


def check_swiglu(N, counts, inner, k, mx=False, rotate=False, per_expert=True, seed=0):
    E = len(counts)
    plan = M.make_plan(N, M.choices(counts, 2 if sum(counts) > 1 else 1, seed, drop=1), E)
    a, w = M.Rows(N, plan, k, 21 + seed, mx), M.Weights(N, E, 2 * inner, k, 300 + seed, mx)
    codes = torch.full((plan.max_rows, inner // 2), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((plan.max_rows * inner // 16,), 0xA5, dtype=torch.uint8, device="cuda")
    g_out = (torch.linspace(0.01, 0.03, E, device="cuda") if per_expert else torch.tensor([0.02], device="cuda"))
    if mx:
        N.mxfp4_linear_grouped_swiglu_quantize(plan, a.codes, a.scales, w.codes, w.scales, inner, k, codes, scales,
                                               rotate=rotate)
    else:
        N.nvfp4_linear_grouped_swiglu_quantize(plan, a.codes, a.scales, a.g, w.codes, w.scales, w.g, inner, k, g_out,
                                               codes, scales)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 0
    sums, mag = M.products(a.values, a.expert, w.values)
    g = (f32(a.g) * f32(w.g)).astype(np.float64)[a.expert] if not mx else np.ones(len(a.at))
    both = (sums * g[:, None]).reshape(len(a.at), inner // 16, 2, 16)
    err = (k * 2.0 ** -23 * mag * g[:, None]).reshape(len(a.at), inner // 16, 2, 16)
    G, U = (both[:, :, i].reshape(len(a.at), inner) for i in (0, 1))
    eG, eU = (err[:, :, i].reshape(len(a.at), inner) for i in (0, 1))
    silu = G / (1 + np.exp(-G))
    h = silu * U
    tol = 1.1 * eG * np.abs(U) + (np.abs(silu) + 1.1 * eG) * eU + (2 + np.abs(G) / 4) * 2.0 ** -21 * np.abs(h) + 1e-30
    c, sc, whole = unpack(plan, codes, scales, a.at, inner, mx)
    if mx:
        assert (whole[:, ::2] == whole[:, 1::2]).all()
        if rotate:
            h, tol = X.rotate_blocks(h), rotated_tolerance(h, tol)
        assert_mxfp4_within(c, sc, h, tol)
    else:
        go = f32(g_out) if per_expert else np.full(E, f32(g_out)[0])
        for e in np.unique(a.expert):
            r = a.expert == e
            assert_nvfp4_within(c[r], sc[r], h[r], tol[r], go[e])
    rest = np.setdiff1d(np.arange(plan.max_rows), a.at)
    rc, _, rs = unpack(plan, codes, scales, rest, inner, mx)
    assert (rc == 0xA5).all() and (rs == 0xA5).all()


@pytest.mark.parametrize("counts", ["one", "none", "first of many", "few", "ragged", "large", "edges", "uneven"],
                         ids=lambda c: c)
@pytest.mark.parametrize("form", ["nvfp4", "mxfp4", "mxfp4 rotated"])
def test_swiglu_rows_of_every_kind(N, counts, form):
    check_swiglu(N, COUNTS[counts], 256, 512, form != "nvfp4", form.endswith("rotated"))


@pytest.mark.parametrize("inner", [128, 256, 384, 768, 1024])
@pytest.mark.parametrize("k", [256, 1280])
@pytest.mark.parametrize("form", ["nvfp4", "mxfp4", "mxfp4 rotated"])
def test_swiglu_sizes(N, inner, k, form):
    check_swiglu(N, [5, 0, 130, 290], inner, k, form != "nvfp4", form.endswith("rotated"), per_expert=False)


@pytest.mark.parametrize("bad", [0.0, -1.0, float("nan"), float("inf")])
def test_an_invalid_output_scale_is_reported_and_its_rows_are_zero(N, bad):
    plan = M.make_plan(N, M.choices([20, 200, 9], 1, 0), 3)
    a, w = M.Rows(N, plan, 256, 2), M.Weights(N, 3, 512, 256, 5)
    g = torch.tensor([0.02, bad, 0.02], device="cuda")
    codes = torch.full((plan.max_rows, 128), 0xA5, dtype=torch.uint8, device="cuda")
    scales = torch.full((plan.max_rows * 16,), 0xA5, dtype=torch.uint8, device="cuda")
    N.nvfp4_linear_grouped_swiglu_quantize(plan, a.codes, a.scales, a.g, w.codes, w.scales, w.g, 256, 256, g, codes, scales)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 1
    c, sc, _ = unpack(plan, codes, scales, a.at, 256, False)
    zero = (c & 0x77 == 0).all(1) & (sc == 0).all(1)
    assert zero[a.expert == 1].all() and not zero[a.expert != 1].any()


def test_an_invalid_output_scale_of_an_expert_without_rows_is_none(N):
    plan = M.make_plan(N, M.choices([20, 0], 1, 0), 2)
    a, w = M.Rows(N, plan, 256, 2), M.Weights(N, 2, 512, 256, 5)
    codes = torch.empty(plan.max_rows, 128, dtype=torch.uint8, device="cuda")
    scales = torch.empty(plan.max_rows * 16, dtype=torch.uint8, device="cuda")
    N.nvfp4_linear_grouped_swiglu_quantize(plan, a.codes, a.scales, a.g, w.codes, w.scales, w.g, 256, 256,
                                           torch.tensor([0.02, 0.0], device="cuda"), codes, scales)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 0


def test_the_same_bits_every_time_and_in_a_graph_on_another_stream(N):
    counts = COUNTS["ragged"]
    plan, a, w, out = check_linear(N, counts, 512, 1024)
    outs = [torch.zeros_like(out) for _ in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        linear(N, plan, a, w, outs[0], 512, 1024, False)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        linear(N, plan, a, w, outs[1], 512, 1024, False)
    linear(N, plan, a, w, outs[2], 512, 1024, False)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    at = torch.as_tensor(a.at, device="cuda")
    for o in outs:
        assert torch.equal(o[at], out[at])


def test_a_plan_beyond_its_buffers_is_cut_to_them(N):
    """Nothing is written past the buffers' rows (guard rows behind them) whatever the plan's numbers are."""
    idx = M.choices([100, 60], 1, 0)
    plan = M.make_plan(N, idx, 2)
    a, w = M.Rows(N, plan, 256, 2), M.Weights(N, 2, 256, 256, 5)
    R = plan.max_rows
    guard = torch.full((R + 512, 256), -7.0, dtype=BF, device="cuda")
    plan.rows.copy_(torch.tensor([100, 5000], dtype=torch.int32))
    linear(N, plan, a, w, guard[:R], 256, 256, False)
    plan.row_start.copy_(torch.tensor([0, R + 128, R + 256], dtype=torch.int32))
    linear(N, plan, a, w, guard[:R], 256, 256, False)
    plan.row_start.copy_(torch.tensor([-128, 64, 128], dtype=torch.int32))
    linear(N, plan, a, w, guard[:R], 256, 256, False)
    torch.cuda.synchronize()
    assert (guard[R:] == -7).all()


@pytest.mark.parametrize("form", ["rows", "nvfp4", "mxfp4", "mxfp4 rotated"])
@pytest.mark.parametrize("counts", [[100, 600], [100, 60] + [0] * 14], ids=["many rows", "few rows"])
def test_a_lost_stage_is_a_timeout_and_the_next_call_is_right(N, form, counts):
    """The injected fault leaves a stage unloaded: the waits run out (2 s), the status says so, the device stays usable."""
    E = len(counts)
    plan = M.make_plan(N, M.choices(counts, 1, 0), E)
    mx = form.startswith("mx")
    a, w = M.Rows(N, plan, 512, 2, mx), M.Weights(N, E, 512, 512, 5, mx)
    out = torch.empty(plan.max_rows, 512, dtype=BF, device="cuda")
    codes = torch.empty(plan.max_rows, 128, dtype=torch.uint8, device="cuda")
    scales = torch.empty(plan.max_rows * 16, dtype=torch.uint8, device="cuda")

    def call():
        if form == "rows":
            linear(N, plan, a, w, out, 512, 512, False)
        elif mx:
            N.mxfp4_linear_grouped_swiglu_quantize(plan, a.codes, a.scales, w.codes, w.scales, 256, 512, codes, scales,
                                                   rotate=form.endswith("rotated"))
        else:
            N.nvfp4_linear_grouped_swiglu_quantize(plan, a.codes, a.scales, a.g, w.codes, w.scales, w.g, 256, 512,
                                                   torch.tensor([0.02], device="cuda"), codes, scales)
    N.nvfp4_debug_inject_fault(N.FAULT_GEMM_SKIP_STAGE)
    call()
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 6
    if form == "rows":
        check_linear(N, counts, 512, 512)
    else:
        check_swiglu(N, counts, 256, 512, mx, form.endswith("rotated"))
