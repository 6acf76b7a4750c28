"""Tokens to their experts' rows and back: the plan by its definition, rows bit for bit, sums and gradients in 64 bits.

Tolerances: half a bf16 step (1 + 2^-6 of it, at a binade's edge and for the rounding to 32 bits before it); a sum of n
products in fp32 besides n 2^-24 of the sum of their magnitudes (n: top_k + 1 terms; for d_weights the at most cols / 8
products of a lane and 10 more additions across lanes and warps, each product exact or fused).
"""
import numpy as np
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


def ok(N):
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 0


def near(got, want, slack):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all()
    over = np.abs(got - want) - M.half_ulp(want) * (1 + 2.0 ** -6) - slack
    assert over.max(initial=-1) <= 0, over.max()


@pytest.mark.parametrize("tokens,top_k,experts,idle", [
    (1, 1, 1, 0.0), (1, 8, 64, 0.0), (1, 32, 1024, 0.0), (3, 2, 2, 0.5), (32, 8, 64, 0.0), (127, 3, 5, 0.1),
    (1024, 4, 1024, 0.0), (1365, 3, 37, 0.2), (512, 8, 256, 0.0), (4099, 8, 64, 0.125), (4097, 1, 1, 0.0),
    (16384, 8, 256, 0.0), (20001, 7, 1000, 0.3), (300000, 4, 64, 0.0), (32769, 1, 340, 0.0), (9000, 1, 365, 0.1),
    (4096, 8, 8, 0.0), (2049, 1, 300, 0.0)])
def test_sort(N, tokens, top_k, experts, idle):
    rng = np.random.default_rng(tokens + top_k)
    p = rng.dirichlet(np.full(experts, 0.3))
    idx = rng.choice(experts, (tokens, top_k), p=p).astype(np.int32)  # an expert may be named twice by a token
    idx[rng.random((tokens, top_k)) < idle] = -1
    idx[rng.random((tokens, top_k)) < idle / 8] = -(1 << 31)
    plan = M.make_plan(N, idx, experts)
    assert int(plan.row_start[-1]) <= plan.max_rows
    again = M.make_plan(N, idx, experts, check=False)
    assert torch.equal(again.row_of, plan.row_of)
    ok(N)


def test_sort_without_tokens_and_without_experts(N):
    plan = N.MoEPlan(0, 4, 9)
    plan.row_start.fill_(7)
    plan.rows.fill_(7)
    N.moe_sort(plan, torch.empty(0, 4, dtype=torch.int32, device="cuda"))
    assert not plan.row_start.any() and not plan.rows.any()
    M.make_plan(N, np.full((5, 3), -1), 4)
    ok(N)


@pytest.mark.parametrize("tokens", [40, 4000])
def test_an_expert_that_is_none_is_reported_and_dropped(N, tokens):
    idx = np.random.default_rng(1).integers(0, 6, (tokens, 2)).astype(np.int32)
    bad = idx.copy()
    bad[7, 1], bad[tokens - 1, 0] = 6, (1 << 31) - 1
    plan = M.make_plan(N, bad, 6, check=False)
    bad[bad >= 6] = -1
    start, rows, row_of = M.plan_of(bad, 6)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 1
    assert np.array_equal(plan.row_of.cpu().numpy(), row_of) and np.array_equal(plan.rows.cpu().numpy(), rows)


def some_plan(N, tokens, top_k=3, experts=7, seed=5):
    idx = np.random.default_rng(seed).integers(-1, experts, (tokens, top_k)).astype(np.int32)
    idx[0] = 2  # the same expert for all of a token's choices
    if tokens > 1:
        idx[1] = -1
    return M.make_plan(N, idx, experts), idx


COLS = [8, 72, 1000, 2048, 2056, 5120, 16392, 65536]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("tokens", [1, 2, 33, 400])
def test_dispatch(N, tokens, cols):
    if tokens == 400 and cols == 65536:
        tokens = 50
    plan, idx = some_plan(N, tokens)
    wide = M.rand_bf16((tokens, cols + 24), 3)
    x = wide[:, 8:8 + cols]
    w = torch.randn(tokens, 3, device="cuda")
    live, _ = M.live_rows(plan)
    between = np.setdiff1d(np.arange(plan.max_rows), live)
    row_of = plan.row_of.cpu().numpy()
    t, j = np.nonzero(row_of >= 0)
    for weights in (None, w):
        rows = torch.full((plan.max_rows, cols), -7.0, dtype=BF, device="cuda")
        N.moe_dispatch(plan, x, rows, weights=weights)
        assert (rows[torch.as_tensor(between, device="cuda")] == -7).all()
        got = rows[torch.as_tensor(row_of[t, j], device="cuda")]
        want = x[torch.as_tensor(t, device="cuda")]
        if weights is None:
            assert torch.equal(got, want)
        else:
            near(got, want.double().cpu().numpy() * w.double().cpu().numpy()[t, j, None], 0)
    ok(N)


@pytest.mark.parametrize("cols", [64, 320, 1536, 4096, 5120])
@pytest.mark.parametrize("tokens", [1, 33, 700])
@pytest.mark.parametrize("form", ["nvfp4", "mxfp4", "mxfp4 rotated"])
def test_quantized_dispatch_is_the_quantizer_of_each_token(N, tokens, cols, form):
    plan, idx = some_plan(N, tokens)
    x = M.rand_bf16((tokens, cols + 8), 3, 4.0)[:, :cols]
    if tokens > 2:
        x[2] = 0
    codes = torch.empty(tokens, cols // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(N.nvfp4_scales_bytes(tokens, cols, N.SCALES_ROWMAJOR), dtype=torch.uint8, device="cuda")
    R = plan.max_rows
    rc = torch.full((R, cols // 2), 0xA5, dtype=torch.uint8, device="cuda")
    rs = torch.full((R * cols // 16,), 0xA5, dtype=torch.uint8, device="cuda")
    g = torch.tensor([0.004], device="cuda")
    if form == "nvfp4":
        N.nvfp4_quantize(x, g, codes, scales, N.SCALES_ROWMAJOR)
        N.moe_dispatch_nvfp4(plan, x, g, rc, rs)
    else:
        rotate = form.endswith("rotated")
        half = torch.empty(tokens, cols // 32, dtype=torch.uint8, device="cuda")
        N.mxfp4_quantize(x, codes, half, N.SCALES_ROWMAJOR, rotate=rotate)
        scales = half.repeat_interleave(2, 1)
        N.moe_dispatch_mxfp4(plan, x, rc, rs, rotate=rotate)
    back = torch.empty(R, cols // 16, dtype=torch.uint8, device="cuda")
    N.nvfp4_scales_relayout(rs, back, R, cols, N.SCALES_MMA, N.SCALES_ROWMAJOR)
    row_of = plan.row_of.cpu().numpy()
    t, j = np.nonzero(row_of >= 0)
    at, t = torch.as_tensor(row_of[t, j], device="cuda"), torch.as_tensor(t, device="cuda")
    assert torch.equal(rc[at], codes[t]) and torch.equal(back[at], scales.view(tokens, -1)[t])
    rest = torch.ones(R, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert (rc[rest] == 0xA5).all() and (back[rest] == 0xA5).all()
    ok(N)


@pytest.mark.parametrize("g", [0.0, -1.0, float("nan"), float("inf")])
def test_an_invalid_scale_gives_zeros_and_is_reported(N, g):
    plan, _ = some_plan(N, 20)
    r = torch.full((plan.max_rows, 32), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((plan.max_rows * 4,), 0xA5, dtype=torch.uint8, device="cuda")
    N.moe_dispatch_nvfp4(plan, M.rand_bf16((20, 64), 1), torch.tensor([g], device="cuda"), r, s)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 1
    at, _ = M.live_rows(plan)
    assert not r[torch.as_tensor(at, device="cuda")].any()


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("tokens", [1, 2, 33, 400])
@pytest.mark.parametrize("weighted,based", [(True, 0), (False, 0), (True, 1), (True, 2)])
def test_combine(N, tokens, cols, weighted, based):
    if tokens == 400 and cols == 65536:
        tokens = 50
    plan, idx = some_plan(N, tokens)
    live, _ = M.live_rows(plan)
    y = torch.full((plan.max_rows, cols), float("nan"), dtype=BF, device="cuda")  # unused rows enter nothing
    y[torch.as_tensor(live, device="cuda")] = M.rand_bf16((len(live), cols), 4)
    w = torch.randn(tokens, 3, device="cuda")
    w[plan.row_of < 0] = float("nan")  # nor do the weights of choices without an expert
    out = torch.full((tokens, cols + 16), 9.0, dtype=BF, device="cuda")
    base = M.rand_bf16((tokens, cols + 16), 6) if based else None
    if based == 2:
        out = base.clone()
    o, b = out[:, :cols], None if not based else (out if based == 2 else base)[:, :cols]
    add = np.zeros((tokens, cols)) if not based else b.double().cpu().numpy()
    N.moe_combine(plan, y, o, weights=w if weighted else None, base=b)
    row_of, yy, ww = plan.row_of.cpu().numpy(), y.double().cpu().numpy(), w.double().cpu().numpy()
    want, mag = add.copy(), np.abs(add)
    for j in range(3):
        has = row_of[:, j] >= 0
        term = yy[row_of[has, j]] * (ww[has, j, None] if weighted else 1.0)
        want[has] += term
        mag[has] += np.abs(term)
    near(o, want, 4 * 2.0 ** -24 * mag)
    assert torch.equal(out[:, cols:], (base if based == 2 else torch.full_like(out, 9.0))[:, cols:])
    ok(N)


@pytest.mark.parametrize("cols", [64, 2048, 4104, 16384])
@pytest.mark.parametrize("tokens", [1, 150, 701])
@pytest.mark.parametrize("top_k", [1, 2, 4, 9, 32])
def test_combine_of_any_number_of_choices(N, top_k, tokens, cols):
    """A token's sum has top_k fused steps: at most that many roundings of at most the sum of magnitudes."""
    plan, _ = some_plan(N, tokens, top_k=top_k, experts=33)
    y, w = M.rand_bf16((plan.max_rows, cols), 8), torch.randn(tokens, top_k, device="cuda")
    out = torch.full((tokens, cols), 9.0, dtype=BF, device="cuda")
    N.moe_combine(plan, y, out, weights=w)
    want = torch.zeros(tokens, cols, dtype=torch.float64, device="cuda")
    mag = want.clone()
    for j in range(top_k):
        has = (plan.row_of[:, j] >= 0).nonzero()[:, 0]
        term = y[plan.row_of[has, j].long()].double() * w[has, j, None].double()
        want[has] += term
        mag[has] += term.abs()
    near(out, want.cpu().numpy(), top_k * 2.0 ** -24 * mag.cpu().numpy())
    ok(N)


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("tokens,top_k", [(1, 3), (2, 1), (33, 8), (400, 5), (3, 32), (900, 2), (701, 5)])
def test_combine_backward(N, tokens, top_k, cols):
    if tokens > 100 and cols == 65536:
        tokens = 40
    plan, idx = some_plan(N, tokens, top_k, 40 if top_k == 32 else 9)
    live, _ = M.live_rows(plan)
    at = torch.as_tensor(live, device="cuda")
    y = torch.full((plan.max_rows, cols), float("nan"), dtype=BF, device="cuda")
    y[at] = M.rand_bf16((len(live), cols), 4)
    g = M.rand_bf16((tokens, cols + 8), 6)[:, 8:]
    w = torch.randn(tokens, top_k, device="cuda")
    d_y = torch.full((plan.max_rows, cols), -7.0, dtype=BF, device="cuda")
    d_w = torch.full((tokens, top_k), float("nan"), device="cuda")
    N.moe_combine_backward(plan, g, y, w, d_y, d_w)
    row_of = plan.row_of.cpu().numpy()
    gg, yy, ww = g.double().cpu().numpy(), y.double().cpu().numpy(), w.double().cpu().numpy()
    t, j = np.nonzero(row_of >= 0)
    r = row_of[t, j]
    near(d_y[torch.as_tensor(r, device="cuda")], ww[t, j, None] * gg[t], 0)
    rest = torch.ones(plan.max_rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert (d_y[rest] == -7).all()
    want, mag = np.zeros((tokens, top_k)), np.zeros((tokens, top_k))
    want[t, j] = (gg[t] * yy[r]).sum(1)
    mag[t, j] = np.abs(gg[t] * yy[r]).sum(1)
    over = np.abs(d_w.double().cpu().numpy() - want) - (cols / 8 + 10) * 2.0 ** -24 * mag
    assert over.max() <= 0
    # Either output alone, the same bits.
    d_y2, d_w2 = torch.empty_like(d_y), torch.empty_like(d_w)
    N.moe_combine_backward(plan, g, y, w, d_y2, None)
    N.moe_combine_backward(plan, g, y, w, None, d_w2)
    assert torch.equal(d_y2[at], d_y[at]) and torch.equal(d_w2, d_w)
    ok(N)


def test_gradients_are_those_of_differences(N):
    """dL/dx and dL/dw of L = <c, combine(dispatch(x), w)> in small integers and powers of two: exact in bf16 and fp32, so
    that a difference of the calls themselves is the gradient."""
    tokens, cols, k = 5, 16, 3
    plan, idx = some_plan(N, tokens, k)
    gen = torch.Generator(device="cuda").manual_seed(2)

    def ints(*shape):
        return torch.randint(-2, 3, shape, generator=gen, device="cuda").float()
    x, c, w = ints(tokens, cols).to(BF), ints(tokens, cols).to(BF), ints(tokens, k)

    def forward(x, w):
        rows = torch.zeros(plan.max_rows, cols, dtype=BF, device="cuda")
        N.moe_dispatch(plan, x, rows)
        out = torch.empty_like(x)
        N.moe_combine(plan, rows, out, weights=w)
        return rows, (out.double() * c.double()).sum().item()
    rows, at = forward(x, w)
    d_y, d_w, d_x = torch.zeros_like(rows), torch.empty_like(w), torch.empty_like(x)
    N.moe_combine_backward(plan, c, rows, w, d_y, d_w)
    N.moe_combine(plan, d_y, d_x)
    for t in range(tokens):
        for j in range(k):
            moved = w.clone()
            moved[t, j] += 1
            assert forward(x, moved)[1] - at == d_w[t, j].item()
        for i in range(0, cols, 5):
            moved = x.clone()
            moved[t, i] += 1
            assert forward(moved, w)[1] - at == d_x[t, i].item()
    ok(N)


def test_calls_without_tokens_do_nothing(N):
    plan = N.MoEPlan(0, 2, 4)
    none = torch.empty(0, 64, dtype=BF, device="cuda")
    u8 = torch.empty(0, dtype=torch.uint8, device="cuda")
    w = torch.empty(0, 2, device="cuda")
    before = N.nvfp4_launch_count()
    N.moe_dispatch(plan, none, none)
    N.moe_dispatch_nvfp4(plan, none, torch.ones(1, device="cuda"), u8, u8)
    N.moe_dispatch_mxfp4(plan, none, u8, u8)
    N.moe_combine(plan, none, none, weights=w)
    N.moe_combine_backward(plan, none, none, w, none, w)
    assert N.nvfp4_launch_count() == before


def test_rows_past_2_to_the_31_elements(N):
    """The last rows of buffers with more than 2^31 elements."""
    cols, tokens = 65536, 33000
    idx = np.full((tokens, 1), -1, np.int32)
    idx[:200, 0], idx[-3:, 0] = 0, 1
    idx[200:32900, 0] = 0
    plan = M.make_plan(N, idx, 2)
    x = torch.empty(tokens, cols, dtype=BF, device="cuda")
    x.copy_(torch.arange(tokens, device="cuda").remainder(251).to(BF)[:, None].expand(-1, cols))
    rows = torch.zeros(plan.max_rows, cols, dtype=BF, device="cuda")
    N.moe_dispatch(plan, x, rows)
    last = int(plan.row_of[-1, 0])
    assert last * cols > 1 << 31 and torch.equal(rows[last], x[-1]) and torch.equal(rows[32899], x[32899])
    out = torch.empty_like(x)
    N.moe_combine(plan, rows, out)
    assert torch.equal(out[-1], x[-1]) and not out[32900:32990].any() and torch.equal(out[32899], x[32899])
    ok(N)
