"""Host-only checks of the mixture-of-experts calls: what they refuse before anything is launched.  No call here reaches a
GPU."""
import ctypes
import itertools

import pytest
import torch

from _util import lib

OK_PTR = 0x10000  # aligned, never dereferenced: validation fails first
INVALID, SHAPE, ALIGN = 1, 2, 3
FAR = 1 << 40


@pytest.fixture(scope="module")
def N():
    return lib()


def ptr(v=OK_PTR):
    return None if v is None else ctypes.c_void_p(v)


def plan(N, **kw):
    p = dict(row_start=OK_PTR, rows=OK_PTR, row_of=OK_PTR, n_tokens=4, top_k=2, num_experts=8)
    p.update(kw)
    return N.MoEPlanStruct(**p)


def call(N, name, p=None, **kw):
    """One call with good arguments but those given."""
    a = dict(x=OK_PTR, ld=256, cols=256, weights=OK_PTR, rows=OK_PTR, g=OK_PTR, codes=OK_PTR, scales=OK_PTR, rotate=0,
             base=OK_PTR, ld_base=256, out=OK_PTR, ld_out=256, d_y=OK_PTR, d_w=OK_PTR, idx=OK_PTR, ws=OK_PTR, ws_bytes=FAR,
             a_codes=OK_PTR, a_scales=OK_PTR, g_a=OK_PTR, a_step=0, w_codes=OK_PTR, w_scales=OK_PTR, g_w=OK_PTR, n=256,
             k=512, inner=256, g_out=OK_PTR, out_step=1, logits=OK_PTR, type=0, tokens=4, experts=8, top_k=2, score=0,
             renormalize=1, scale=1.0, bias=None, options=True)
    a.update(kw)
    P = {n: ptr(a[n]) for n in a if n in ("x", "weights", "rows", "g", "codes", "scales", "base", "out", "d_y", "d_w", "idx",
                                          "ws", "a_codes", "a_scales", "g_a", "w_codes", "w_scales", "g_w", "g_out",
                                          "logits")}
    pl = None if p is False else ctypes.byref(plan(N) if p is None else p)
    o = ctypes.byref(N.MoERouteOptionsStruct(a["score"], a["renormalize"], a["scale"], a["bias"])) if a["options"] else None
    s, L = ctypes.c_void_p(0), N._lib
    operands = (P["a_codes"], P["a_scales"])
    w = (P["w_codes"], P["w_scales"])
    if name == "moe_sort":
        return L.moe_sort(pl, P["idx"], P["ws"], a["ws_bytes"], s)
    if name == "moe_dispatch":
        return L.moe_dispatch(pl, P["x"], a["ld"], a["cols"], P["weights"], P["rows"], s)
    if name == "moe_dispatch_nvfp4":
        return L.moe_dispatch_nvfp4(pl, P["x"], a["ld"], a["cols"], P["g"], P["codes"], P["scales"], s)
    if name == "moe_dispatch_mxfp4":
        return L.moe_dispatch_mxfp4(pl, P["x"], a["ld"], a["cols"], a["rotate"], P["codes"], P["scales"], s)
    if name == "moe_combine":
        return L.moe_combine(pl, P["x"], a["cols"], P["weights"], P["base"], a["ld_base"], P["out"], a["ld_out"], s)
    if name == "moe_combine_backward":
        return L.moe_combine_backward(pl, P["out"], a["ld_out"], P["x"], a["cols"], P["weights"], P["d_y"], P["d_w"], s)
    if name == "nvfp4_linear_grouped":
        return L.nvfp4_linear_grouped(pl, *operands, P["g_a"], a["a_step"], *w, P["g_w"], a["n"], a["k"], P["out"],
                                      a["ld_out"], s)
    if name == "mxfp4_linear_grouped":
        return L.mxfp4_linear_grouped(pl, *operands, *w, a["n"], a["k"], P["out"], a["ld_out"], s)
    if name == "nvfp4_linear_grouped_swiglu_quantize":
        return L.nvfp4_linear_grouped_swiglu_quantize(pl, *operands, P["g_a"], a["a_step"], *w, P["g_w"], a["inner"], a["k"],
                                                      P["g_out"], a["out_step"], P["codes"], P["scales"], s)
    if name == "mxfp4_linear_grouped_swiglu_quantize":
        return L.mxfp4_linear_grouped_swiglu_quantize(pl, *operands, *w, a["inner"], a["k"], a["rotate"], P["codes"],
                                                      P["scales"], s)
    route = (P["logits"], a["type"], a["ld"], a["tokens"], a["experts"], a["top_k"], o, P["idx"], P["weights"])
    return L.moe_route(*route, s) if name == "moe_route" else L.moe_route_backward(*route, P["out"], s)


ROWS = ["moe_sort", "moe_dispatch", "moe_dispatch_nvfp4", "moe_dispatch_mxfp4", "moe_combine", "moe_combine_backward"]
LINEARS = ["nvfp4_linear_grouped", "mxfp4_linear_grouped", "nvfp4_linear_grouped_swiglu_quantize",
           "mxfp4_linear_grouped_swiglu_quantize"]
ROUTES = ["moe_route", "moe_route_backward"]

BAD_PLANS = [(dict(row_start=None), INVALID), (dict(rows=None), INVALID), (dict(row_of=None), INVALID),
             (dict(n_tokens=-1), SHAPE), (dict(top_k=0), SHAPE), (dict(top_k=33), SHAPE), (dict(num_experts=0), SHAPE),
             (dict(num_experts=1025), SHAPE), (dict(n_tokens=1 << 30), SHAPE), (dict(n_tokens=1 << 62), SHAPE),
             (dict(row_start=OK_PTR + 2), ALIGN), (dict(rows=OK_PTR + 1), ALIGN), (dict(row_of=OK_PTR + 2), ALIGN)]


@pytest.mark.parametrize("name", ROWS + LINEARS)
def test_the_plan_is_checked_by_every_call(N, name):
    before = N.nvfp4_launch_count()
    assert call(N, name, p=False) == INVALID
    for kw, code in BAD_PLANS:
        assert call(N, name, p=plan(N, **kw)) == code, kw
    assert N.nvfp4_launch_count() == before


TOKENS = [(dict(cols=0), SHAPE), (dict(cols=-8), SHAPE), (dict(cols=65536 + 64, ld=1 << 20, ld_out=1 << 20, ld_base=1 << 20), SHAPE)]
REFUSALS = {
    "moe_sort": [(dict(idx=None), INVALID), (dict(idx=OK_PTR + 2), ALIGN)],
    "moe_dispatch": TOKENS + [(dict(cols=252), SHAPE), (dict(ld=248), SHAPE), (dict(ld=260), ALIGN), (dict(x=None), INVALID),
                              (dict(rows=None), INVALID), (dict(x=OK_PTR + 8), ALIGN), (dict(rows=OK_PTR + 8), ALIGN),
                              (dict(weights=OK_PTR + 2), ALIGN)],
    "moe_dispatch_nvfp4": TOKENS + [(dict(cols=224), SHAPE), (dict(ld=192), SHAPE), (dict(g=None), INVALID),
                                    (dict(codes=None), INVALID), (dict(scales=None), INVALID), (dict(x=None), INVALID),
                                    (dict(codes=OK_PTR + 8), ALIGN), (dict(scales=OK_PTR + 2), ALIGN),
                                    (dict(g=OK_PTR + 2), ALIGN), (dict(ld=260), ALIGN)],
    "moe_dispatch_mxfp4": TOKENS + [(dict(cols=224), SHAPE), (dict(rotate=2), INVALID), (dict(rotate=-1), INVALID),
                                    (dict(codes=None), INVALID), (dict(codes=OK_PTR + 8), ALIGN),
                                    (dict(scales=OK_PTR + 1), ALIGN)],
    "moe_combine": TOKENS + [(dict(cols=252), SHAPE), (dict(ld_out=248), SHAPE), (dict(ld_base=248), SHAPE),
                             (dict(ld_out=260), ALIGN), (dict(ld_base=260), ALIGN), (dict(x=None), INVALID),
                             (dict(out=None), INVALID), (dict(x=OK_PTR + 8), ALIGN), (dict(out=OK_PTR + 8), ALIGN),
                             (dict(base=OK_PTR + 8), ALIGN), (dict(weights=OK_PTR + 1), ALIGN)],
    "moe_combine_backward": TOKENS + [(dict(cols=252), SHAPE), (dict(ld_out=248), SHAPE), (dict(ld_out=260), ALIGN),
                                      (dict(out=None), INVALID), (dict(x=None), INVALID), (dict(weights=None), INVALID),
                                      (dict(d_y=None, d_w=None), INVALID), (dict(d_y=OK_PTR + 8), ALIGN),
                                      (dict(d_w=OK_PTR + 2), ALIGN)],
}
_LINEAR = [(dict(a_codes=None), INVALID), (dict(a_scales=None), INVALID), (dict(w_codes=None), INVALID),
           (dict(w_scales=None), INVALID), (dict(k=0), SHAPE), (dict(k=384), SHAPE), (dict(k=1 << 21), SHAPE),
           (dict(a_codes=OK_PTR + 8), ALIGN), (dict(a_scales=OK_PTR + 4), ALIGN), (dict(w_codes=OK_PTR + 8), ALIGN),
           (dict(w_scales=OK_PTR + 4), ALIGN)]
_G = [(dict(g_a=None), INVALID), (dict(g_w=None), INVALID), (dict(a_step=2), INVALID), (dict(a_step=-1), INVALID),
      (dict(g_a=OK_PTR + 2), ALIGN), (dict(g_w=OK_PTR + 1), ALIGN)]
_PLAIN = [(dict(n=0), SHAPE), (dict(n=250), SHAPE), (dict(n=1 << 21), SHAPE), (dict(ld_out=248), SHAPE),
          (dict(ld_out=260), SHAPE), (dict(out=None), INVALID), (dict(out=OK_PTR + 8), ALIGN)]
_FUSED = [(dict(inner=0), SHAPE), (dict(inner=192), SHAPE), (dict(codes=None), INVALID), (dict(scales=None), INVALID),
          (dict(codes=OK_PTR + 8), ALIGN), (dict(scales=OK_PTR + 2), ALIGN)]
REFUSALS["nvfp4_linear_grouped"] = _LINEAR + _G + _PLAIN
REFUSALS["mxfp4_linear_grouped"] = _LINEAR + _PLAIN
REFUSALS["nvfp4_linear_grouped_swiglu_quantize"] = _LINEAR + _G + _FUSED + [
    (dict(g_out=None), INVALID), (dict(out_step=2), INVALID), (dict(g_out=OK_PTR + 2), ALIGN)]
REFUSALS["mxfp4_linear_grouped_swiglu_quantize"] = _LINEAR + _FUSED + [(dict(rotate=2), INVALID)]
_ROUTE = [(dict(options=False), INVALID), (dict(type=2), INVALID), (dict(type=-1), INVALID), (dict(score=2), INVALID),
          (dict(renormalize=2), INVALID), (dict(bias=OK_PTR), INVALID), (dict(scale=float("inf")), INVALID),
          (dict(scale=float("nan")), INVALID), (dict(score=1, bias=OK_PTR + 2), ALIGN), (dict(tokens=-1), SHAPE),
          (dict(experts=0), SHAPE), (dict(experts=1025, ld=2000), SHAPE), (dict(top_k=0), SHAPE),
          (dict(top_k=9), SHAPE), (dict(ld=7), SHAPE), (dict(tokens=1 << 40), SHAPE), (dict(logits=None), INVALID),
          (dict(idx=None), INVALID), (dict(weights=None), INVALID), (dict(logits=OK_PTR + 2), ALIGN),
          (dict(logits=OK_PTR + 1, type=1), ALIGN), (dict(idx=OK_PTR + 2), ALIGN), (dict(weights=OK_PTR + 2), ALIGN)]
REFUSALS["moe_route"] = _ROUTE
REFUSALS["moe_route_backward"] = _ROUTE + [(dict(out=None), INVALID), (dict(out=OK_PTR + 2), ALIGN)]


@pytest.mark.parametrize("name,kw,code", [(n, kw, c) for n, many in REFUSALS.items() for kw, c in many])
def test_refusals(N, name, kw, code):
    before = N.nvfp4_launch_count()
    assert call(N, name, **kw) == code
    assert N.nvfp4_launch_count() == before


@pytest.mark.parametrize("name", ROWS[1:] + LINEARS)
def test_no_tokens_is_nothing(N, name):
    before = N.nvfp4_launch_count()
    assert call(N, name, p=plan(N, n_tokens=0, row_of=None), x=None, out=OK_PTR, weights=OK_PTR) == 0
    assert N.nvfp4_launch_count() == before


@pytest.mark.parametrize("name", ROUTES)
def test_no_tokens_to_route_is_nothing(N, name):
    assert call(N, name, tokens=0, logits=None, idx=None, weights=None) == 0


def test_a_sort_of_many_choices_needs_its_workspace(N):
    p = plan(N, n_tokens=100000)
    need = N.moe_sort_workspace_size(100000, 2, 8)
    assert need > 0 and N.moe_sort_workspace_size(4, 2, 8) == 0
    assert call(N, "moe_sort", p=p, ws=None) == INVALID
    assert call(N, "moe_sort", p=p, ws_bytes=need - 1) == SHAPE
    assert call(N, "moe_sort", p=p, ws=OK_PTR + 8) == ALIGN


def test_sizes_that_the_buffers_do_not_address(N):
    """num_experts * ceil(N / 128) * (K / 32) and num_experts * N reach 2^31."""
    p = plan(N, num_experts=1024)
    big = 1 << 20
    assert call(N, "nvfp4_linear_grouped", p=p, n=big, k=8192, ld_out=big) == SHAPE
    assert call(N, "mxfp4_linear_grouped", p=plan(N, num_experts=1024), n=65536, k=big, ld_out=65536) == SHAPE
    assert call(N, "nvfp4_linear_grouped_swiglu_quantize", p=p, inner=big, k=256) == SHAPE


def test_max_rows(N):
    for tokens, k, experts in itertools.product([0, 1, 2, 7, 128, 1000], [1, 3, 8], [1, 2, 8, 100]):
        n = tokens * k
        # The worst plan: each expert that can have a row has one past a tile.
        worst, left = 0, n
        for _ in range(min(experts, n)):
            left -= 1
            worst += 128
        worst += left // 128 * 128
        got = N.moe_max_rows(tokens, k, experts)
        assert got % 128 == 0 and worst <= got <= n + 127 * min(experts, n)
    assert N.moe_max_rows(-1, 1, 1) == 0 and N.moe_max_rows(1, 33, 64) == 0 and N.moe_max_rows(1 << 31, 1, 1) == 0
    assert N.moe_sort_workspace_size(1, 0, 1) == 0


class TestBinding:
    """The Python binding's own checks: shapes, types and sizes of its tensors (on the CPU: nothing is launched)."""

    def made(self, N):
        return N.MoEPlan(6, 2, 4, device="cpu")

    def test_plan(self, N):
        for bad in ((4, 0, 3), (4, 33, 64), (4, 2, 0), (4, 2, 1025), (-1, 2, 3)):
            with pytest.raises(ValueError):
                N.MoEPlan(*bad, device="cpu")
        assert N.MoEPlan(0, 2, 4, device="cpu").max_rows == 0

    @pytest.mark.parametrize("kw", [dict(x=(5, 64)), dict(x=(6, 64), rows=(6, 64)), dict(w=(6, 3)),
                                    dict(xt=torch.float32), dict(rt=torch.float16), dict(wt=torch.float64)])
    def test_dispatch(self, N, kw):
        p = self.made(N)
        x = torch.zeros(kw.get("x", (6, 64)), dtype=kw.get("xt", torch.bfloat16))
        rows = torch.zeros(kw.get("rows", (p.max_rows, 64)), dtype=kw.get("rt", torch.bfloat16))
        w = torch.zeros(kw.get("w", (6, 2)), dtype=kw.get("wt", torch.float32))
        with pytest.raises(ValueError):
            N.moe_dispatch(p, x, rows, weights=w)
        with pytest.raises(ValueError):
            N.moe_combine(p, rows, x, weights=w)
        with pytest.raises(ValueError):
            N.moe_combine_backward(p, x, rows, w, None, torch.zeros(6, 2))

    def test_quantized_rows(self, N):
        p = self.made(N)
        x, g = torch.zeros(6, 64, dtype=torch.bfloat16), torch.ones(1)
        codes, scales = torch.zeros(p.max_rows, 32, dtype=torch.uint8), torch.zeros(p.max_rows * 4, dtype=torch.uint8)
        for c, s in ((codes[:-1], scales), (codes, scales[:-1]), (codes.int(), scales), (codes[:, ::2], scales)):
            with pytest.raises(ValueError):
                N.moe_dispatch_nvfp4(p, x, g, c, s)
            with pytest.raises(ValueError):
                N.moe_dispatch_mxfp4(p, x, c, s)
        with pytest.raises(ValueError):
            N.moe_dispatch_nvfp4(p, x, torch.ones(2), codes, scales)

    def test_linears(self, N):
        p, n, k = self.made(N), 256, 256
        a = (torch.zeros(p.max_rows, k // 2, dtype=torch.uint8), torch.zeros(p.max_rows * k // 16, dtype=torch.uint8))
        w = (torch.zeros(4, n, k // 2, dtype=torch.uint8), torch.zeros(4 * n * k // 16, dtype=torch.uint8))
        g, gw, out = torch.ones(1), torch.ones(4), torch.zeros(p.max_rows, n, dtype=torch.bfloat16)
        for bad in (dict(w=(w[0][:3], w[1])), dict(w=(w[0], w[1][:-1])), dict(a=(a[0][:-1], a[1])), dict(g=torch.ones(3)),
                    dict(gw=torch.ones(1)), dict(out=out[:-1]), dict(out=out.float()), dict(out=out[:, :128])):
            aa, ww, o = bad.get("a", a), bad.get("w", w), bad.get("out", out)
            with pytest.raises(ValueError):
                N.nvfp4_linear_grouped(p, *aa, bad.get("g", g), *ww, bad.get("gw", gw), o, n, k)
        h = (torch.zeros(p.max_rows, 64, dtype=torch.uint8), torch.zeros(p.max_rows * 8, dtype=torch.uint8))
        with pytest.raises(ValueError):
            N.nvfp4_linear_grouped_swiglu_quantize(p, *a, g, *w, gw, 128, k, torch.ones(2), *h)
        with pytest.raises(ValueError):
            N.mxfp4_linear_grouped_swiglu_quantize(p, *a, *w, 128, k, h[0], h[1][:-1])

    def test_route(self, N):
        l, idx, w = torch.zeros(6, 8), torch.zeros(6, 2, dtype=torch.int32), torch.zeros(6, 2)
        for bad in (dict(l=l.half()), dict(idx=idx.long()), dict(idx=idx[:5]), dict(w=w.double()), dict(w=w[:, :1]),
                    dict(l=l.t()), dict(bias=torch.zeros(7)), dict(bias=torch.zeros(8).half())):
            with pytest.raises(ValueError):
                N.moe_route(bad.get("l", l), bad.get("idx", idx), bad.get("w", w), score=N.MOE_SIGMOID, bias=bad.get("bias"))
        for bad in (dict(d=torch.zeros(6, 8).half()), dict(d=torch.zeros(6, 7)), dict(w=w[:5])):
            with pytest.raises(ValueError):
                N.moe_route_backward(l, idx, bad.get("w", w), bad.get("d", torch.zeros(6, 8)))
