"""A layer of bf16 experts, forward and backward through the library's calls (the experts' own products are torch's), against
the same layer in 64 bits with the library's choice of experts; and the calls beside each other on streams and in graphs.

Tolerance: every bf16 tensor that passes between two calls is rounded (2^-9 relative, half a step), and there are at most
six in a path: 6 * 2^-9 of the gradient's norm, and twice that for what the products of rounded tensors add.
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


class Layer:
    """logits = x Wr; out = base + sum_j w_j silu(x A_e) B_e."""

    def __init__(self, N, tokens, hidden, inner, experts, top_k, score, renormalize, seed=0):
        self.N, self.kw = N, dict(score=N.MOE_SIGMOID if score == "sigmoid" else N.MOE_SOFTMAX, renormalize=renormalize)
        self.x, self.base = M.rand_bf16((tokens, hidden), seed + 1), M.rand_bf16((tokens, hidden), seed + 2)
        self.Wr = M.rand_bf16((hidden, experts), seed + 3, 2 / np.sqrt(hidden))
        self.A = M.rand_bf16((experts, hidden, inner), seed + 4, 1 / np.sqrt(hidden))
        self.B = M.rand_bf16((experts, inner, hidden), seed + 5, 1 / np.sqrt(inner))
        self.plan = N.MoEPlan(tokens, top_k, experts)
        self.idx = torch.empty(tokens, top_k, dtype=torch.int32, device="cuda")
        self.w = torch.empty(tokens, top_k, device="cuda")
        R = self.plan.max_rows
        self.rows, self.y, self.d_y, self.d_rows = (torch.zeros(R, hidden, dtype=BF, device="cuda") for _ in range(4))
        self.d_w = torch.empty_like(self.w)
        self.out, self.d_x = torch.empty_like(self.x), torch.empty_like(self.x)
        self.logits = self.x @ self.Wr
        self.d_logits = torch.empty_like(self.logits)

    def spans(self):
        return [(e, s, s + n) for e, (s, n) in enumerate(zip(self.plan.row_start.tolist(), self.plan.rows.tolist())) if n]

    def forward(self):
        N = self.N
        N.moe_route(self.logits, self.idx, self.w, **self.kw)
        N.moe_sort(self.plan, self.idx)
        N.moe_dispatch(self.plan, self.x, self.rows)
        for e, a, b in self.spans():
            z = (self.rows[a:b] @ self.A[e]).float()
            self.y[a:b] = (z * torch.sigmoid(z)).to(BF) @ self.B[e]
        N.moe_combine(self.plan, self.y, self.out, weights=self.w, base=self.base)

    def backward(self, g):
        N = self.N
        N.moe_combine_backward(self.plan, g, self.y, self.w, self.d_y, self.d_w)
        self.d_A, self.d_B = torch.zeros_like(self.A), torch.zeros_like(self.B)
        for e, a, b in self.spans():
            z = (self.rows[a:b] @ self.A[e]).float()
            s = torch.sigmoid(z)
            self.d_B[e] = (z * s).to(BF).T @ self.d_y[a:b]
            d_z = ((self.d_y[a:b] @ self.B[e].T).float() * (s + z * s * (1 - s))).to(BF)
            self.d_A[e] = self.rows[a:b].T @ d_z
            self.d_rows[a:b] = d_z @ self.A[e].T
        N.moe_combine(self.plan, self.d_rows, self.d_x)
        N.moe_route_backward(self.logits, self.idx, self.d_w, self.d_logits, **self.kw)

    def exact(self, g):
        """The same in 64 bits by autograd, with the chosen experts."""
        leaves = [t.double().requires_grad_() for t in (self.x, self.logits, self.A, self.B)]
        x, l, A, B = leaves
        p = torch.sigmoid(l) if self.kw["score"] else torch.softmax(l, 1)
        w = p.gather(1, self.idx.long())
        if self.kw["renormalize"]:
            w = w / w.sum(1, keepdim=True)
        i = self.idx.long()
        out = self.base.double()
        for j in range(i.shape[1]):
            z = torch.einsum("th,thi->ti", x, A[i[:, j]])
            out = out + w[:, j, None] * torch.einsum("ti,tih->th", z * torch.sigmoid(z), B[i[:, j]])
        out.backward(g.double())
        return out.detach(), [t.grad for t in leaves]


@pytest.mark.parametrize("tokens,hidden,inner,experts,top_k", [(1, 64, 32, 8, 2), (7, 128, 64, 4, 4), (150, 256, 64, 16, 3),
                                                               (400, 64, 128, 5, 1)])
@pytest.mark.parametrize("score,renormalize", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_forward_and_backward(N, tokens, hidden, inner, experts, top_k, score, renormalize):
    layer = Layer(N, tokens, hidden, inner, experts, top_k, score, renormalize)
    g = M.rand_bf16((tokens, hidden), 77)
    layer.forward()
    layer.backward(g)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 0
    out, (d_x, d_l, d_A, d_B) = layer.exact(g)
    degenerate = top_k == 1 and renormalize  # the one weight is 1 whatever the logits are
    for name, got, want in (("out", layer.out, out), ("d_x", layer.d_x, d_x), ("d_A", layer.d_A, d_A),
                            ("d_B", layer.d_B, d_B), ("d_logits", layer.d_logits, d_l)):
        if name == "d_logits" and degenerate:
            assert got.abs().max() <= 2.0 ** -20 * layer.d_w.abs().max()
            continue
        err = ((got.double() - want).norm() / want.norm()).item()
        assert err <= 12 * 2.0 ** -9, f"{name}: {err}"


def test_two_layers_at_once_and_replayed(N):
    """Two layers' calls on two streams, and both captured into one graph with parallel branches: the bits of each alone.
    Plans and workspaces are the layers' own."""
    layers = [Layer(N, 600, 512, 64, 32, 4, "softmax", True, seed=s) for s in (0, 50)]
    alone = []
    for layer in layers:
        layer.forward()
        alone.append([t.clone() for t in (layer.out, layer.idx, layer.plan.row_of)])

    def calls(layer):  # without the products, which need the host
        N.moe_route(layer.logits, layer.idx, layer.w, **layer.kw)
        N.moe_sort(layer.plan, layer.idx)
        N.moe_dispatch(layer.plan, layer.x, layer.rows)
        N.moe_combine(layer.plan, layer.y, layer.out, weights=layer.w, base=layer.base)

    def clear():
        for layer in layers:
            layer.out.zero_()
            layer.idx.fill_(-9)
            layer.plan.row_of.fill_(-9)
        torch.cuda.synchronize()

    def check():
        torch.cuda.synchronize()
        for layer, want in zip(layers, alone):
            assert all(torch.equal(a, b) for a, b in zip((layer.out, layer.idx, layer.plan.row_of), want))
    streams = [torch.cuda.Stream() for _ in layers]
    clear()
    for _ in range(5):
        for layer, s in zip(layers, streams):
            with torch.cuda.stream(s):
                calls(layer)
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        for layer, s in zip(layers, streams):
            s.wait_stream(main)
            with torch.cuda.stream(s):
                calls(layer)
            main.wait_stream(s)
    clear()
    for _ in range(3):
        graph.replay()
    check()
    assert N.nvfp4_get_device_status() == 0


def test_the_backward_pass_from_a_graph(N):
    layer = Layer(N, 300, 256, 64, 16, 2, "sigmoid", True)
    g = M.rand_bf16((300, 256), 5)
    layer.forward()
    layer.backward(g)
    want = [t.clone() for t in (layer.d_x, layer.d_w, layer.d_logits)]

    def calls():
        N.moe_combine_backward(layer.plan, g, layer.y, layer.w, layer.d_y, layer.d_w)
        N.moe_combine(layer.plan, layer.d_rows, layer.d_x)
        N.moe_route_backward(layer.logits, layer.idx, layer.d_w, layer.d_logits, **layer.kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for t in (layer.d_x, layer.d_w, layer.d_logits):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip((layer.d_x, layer.d_w, layer.d_logits), want):
        assert torch.equal(a, b)
