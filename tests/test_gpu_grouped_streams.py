"""The experts' linears beside other kernels with tensor memory: two layers' products on two streams at once, with the dense
linears between them, and all of it in one graph with parallel branches.  The bits of each alone."""
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


class Products:
    """gate_up and down of a plan in both formats, and a dense linear: random codes, block scales of 1."""

    def __init__(self, N, counts, hidden, inner, seed):
        E = len(counts)
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def codes(*shape):
            return torch.randint(0, 256, shape, generator=gen, device="cuda", dtype=torch.uint8)

        def ones(n, mx):
            return torch.full((n // 16,), 127 if mx else 0x38, dtype=torch.uint8, device="cuda")
        self.N, self.hidden, self.inner = N, hidden, inner
        self.plan = M.make_plan(N, M.choices(counts, 2, seed), E)
        R = self.plan.max_rows
        self.a = codes(R, hidden // 2), [ones(R * hidden, mx) for mx in (False, True)]
        self.up = codes(E, 2 * inner, hidden // 2), [ones(E * 2 * inner * hidden, mx) for mx in (False, True)]
        self.down = codes(E, hidden, inner // 2), [ones(E * hidden * inner, mx) for mx in (False, True)]
        self.g, self.g_w = torch.tensor([0.01], device="cuda"), torch.linspace(0.01, 0.03, E, device="cuda")
        self.h = [torch.zeros(R, inner // 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.hs = [torch.zeros(R * inner // 16, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.y = [torch.zeros(R, hidden, dtype=BF, device="cuda") for _ in range(2)]
        self.dense = torch.zeros(128, hidden, dtype=BF, device="cuda")
        self.x = codes(128, inner // 2), ones(128 * inner, False)

    def outputs(self):
        return [*self.h, *self.hs, *self.y, self.dense]

    def run(self):
        N, p, H, I = self.N, self.plan, self.hidden, self.inner
        N.nvfp4_linear_grouped_swiglu_quantize(p, self.a[0], self.a[1][0], self.g, self.up[0], self.up[1][0], self.g_w, I, H,
                                               self.g, self.h[0], self.hs[0])
        N.nvfp4_linear(*self.x, self.g, self.down[0][0], self.down[1][0][:H * I // 16], self.g, self.dense, 128, H, I)
        N.nvfp4_linear_grouped(p, self.h[0], self.hs[0], self.g, self.down[0], self.down[1][0], self.g_w, self.y[0], H, I)
        N.mxfp4_linear_grouped_swiglu_quantize(p, self.a[0], self.a[1][1], self.up[0], self.up[1][1], I, H, self.h[1],
                                               self.hs[1], rotate=True)
        N.mxfp4_linear_grouped(p, self.h[1], self.hs[1], self.down[0], self.down[1][1], self.y[1], H, I)


# Two launches of tiles of 64 tokens share an SM; tiles of 256 take one each.
@pytest.mark.parametrize("first,second", [([9] * 40, [3, 0, 17, 1] * 8), ([400, 0, 77, 900], [1200, 300]),
                                          ([9] * 40, [1200, 300])], ids=["small tiles", "large tiles", "both"])
def test_products_of_two_layers_at_once(N, first, second):
    layers = [Products(N, first, 1024, 512, 1), Products(N, second, 512, 768, 2)]
    alone = []
    for layer in layers:
        layer.run()
        torch.cuda.synchronize()
        alone.append([t.clone() for t in layer.outputs()])

    def clear():
        for layer in layers:
            for t in layer.outputs():
                t.zero_()
        torch.cuda.synchronize()

    def check():
        torch.cuda.synchronize()
        assert N.nvfp4_get_device_status() == 0
        for layer, want in zip(layers, alone):
            for a, b in zip(layer.outputs(), want):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    streams = [torch.cuda.Stream() for _ in layers]
    clear()
    for _ in range(20):
        for layer, s in zip(layers, streams):
            with torch.cuda.stream(s):
                layer.run()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        for layer, s in zip(layers, streams):
            s.wait_stream(main)
            with torch.cuda.stream(s):
                layer.run()
        for s in streams:
            main.wait_stream(s)
    clear()
    for _ in range(20):
        graph.replay()
    check()
