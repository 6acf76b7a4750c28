"""Layers of experts in the serving example: every operator's result, in the chain, against the chain's own inputs.

Tolerances: the router's choice and the rows exactly; weights 100 units of 2^-23 (its own tests); the down products half a
bf16 step, and K 2^-23 of the sum of magnitudes; the sum over a token's rows half a step and 2^-21 of its terms.
"""
import numpy as np
import pytest
import torch

import _moe as M
from _util import f32, lib
from test_gpu_moe_route import choice, weights_of

pytestmark = pytest.mark.gpu
H, I, HQ, HKV, PAGE, B = 512, 256, 10, 2, 16, 3


@pytest.fixture(scope="module")
def S():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    lib()
    from paper_2606_15682_gb300 import serve
    return serve


class Setup:
    def __init__(self, S, layers, top, experts, top_k):
        per = -(-top // PAGE)
        self.layers = [S.random_layer(H, I, HQ, HKV, B * per, PAGE, 7 + i, experts=experts, top_k=top_k)[1]
                       for i in range(layers)]
        gen = torch.Generator(device="cuda").manual_seed(3)
        self.table = torch.randperm(B * per, generator=gen, device="cuda").to(torch.int32).view(B, per)
        self.lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.rope = torch.empty(top, 64, 2, dtype=torch.float32, device="cuda")
        S.N.nvfp4_rope_table(self.rope)
        self.norm = torch.linspace(0.5, 1.5, H, device="cuda").to(torch.bfloat16)
        self.x = torch.randn(B, top, H, generator=gen, device="cuda").to(torch.bfloat16)

    def batch(self, S, n_new):
        return S.Batch(self.layers[0], self.table, self.lens, n_new, self.rope)


@pytest.mark.parametrize("experts,top_k", [(16, 1), (16, 4), (64, 8)])
@pytest.mark.parametrize("steps", [[40, 1, 3], [200, 1]])
def test_each_operator_in_the_chain(S, experts, top_k, steps):
    N = S.N
    s = Setup(S, 1, sum(steps), experts, top_k)
    layer, at = s.layers[0], 0
    down = [M.operand(layer.down[0][e].cpu().numpy(), layer.down[1][e].cpu().numpy(), H, I, False) for e in range(experts)]
    for n in steps:
        b = s.batch(S, n)
        h = b.run(s.layers, s.x[:, at:at + n].reshape(-1, H), s.norm)
        at += n
        torch.cuda.synchronize()
        assert N.nvfp4_get_device_status() == 0 and torch.isfinite(h).all()
        idx, w = b.expert_idx.cpu().numpy(), b.expert_weights.double().cpu().numpy()
        l = b.logits.double().cpu().numpy()
        assert np.array_equal(idx, choice(l, top_k))
        want = weights_of(l, idx, False, True, 1.0)
        assert (np.abs(w - want) <= 100 * 2.0 ** -23 * want).all()
        start, rows, row_of = M.plan_of(idx, experts)
        p = b.plan
        assert np.array_equal(p.row_of.cpu().numpy(), row_of) and np.array_equal(p.rows.cpu().numpy(), rows)
        # The rows are the norm's own codes, which the router's linear read.
        t, j = np.nonzero(row_of >= 0)
        assert torch.equal(b.a_rows[0][row_of[t, j]], b.a_gu[0][t])
        live, expert = M.live_rows(p)
        a = M.operand(b.a_down[0].cpu().numpy(), b.a_down[1].cpu().numpy(), p.max_rows, I, False)[live]
        sums, mag = M.products(a, expert, down)
        g = (f32(layer.g[3]) * f32(layer.down[2])).astype(np.float64)[expert][:, None]
        y = b.y_rows.double().cpu().numpy()
        over = np.abs(y[live] - sums * g) - M.half_ulp(sums * g) * (1 + 2.0 ** -6) - I * 2.0 ** -23 * mag * g
        assert over.max() <= 0
        terms = y[row_of] * w[..., None]
        out = b.y.double().cpu().numpy()
        over = np.abs(out - terms.sum(1)) - M.half_ulp(out) * (1 + 2.0 ** -6) - 2.0 ** -21 * np.abs(terms).sum(1)
        assert over.max() <= 0
        assert sums.std() > 0 and rows.max() > 0


def test_decode_steps_replayed_from_a_graph(S):
    """Captured once, replayed for three tokens: the same bits as three direct steps."""
    T, results = 60, []
    for graphed in (False, True):
        s = Setup(S, 2, T + 5, 16, 4)
        s.batch(S, T).run(s.layers, s.x[:, :T].reshape(-1, H), s.norm)
        one = s.batch(S, 1)
        x = s.x[:, T].contiguous()
        if graphed:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                one.run(s.layers, x, s.norm)  # warm-up: its token is taken back and overwritten
                s.lens -= 1
            side.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                x.copy_(one.run(s.layers, x, s.norm))
        for _ in range(3):
            g.replay() if graphed else x.copy_(one.run(s.layers, x, s.norm))
        torch.cuda.synchronize()
        results.append((x.clone(), s.lens.clone(), one.expert_idx.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert S.N.nvfp4_get_device_status() == 0


def test_layers_that_do_not_fit_are_refused(S):
    s = Setup(S, 1, 8, 16, 4)
    plain = S.random_layer(H, I, HQ, HKV, 4, PAGE, 1)[1]
    b = s.batch(S, 2)
    x = s.x[:, :2].reshape(-1, H)
    for layers in ([plain], [s.layers[0], plain], [S.random_layer(H, I, HQ, HKV, 4, PAGE, 1, experts=16, top_k=2)[1]]):
        with pytest.raises(ValueError, match="experts"):
            b.run(layers, x, s.norm)
    for kw in (dict(experts=8, top_k=2), dict(experts=16, top_k=0), dict(experts=16, top_k=17), dict(top_k=2)):
        with pytest.raises(ValueError):
            S.random_layer(H, I, HQ, HKV, 4, PAGE, 1, **kw)
    assert (s.lens == 0).all()
