"""The layer that serves from a paged cache: every operator's result, in the chain, against the chain's own inputs.

Each step's buffers hold what passed between the calls, so each new operator is judged by 64-bit arithmetic on
what it was given there; the two linears' own errors do not enter.  Tolerances: attention as in its own tests (a bf16
rounding and 2^-10 of sum(weight * |v|)); sums and norms half a bf16 ulp and 2^-18 of their terms; quantized K and V half
of the widest E2M1 step (1 of 6) of their block's amax plus the E4M3 scale's 1/16.
"""
import math

import numpy as np
import pytest
import torch

import _paged as P
from _util import lib

pytestmark = pytest.mark.gpu
H, I, HQ, HKV, PAGE, B = 512, 256, 10, 2, 16, 3


@pytest.fixture(scope="module")
def S():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    lib()
    from paper_2606_15682_gb300 import serve
    return serve


class Setup:
    def __init__(self, S, layers, top, kv_format=0):
        per = -(-top // PAGE)
        made = [S.random_layer(H, I, HQ, HKV, B * per + 2, PAGE, 7 + i, kv_format=kv_format) for i in range(layers)]
        self.layers = [m[1] for m in made]
        gen = torch.Generator(device="cuda").manual_seed(3)
        self.table = torch.randperm(B * per + 2, generator=gen, device="cuda")[:B * per].to(torch.int32).view(B, per)
        self.lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.rope = torch.empty(top, 64, 2, dtype=torch.float32, device="cuda")
        S.N.nvfp4_rope_table(self.rope)
        self.norm = torch.linspace(0.5, 1.5, H, device="cuda").to(torch.bfloat16)
        self.x = torch.randn(B, top, H, generator=gen, device="cuda").to(torch.bfloat16)

    def batch(self, S, n_new):
        return S.Batch(self.layers[0], self.table, self.lens, n_new, self.rope)


def near(got, want, slack):
    got, want = got.double().cpu().numpy(), want.double().cpu().numpy()
    slack = slack.double().cpu().numpy()
    assert np.isfinite(got).all()
    over = np.abs(got - want) - P.half_ulp(want) * (1 + 2.0 ** -6) - slack
    assert over.max() <= 0, f"worst excess {over.max():.3e}"


@pytest.mark.parametrize("kv_format", [0, 1])
@pytest.mark.parametrize("steps", [[40, 1, 1, 3, 1], [1, 17, 90], [600, 5, 1, 1]])
def test_each_operator_in_the_chain(S, steps, kv_format):
    N = S.N
    s = Setup(S, 1, sum(steps) + 3, kv_format)
    layer, at = s.layers[0], 0
    k_all, v_all = [], []
    for n in steps:
        b = s.batch(S, n)
        x = s.x[:, at:at + n].reshape(-1, H)
        h = b.run(s.layers, x, s.norm)
        at += n
        torch.cuda.synchronize()
        assert N.nvfp4_get_device_status() == 0 and (s.lens == at).all()
        # What the norms gave the linears: the codes of the plain norm, but where it lies on a rounding edge.
        one = torch.ones(H, dtype=torch.float64, device="cuda")

        def plain_norm(r, w):
            r = r.double()
            return r / (r * r).mean(1, keepdim=True).add(1e-6).sqrt() * w
        for r, (codes, _), g in ((x, b.a_qkv, layer.g[0]),):
            c2, s2 = torch.empty_like(codes), torch.empty_like(b.a_qkv[1])
            N.nvfp4_quantize(plain_norm(r, one).to(torch.bfloat16), g, c2, s2, N.SCALES_MMA)
            assert (c2 != codes).float().mean() < 0.02
        # Rotated queries and the cache's rows.
        q0, k0, v0 = b.qkv.view(B, n, HQ + 2 * HKV, 128).double().split([HQ, HKV, HKV], 2)
        cs = s.rope[at - n:at].double()[None, :, None]

        def rotated(t):
            a, c = t[..., :64], t[..., 64:]
            return torch.cat([a * cs[..., 0] - c * cs[..., 1], a * cs[..., 1] + c * cs[..., 0]], -1)
        near(b.q.view(B, n, HQ, 128), rotated(q0), 2.0 ** -18 * (q0.abs() + q0.roll(64, -1).abs()))
        k_all.append(rotated(k0))
        v_all.append(v0)
        k_want, v_want = torch.cat(k_all, 1), torch.cat(v_all, 1)
        kv = [b.cached(layer, i, 0, at) for i in range(B)]
        k_got, v_got = (torch.stack([t[j] for t in kv]).double() for j in (0, 1))
        for got, want in ((k_got, k_want), (v_got, v_want)):
            amax = want.unflatten(-1, (8, 16)).abs().amax(-1).repeat_interleave(16, -1)
            assert ((got - want).abs() <= amax * (1 / 6 + 1 / 16) + 2.0 ** -9 * layer.cache.k_gscale).all()
        # Attention over exactly those rows (bf16 of them: 2^-9 of a score's terms, and of V).
        q = b.q.view(B, n, HQ, 128).double()
        kk, vv = (t.repeat_interleave(HQ // HKV, 2) for t in (k_got, v_got))
        z = torch.einsum("bnhd,bthd->bhnt", q, kk) / math.sqrt(128)
        dz = 2.0 ** -8 * torch.einsum("bnhd,bthd->bhnt", q.abs(), kk.abs()) / math.sqrt(128)
        hidden = torch.arange(at, device="cuda")[None] > (at - n + torch.arange(n, device="cuda"))[:, None]
        w = torch.softmax(z.masked_fill(hidden, -math.inf), -1)
        want = torch.einsum("bhnt,bthd->bnhd", w, vv)
        # A score off by dz moves its weight by that part of it, and the sum of weights by as much at most.
        slack = torch.einsum("bhnt,bthd->bnhd", w * (2 * dz + 2.0 ** -8), vv.abs())
        slack = slack + torch.einsum("bhnt,bhnt->bhn", w, 2 * dz).transpose(1, 2)[..., None] * want.abs()
        near(b.attn.view(B, n, HQ, 128), want, slack + 2.0 ** -10 * torch.einsum("bhnt,bthd->bnhd", w, vv.abs()))
        # The residual stream and the last norm: r = (x + o, rounded) + y.
        r1 = (x.double() + b.o.double()).to(torch.bfloat16).double()
        near(b.r, r1 + b.y.double(), 2.0 ** -18 * (r1.abs() + b.y.double().abs()))
        near(h, plain_norm(r1 + b.y.double(), s.norm.double()), 2.0 ** -18 * torch.full_like(r1, 8.0))


def test_chunks_agree_with_the_whole_prompt(S):
    """The same tokens in one call and in chunks: the last norm's outputs differ by what the linears' order of
    summation moves across FP4 rounding edges, far below the size of the outputs."""
    T = 150
    outs = []
    for steps in ([T], [64, 64, 22], [100] + [1] * 10 + [40]):
        s, at, rows = Setup(S, 2, T), 0, []
        for n in steps:
            rows.append(s.batch(S, n).run(s.layers, s.x[:, at:at + n].reshape(-1, H), s.norm).view(B, n, H).clone())
            at += n
        outs.append(torch.cat(rows, 1).double())
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert ((o - outs[0]).norm() / outs[0].norm()).item() < 0.1


def test_decode_steps_replayed_from_a_graph(S):
    """Captured once, replayed for three tokens: the same bits as three direct steps."""
    T, results = 60, []
    for graphed in (False, True):
        s = Setup(S, 2, T + 5)
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
        results.append((x.clone(), s.lens.clone(), one.cached(s.layers[1], 2, 0, T + 3)))
    (x0, l0, kv0), (x1, l1, kv1) = results
    assert torch.equal(x0, x1) and torch.equal(l0, l1) and all(torch.equal(a, b) for a, b in zip(kv0, kv1))
    assert S.N.nvfp4_get_device_status() == 0
