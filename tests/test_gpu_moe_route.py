"""The router's choice, weights and gradient against 64 bits.

Tolerances.  CUDA's fast exponential is within 2 + 1.173 |x| units of 2^-23, with |x| the distance to the largest logit
(at most 24 here): 30 units; a sum of experts has the units of its terms and one for each of the at most 37 additions of a
lane and the warp, and a quotient adds both: 100 units of 2^-23 relative to a weight.  Sigmoid: expf 1 unit, a sum, a
reciprocal: 3 units, 40 with the sum and quotient.  A gradient w (D - sum D w) has such an error of each of its terms.  A
choice under a bias is by 32 bits: in 64 bits, neighbours in the order may lie 2^-21 of their sizes the wrong way round.
"""
import numpy as np
import pytest
import torch

import _moe as M
from _util import lib

pytestmark = pytest.mark.gpu
UNIT = 2.0 ** -23


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


def logits(tokens, experts, seed, dtype=torch.float32, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    l = (2 * torch.randn(tokens, experts + pad, generator=g, device="cuda")).clamp(-12, 12).to(dtype)
    return l[:, :experts]


def scores(l, sigmoid):
    l = np.where(np.isnan(l), -np.inf, l)
    if sigmoid:
        return 1 / (1 + np.exp(-l))
    top = l.max(1, keepdims=True)
    e = np.where(l == top, 1.0, np.where(np.isfinite(top), np.exp(np.minimum(l - np.where(np.isfinite(top), top, 0), 0)), 0.0))
    e = np.where(l == -np.inf, 0.0, e)  # beside a logit of +inf every finite one has nothing
    return e / np.maximum(e.sum(1, keepdims=True), 1e-300)


def weights_of(l, idx, sigmoid, renormalize, scale):
    p = np.take_along_axis(scores(l, sigmoid), np.maximum(idx, 0).astype(np.int64), 1) * (idx >= 0)
    if renormalize:
        total = p.sum(1, keepdims=True)
        p = np.where(total > 0, p / np.where(total > 0, total, 1), 0)
    return p * float(np.float32(scale))


def choice(key, k):
    """The k largest, the lowest index among equal ones, -1 in place of -inf and NaN."""
    key = np.where(np.isnan(key), -np.inf, key)
    idx = np.argsort(-key, axis=1, kind="stable")[:, :k]
    return np.where(np.take_along_axis(key, idx, 1) == -np.inf, -1, idx)


def run(N, l, k, **kw):
    idx = torch.full((l.shape[0], k), 99999, dtype=torch.int32, device="cuda")
    w = torch.full((l.shape[0], k), float("nan"), device="cuda")
    N.moe_route(l, idx, w, **kw)
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 0
    return idx.cpu().numpy(), w.double().cpu().numpy()


SHAPES = [(1, 1, 1), (1, 2, 1), (5, 2, 2), (3, 31, 5), (33, 32, 32), (130, 64, 8), (7, 33, 4), (65, 128, 6), (257, 256, 8),
          (4, 300, 8), (9, 512, 16), (6, 1000, 32), (5, 1024, 8)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("tokens,experts,k", SHAPES)
def test_choice_and_weights(N, tokens, experts, k, score, renormalize, dtype):
    l = logits(tokens, experts, experts + k, dtype, pad=5)  # bf16: many equal logits
    sig = score == "sigmoid"
    idx, w = run(N, l, k, score=N.MOE_SIGMOID if sig else N.MOE_SOFTMAX, renormalize=renormalize, scale=1.7)
    l64 = l.double().cpu().numpy()
    assert np.array_equal(idx, choice(l64, k))
    want = weights_of(l64, idx, sig, renormalize, 1.7)
    assert (np.abs(w - want) <= 100 * UNIT * want + 1e-37).all()


@pytest.mark.parametrize("tokens,experts,k", [(40, 8, 2), (300, 256, 8), (20, 1000, 12)])
def test_a_bias_moves_the_choice_alone(N, tokens, experts, k):
    l = logits(tokens, experts, 4)
    bias = 0.3 * torch.randn(experts, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda")
    idx, w = run(N, l, k, score=N.MOE_SIGMOID, bias=bias)
    l64, b64 = l.double().cpu().numpy(), bias.double().cpu().numpy()
    key = scores(l64, True) + b64
    got = np.take_along_axis(key, idx.astype(np.int64), 1)
    slack = 2.0 ** -21 * (1 + np.abs(b64).max())
    assert (np.diff(got, axis=1) <= slack).all() and all(len(set(r)) == k for r in idx)
    rest = key.copy()
    np.put_along_axis(rest, idx.astype(np.int64), -np.inf, 1)
    assert (rest.max(1) <= got[:, -1] + slack).all()
    assert (idx != choice(l64, k)).any()
    want = weights_of(l64, idx, True, True, 1.0)
    assert (np.abs(w - want) <= 100 * UNIT * want).all()


def test_equal_scores_go_to_the_lowest_index(N):
    l = torch.zeros(3, 70, device="cuda")
    l[1, 40:] = 1.0
    l[2, ::2] = -0.0  # both zeros are one
    idx, w = run(N, l, 4)
    assert idx.tolist() == [[0, 1, 2, 3], [40, 41, 42, 43], [0, 1, 2, 3]] and (w == 0.25).all()
    bias = torch.zeros(70, device="cuda")
    bias[50] = 0.5
    idx, _ = run(N, l, 3, score=N.MOE_SIGMOID, bias=bias)
    assert idx.tolist() == [[50, 0, 1], [50, 40, 41], [50, 0, 1]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_experts_and_tokens(N, score, renormalize, dtype):
    inf, nan = float("inf"), float("nan")
    l = logits(8, 40, 2, dtype)
    l[0] = -inf
    l[1, 3:] = -inf
    l[2, 5:] = nan
    l[3] = nan
    l[4, 7], l[4, 30] = inf, inf
    l[5, 0] = torch.finfo(dtype).min
    l[6, 1:] = torch.finfo(dtype).min
    l[7, 20] = inf
    sig = score == "sigmoid"
    idx, w = run(N, l, 6, score=N.MOE_SIGMOID if sig else N.MOE_SOFTMAX, renormalize=renormalize)
    l64 = l.double().cpu().numpy()
    assert np.array_equal(idx, choice(l64, 6))
    with np.errstate(over="ignore", invalid="ignore"):
        want = weights_of(l64, idx, sig, renormalize, 1.0)
    assert np.isfinite(w).all() and (np.abs(w - want) <= 100 * UNIT * want + 1e-37).all()
    d = torch.randn(8, 6, device="cuda")
    out = torch.full_like(l, nan)
    N.moe_route_backward(l, torch.as_tensor(idx, device="cuda"), d, out, score=N.MOE_SIGMOID if sig else N.MOE_SOFTMAX,
                         renormalize=renormalize)
    assert torch.isfinite(out).all() and not out[0].any() and not out[3].any()
    if not sig:
        assert not out[1, 3:].any()


def test_a_bias_of_minus_infinity_shuts_an_expert(N):
    l = logits(50, 12, 1)
    bias = torch.zeros(12, device="cuda")
    bias[3], bias[5] = -float("inf"), float("nan")
    idx, w = run(N, l, 11, score=N.MOE_SIGMOID, bias=bias)
    assert not np.isin(idx, [3, 5]).any() and (idx[:, 10] == -1).all() and (w[:, 10] == 0).all()
    assert (idx[:, :10] >= 0).all()


def gradient(l, idx, d, sigmoid, renormalize, scale):
    """(d_logits, the magnitudes that an error is relative to), 64 bits."""
    p, D = scores(l, sigmoid), d * float(np.float32(scale))
    out, mag = np.zeros_like(l), np.zeros_like(l)
    for t in range(len(l)):
        has = np.nonzero(idx[t] >= 0)[0]
        q, g = p[t, idx[t, has]], D[t, has]
        if renormalize:
            w = q / q.sum()
            part, size = w * (g - (g * w).sum()), w * (np.abs(g) + (np.abs(g) * w).sum())
            if sigmoid:
                part, size = part * (1 - q), size * (1 - q)
        elif sigmoid:
            part, size = g * q * (1 - q), np.abs(g) * q * (1 - q)
        else:
            part, size = g * q, np.abs(g) * q
            out[t] -= p[t] * part.sum()
            mag[t] += p[t] * size.sum()
        np.add.at(out[t], idx[t, has], part)
        np.add.at(mag[t], idx[t, has], size)
    return out, mag


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("tokens,experts,k", SHAPES)
def test_gradient(N, tokens, experts, k, score, renormalize, dtype):
    l = logits(tokens, experts, experts, dtype, pad=3)
    sig = score == "sigmoid"
    kw = dict(score=N.MOE_SIGMOID if sig else N.MOE_SOFTMAX, renormalize=renormalize, scale=0.8)
    idx = torch.empty(tokens, k, dtype=torch.int32, device="cuda")
    w = torch.empty(tokens, k, device="cuda")
    N.moe_route(l, idx, w, **kw)
    if tokens > 4:
        idx[1, 0], idx[2, 0], idx[3] = -1, experts, idx[3, 0]  # none, no expert's number, one expert k times
    d = torch.randn(tokens, k, device="cuda")
    out = torch.full((tokens, experts), float("nan"), dtype=dtype, device="cuda")
    N.moe_route_backward(l, idx, d, out, **kw)
    ii = idx.cpu().numpy()
    want, mag = gradient(l.double().cpu().numpy(), np.where(ii >= experts, -1, ii), d.double().cpu().numpy(), sig,
                         renormalize, 0.8)
    got = out.double().cpu().numpy()
    half = M.half_ulp(want) * (1 + 2.0 ** -6) if dtype == torch.bfloat16 else 0
    assert (np.abs(got - want) <= half + 200 * UNIT * mag + 1e-37).all()
    torch.cuda.synchronize()
    assert N.nvfp4_get_device_status() == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("experts", [20, 40, 256])
@pytest.mark.parametrize("renormalize", [True, False])
def test_gradient_of_choices_far_below_the_largest_logit(N, renormalize, experts, dtype):
    """A caller's own choices: normed weights are shares among the chosen, however little softmax leaves to all of them;
    beside a logit of +inf it leaves nothing."""
    l = logits(6, experts, 3, dtype)
    l[1, 0], l[2, 0], l[3, 0], l[4, 0] = 60, 150, 3e38, float("inf")
    idx = torch.arange(1, 6, dtype=torch.int32, device="cuda").repeat(6, 1)
    d = torch.randn(6, 5, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    out = torch.full((6, experts), float("nan"), dtype=dtype, device="cuda")
    N.moe_route_backward(l, idx, d, out, renormalize=renormalize, scale=0.8)
    l64 = l.double().cpu().numpy()
    got = out.double().cpu().numpy()
    assert (got[4] == 0).all()
    if renormalize:
        l64[3, 0] = 150  # the shares do not depend on it, and 64 bits have e^-150
    else:
        assert (got[3] == 0).all()
    some = [0, 1, 2] + [3] * renormalize + [5]
    want, mag = gradient(l64[some], idx.cpu().numpy()[some], d.double().cpu().numpy()[some], False, renormalize, 0.8)
    half = M.half_ulp(want) * (1 + 2.0 ** -6) if dtype == torch.bfloat16 else 0
    assert (np.abs(got[some] - want) <= half + 200 * UNIT * mag + 1e-37).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
def test_gradient_is_that_of_differences(N, score, renormalize):
    """Of the weights' definition in 64 bits, with the choice held: central differences, h = 2^-17, error h^2 + 2^-53 / h."""
    tokens, experts, k, sig = 6, 20, 4, score == "sigmoid"
    l = logits(tokens, experts, 9)
    kw = dict(score=N.MOE_SIGMOID if sig else N.MOE_SOFTMAX, renormalize=renormalize, scale=1.25)
    idx, w = torch.empty(tokens, k, dtype=torch.int32, device="cuda"), torch.empty(tokens, k, device="cuda")
    N.moe_route(l, idx, w, **kw)
    d = torch.randn(tokens, k, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    out = torch.empty_like(l)
    N.moe_route_backward(l, idx, d, out, **kw)
    l64, ii, d64, h = l.double().cpu().numpy(), idx.cpu().numpy(), d.double().cpu().numpy(), 2.0 ** -17
    for e in range(experts):
        side = []
        for s in (h, -h):
            moved = l64.copy()
            moved[:, e] += s
            side.append((weights_of(moved, ii, sig, renormalize, 1.25) * d64).sum(1))
        want = (side[0] - side[1]) / (2 * h)
        assert np.abs(out[:, e].double().cpu().numpy() - want).max() < 1e-6 * np.abs(d64).sum(1).max()


@pytest.mark.parametrize("experts", [40, 256, 1000])
@pytest.mark.parametrize("scale", [1e-7, 1.0, 1e6])
def test_a_choice_between_close_biased_scores_is_by_their_32_bits(N, experts, scale):
    """Scores that differ by a few units, and biases that hide them or drown in them: the choice is the one by 1 / (1 + e^-l)
    + bias with one rounding for each operation, which torch's elementwise operations on the GPU have too."""
    g = torch.Generator(device="cuda").manual_seed(experts)
    l = 0.3 + 1e-6 * torch.randn(500, experts, generator=g, device="cuda")
    bias = scale * torch.randint(-2, 3, (experts,), generator=g, device="cuda").float()
    idx, _ = run(N, l, 8, score=N.MOE_SIGMOID, bias=bias)
    key = torch.reciprocal(1 + torch.exp(-l)) + bias
    assert np.array_equal(idx, choice(key.double().cpu().numpy(), 8))
