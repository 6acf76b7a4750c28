"""extend_attention_nvfp4 on scores of 2^24 to 2^28 (in units of log2) that lie 8 to 32 apart.

The caches are built so that every score is a whole number that fp32 holds exactly: channel 0 carries the large part,
channel 16 (another block) the step, and the softmax scale is the fp32 number whose product with log2(e) rounds to 1.
The tolerance is that of a few f16-rounded weights, 2^-10 of sum(weight * |v|), and half a bf16 ulp.
"""
import math

import numpy as np
import pytest
import torch

import _paged as P
from _util import lib
from test_gpu_extend_attention import queries, run
from test_gpu_extend_attention_long import reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def N():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return lib()


def unit_scale():
    """fp32 s with fl(s * fl(log2 e)) == 1."""
    log2e = np.float32(math.log2(math.e))
    s = np.float32(math.log(2))
    for _ in range(64):
        if np.float32(s * log2e) == np.float32(1):
            return float(s)
        s = np.nextafter(s, np.float32(0 if s * log2e > 1 else 1))
    raise AssertionError("no such number")


def e4m3_of(power):
    """The E4M3 byte of 2^power."""
    return (power + 7) << 3


def built_case(N, length, base, steps, kv_format=0):
    """One KV head whose key t scores base + steps[t] for the query of `built_query`; base even, steps multiples of 4."""
    case = P.Case(N, [length], 1, 0, kv_format, seed=500)
    codes, scales = np.zeros((1, 1, length, 64), np.uint8), np.full((1, 1, length, 8), e4m3_of(0), np.uint8)
    two = 4                                       # the nibble of 2.0 in both formats
    codes[..., 0] = two                           # channel 0
    scales[..., 1] = e4m3_of(-6)                  # channels 16..31
    grid = list(P.E1M2[:8] if kv_format else P.E2M1[:8])
    codes[0, 0, :, 8] = [grid.index(s / 8) for s in steps]
    case.data["k"] = (codes, scales)
    case.cache.k_codes.copy_(torch.from_numpy(codes))
    case.cache.k_scales.copy_(torch.from_numpy(scales))
    case.cache.k_gscale = 1.0
    return case


def built_query(base, tokens, heads):
    """base / 2 in channel 0, 2^9 in channel 16: exact in f16 beside one another."""
    q = torch.zeros(tokens, heads, 128, device="cuda")
    q[:, :, 0] = base / 2
    q[:, :, 16] = 2.0 ** 9
    b = q.to(torch.bfloat16)
    assert (b.float() == q).all()
    return b


# (base, step): a running maximum of `base`, then a key that is `step` above it.
STEPS = [(2 ** 24, 8), (2 ** 24, 12), (2 ** 24, 16), (2 ** 25, 12), (2 ** 25, 16), (2 ** 26, 16), (2 ** 26 + 2 ** 19, 8),
         (2 ** 26 + 2 ** 19, 16), (2 ** 27, 16), (2 ** 20, 12), (2 ** 16, 16)]


@pytest.mark.parametrize("tokens", [1, 4, 60])
@pytest.mark.parametrize("base,step", STEPS)
@pytest.mark.parametrize("kv_format", [0, 1])
@pytest.mark.parametrize("bias", [False, True])
def test_a_step_above_the_running_maximum(N, tokens, base, step, kv_format, bias):
    """64 keys at the base, then 64 of which two in three are a step above it, and so on: within any part of the keys."""
    length = 1400
    t = np.arange(length)
    steps = np.where((t // 64 % 2 == 1) & (t % 3 != 0), step, 0).astype(float)
    case = built_case(N, length, base, steps, kv_format)
    q = built_query(base, tokens, 5)
    slopes = torch.zeros(5, device="cuda") if bias else None  # no bias, by the kernels that have one
    out = run(N, case, q, [tokens], scale=unit_scale(), slopes=slopes)
    torch.cuda.synchronize()
    v = case.rows_of("v", 0)[0][0] * float(np.float32(P.GV))
    y = out.double().cpu().numpy()
    assert np.isfinite(y).all()
    for j in range(tokens):
        seen = length - tokens + j + 1
        w = 2.0 ** (steps[:seen] - steps[:seen].max())
        want, mass = w @ v[:seen] / w.sum(), w @ np.abs(v[:seen]) / w.sum()
        over = np.abs(y[j] - want) - (P.half_ulp(want) * (1 + 2.0 ** -6) + 2.0 ** -10 * mass)
        assert over.max() <= 0, f"worst excess {over.max():.3e}"


@pytest.mark.parametrize("tokens", [1, 4, 60])
@pytest.mark.parametrize("base", [2 ** 24, 2 ** 26 + 2 ** 19, 2 ** 27])
def test_parts_and_tiles_that_join_far_apart_maxima(N, tokens, base):
    """Long enough for several parts: each part of the keys has another maximum."""
    length = 9000
    heights = (0, 16, 32, 48) if base >= 2 ** 27 else (0, 8, 16, 24)  # multiples of fp32's step there
    steps = np.array([heights[t * 7 // length % 4] for t in range(length)], float)
    case = built_case(N, length, base, steps)
    out = run(N, case, built_query(base, tokens, 5), [tokens], scale=unit_scale())
    torch.cuda.synchronize()
    v = case.rows_of("v", 0)[0][0] * float(np.float32(P.GV))
    for j in range(tokens):
        seen = length - tokens + j + 1
        w = 2.0 ** (steps[:seen] - steps[:seen].max())
        want, mass = w @ v[:seen] / w.sum(), w @ np.abs(v[:seen]) / w.sum()
        over = np.abs(out[j].double().cpu().numpy() - want) - (P.half_ulp(want) * (1 + 2.0 ** -6) + 2.0 ** -10 * mass)
        assert over.max() <= 0, f"worst excess {over.max():.3e}"


@pytest.mark.parametrize("news", [[1, 1], [4, 4], [150, 20]])
@pytest.mark.parametrize("log_spread", [24, 40])
def test_capped_scores_past_fp32s_integers(N, news, log_spread):
    """Where every visible score is clear of zero by far more than the cap and its own error, each is +-c: values compared."""
    case = P.Case(N, [1500, 800], 2, 0, 0, seed=510)
    cap = 20.0
    q = queries(sum(news), 10, 30, spread=2.0 ** log_spread)
    out = run(N, case, q, news, logit_cap=cap)
    torch.cuda.synchronize()
    clear, first = np.zeros((len(q), 10), bool), 0
    for b, n in enumerate(news):
        k = torch.from_numpy(case.rows_of("k", b)[0]).cuda() * float(np.float32(P.GK)) / math.sqrt(128)
        hidden = torch.arange(case.lens[b], device="cuda") > (case.lens[b] - n + torch.arange(n, device="cuda"))[:, None]
        for h in range(10):
            qq, kk = q[first:first + n, h].double(), k[h // 5]
            s = (qq @ kk.T).abs() - 2.0 ** -18 * (qq.abs() @ kk.abs().T)
            clear[first:first + n, h] = (s.masked_fill(hidden, math.inf).amin(1) > 10 * cap).cpu().numpy()
        first += n
    assert clear.any()
    ref, bound, _ = reference(case, q, news, logit_cap=cap)
    over = np.abs(out.double().cpu().numpy() - ref) - (P.half_ulp(ref) * (1 + 2.0 ** -6) + bound)
    assert over[clear].max() <= 0
