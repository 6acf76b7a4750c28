"""Plain forms of the mixture-of-experts operators in 64 bits, and inputs for them."""
import numpy as np
import torch

from oracle import nvfp4_oracle as O

TILE = 128


def half_ulp(y):
    """Half a bf16 step at y."""
    a = np.maximum(np.abs(np.asarray(y, np.float64)), 2.0 ** -126)
    return np.ldexp(1.0, (np.floor(np.log2(a)) - 8).astype(np.int64))


def rand_bf16(shape, seed, scale=1.0, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=device) * scale).to(torch.bfloat16)


def choices(counts, top_k, seed, drop=0):
    """expert_idx [tokens, top_k] in which expert e is asked for counts[e] times, and `drop` places are -1."""
    flat = np.concatenate([np.full(n, e) for e, n in enumerate(counts)] + [np.full(drop, -1)])
    flat = np.concatenate([flat, np.full(-len(flat) % top_k, -1)])
    return np.random.default_rng(seed).permutation(flat).reshape(-1, top_k).astype(np.int32)


def plan_of(idx, experts):
    """(row_start [E + 1], rows [E], row_of like idx) by the definition."""
    start, rows, row_of = np.zeros(experts + 1, np.int64), np.zeros(experts, np.int64), np.full(idx.size, -1, np.int64)
    flat, at = idx.reshape(-1), 0
    for e in range(experts):
        p = np.nonzero(flat == e)[0]
        start[e], rows[e] = at, len(p)
        row_of[p] = at + np.arange(len(p))
        at += -(-len(p) // TILE) * TILE
    start[experts] = at
    return start, rows, row_of.reshape(idx.shape)


def make_plan(N, idx, experts, check=True):
    idx = torch.as_tensor(idx, dtype=torch.int32, device="cuda").contiguous()
    p = N.MoEPlan(idx.shape[0], idx.shape[1], experts)
    N.moe_sort(p, idx)
    if check:
        start, rows, row_of = plan_of(idx.cpu().numpy(), experts)
        assert np.array_equal(p.row_start.cpu().numpy(), start) and np.array_equal(p.rows.cpu().numpy(), rows)
        assert np.array_equal(p.row_of.cpu().numpy(), row_of)
    return p


def live_rows(plan):
    """Indexes of the rows in use, and each one's expert."""
    start, rows = plan.row_start.cpu().numpy(), plan.rows.cpu().numpy()
    at = [np.arange(s, s + n) for s, n in zip(start, rows)]
    return np.concatenate(at).astype(np.int64), np.repeat(np.arange(len(rows)), rows)


E2M1 = np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6])


def operand(codes, scales, rows, K, mx):
    """Element times block scale, 64 bits, of `rows` rows with tensor-core-ordered scales (numpy uint8)."""
    nib = np.stack([codes & 15, codes >> 4], -1).reshape(rows, K)
    sc = O.scales_from_mma(scales, rows, K).astype(np.int64)
    if mx:
        v = np.ldexp(1.0, sc - 127)
    else:
        v = np.where(sc >> 3 == 0, (sc & 7) / 512.0, np.ldexp(1 + (sc & 7) / 8.0, (sc >> 3) - 7))
    return E2M1[nib] * np.repeat(v, 16, axis=1)


class Weights:
    """E experts' quantized weights [N, K] and their values in 64 bits (without g)."""

    def __init__(self, N_, E, N, K, seed, mx=False, spread=0.3):
        self.codes = torch.empty(E, N, K // 2, dtype=torch.uint8, device="cuda")
        size = N_.nvfp4_scales_bytes(N, K, N_.SCALES_MMA)
        self.scales = torch.empty(E, size, dtype=torch.uint8, device="cuda")
        self.g = torch.ones(E, device="cuda")
        for e in range(E):
            w = rand_bf16((N, K), seed + e, 1 / np.sqrt(K) * (1 + spread * e))
            if mx:
                N_.mxfp4_quantize(w, self.codes[e], self.scales[e], N_.SCALES_MMA)
            else:
                N_.nvfp4_tensor_scale(w, self.g[e:e + 1])
                N_.nvfp4_quantize(w, self.g[e:e + 1], self.codes[e], self.scales[e], N_.SCALES_MMA)
        c, s = self.codes.cpu().numpy(), self.scales.cpu().numpy()
        self.values = [operand(c[e], s[e], N, K, mx) for e in range(E)]


class Rows:
    """The rows of tokens x (with values spread over channels) in a plan, quantized, with junk in the rows between."""

    def __init__(self, N_, plan, K, seed, mx=False, rotate=False):
        self.x = rand_bf16((plan.n_tokens, K), seed, 2.0)
        R = plan.max_rows
        self.codes = torch.full((R, K // 2), 0x77, dtype=torch.uint8, device="cuda")
        self.scales = torch.full((R * K // 16,), 0xFF if mx else 0x7F, dtype=torch.uint8, device="cuda")  # NaN
        self.g = torch.tensor([0.0031], device="cuda")
        if mx:
            N_.moe_dispatch_mxfp4(plan, self.x, self.codes, self.scales, rotate=rotate)
        else:
            N_.moe_dispatch_nvfp4(plan, self.x, self.g, self.codes, self.scales)
        self.at, self.expert = live_rows(plan)
        self.values = operand(self.codes.cpu().numpy(), self.scales.cpu().numpy(), R, K, mx)[self.at]


def products(values, expert, weights):
    """(sum a w, sum |a w|) of each row with its expert's weight, 64 bits."""
    N = weights[0].shape[0]
    out, mag = np.zeros((len(values), N)), np.zeros((len(values), N))
    for e in np.unique(expert):
        r = expert == e
        out[r] = values[r] @ weights[e].T
        mag[r] = np.abs(values[r]) @ np.abs(weights[e]).T
    return out, mag
