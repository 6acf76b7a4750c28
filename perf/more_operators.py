"""A mixture-of-experts layer's operators between its router's logits and its output, and the same in plain torch.

  route    moe_route: each token's experts and their weights from the router's logits, and moe_sort: the rows of the
           tokens sorted by expert; or moe_route_backward: the logits' gradient
  tokens   moe_dispatch: tokens to their experts' rows, and moe_combine: the experts' rows back, weighted and summed;
           or the gradients of both: moe_combine_backward, and moe_combine without weights
  experts  moe_sort, moe_dispatch_nvfp4, nvfp4_linear_grouped_swiglu_quantize, nvfp4_linear_grouped, moe_combine: the
           experts' W4A4 products from bf16 tokens to the layer's bf16 output; the same in MXFP4

Rows of an expert are together, token by token, and each expert's first row is a multiple of 128: the tensor core's
scale tiles.  listed() names twelve cases, draw() gives more of the same ranges; hidden sizes are 1536 and 5120 of
paper_2606_15682_gb300/synth.py and powers of two.  `run` computes the plain form in 32 bits, or calls the framework
where `own` is true.
"""
import functools
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
BF = torch.bfloat16
TILE = 128


# ------------------------------------------------------------------ cases ---

def _route(name, tokens, experts, top_k, score="softmax", renormalize=True, bias=False, bf16=False, grad=False):
    return dict(name=name, kind="route", tokens=tokens, experts=experts, top_k=top_k, score=score,
                renormalize=renormalize, bias=bias, bf16=bf16, grad=grad, skew=1.0, idle=0.0)


def _tokens(name, tokens, hidden, experts, top_k, base=False, grad=False, skew=1.0, idle=0.0):
    return dict(name=name, kind="tokens", tokens=tokens, hidden=hidden, experts=experts, top_k=top_k, base=base,
                grad=grad, skew=skew, idle=idle)


def _experts(name, tokens, hidden, inner, experts, top_k, fmt="nvfp4", base=True, skew=1.0, idle=0.0):
    return dict(name=name, kind="experts", tokens=tokens, hidden=hidden, inner=inner, experts=experts, top_k=top_k,
                fmt=fmt, base=base, skew=skew, idle=idle)


def listed():
    return [
        # A decode step of a small batch: the choice and the rows of 32 tokens, latency only.
        _route("route_t32_e64", 32, 64, 8),
        # A long prompt's tokens on many experts, scores that a bias balances for the choice.
        _route("route_t16384_e256", 16384, 256, 8, score="sigmoid", bias=True),
        # The router's backward pass of a training step, logits in bf16.
        _route("route_grad_t8191_e128", 8191, 128, 4, bf16=True, grad=True),
        # One token's hidden state to its experts and back.
        _tokens("tokens_t1", 1, 2048, 64, 8),
        # A prompt's tokens to their experts and back, added to what a shared expert gave.
        _tokens("tokens_t8192_h5120", 8192, 5120, 32, 4, base=True),
        # The gradients of both in a training step, a padded batch (an eighth of the tokens have no expert).
        _tokens("tokens_grad_t4099_h2048", 4099, 2048, 64, 8, grad=True, idle=0.125),
        # One new token through the layer: the weights of its experts are what is read.
        _experts("experts_t1_h2048", 1, 2048, 1024, 64, 8),
        # A decode batch on many small experts: a few rows each.
        _experts("experts_t64_h2048", 64, 2048, 768, 128, 8),
        # A decode batch on few large experts.
        _experts("experts_t128_h5120", 128, 5120, 2048, 16, 2),
        # Ragged chunks of prompts in MXFP4, some experts much more asked for than others, tokens without experts.
        _experts("experts_t777_h1536_mx", 777, 1536, 1280, 40, 3, fmt="mxfp4", skew=2.0, idle=0.1),
        # A batch of drafts and short prompts: tens of rows an expert.
        _experts("experts_t500_h4096", 500, 4096, 1280, 64, 6, base=False),
        # A long prompt, the largest products.
        _experts("experts_t8192_h5120", 8192, 5120, 1024, 64, 4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "tokens", "experts", "experts"])
    experts = rng.choice([_log(rng, 2, 256), 8, 64, 128])
    top_k = min(experts, rng.choice([1, 2, 3, 4, 6, 8]))
    skew, idle = rng.choice([0.0, 1.0, 2.0]), rng.choice([0.0, 0.0, 0.1])
    if kind == "route":
        sigmoid, renormalize = rng.random() < 0.5, rng.random() < 0.7 and top_k > 1  # the sum of one weight is it
        c = _route("", _log(rng, 1, 12000), experts, top_k, "sigmoid" if sigmoid else "softmax", renormalize,
                   sigmoid and rng.random() < 0.5, rng.random() < 0.5, rng.random() < 0.4)
    elif kind == "tokens":
        hidden = rng.choice([8, 1000, 1536, 2048, 4096, 5120])
        c = _tokens("", _log(rng, 1, min(8192, 8192 * 4 * 5120 // (top_k * hidden))), hidden, experts, top_k,
                    rng.random() < 0.5, rng.random() < 0.5, skew, idle)
    else:
        hidden, inner = rng.choice([512, 1536, 2048, 4096, 5120]), 256 * rng.choice([1, 2, 3, 4, 5, 8])
        experts = min(experts, max(2, int(64 * 5120 * 1024 / (hidden * inner))))
        top_k = min(top_k, experts)
        c = _experts("", _log(rng, 1, min(8192, 8192 * 4 * 5120 * 1024 // (top_k * hidden * inner))), hidden, inner,
                     experts, top_k, rng.choice(["nvfp4", "nvfp4", "mxfp4"]), rng.random() < 0.5, skew, idle)
    del c["name"]
    return c


# ---------------------------------------------------------------- prepare ---

def _choices(case, seed):
    """Each token's experts [tokens, top_k], unequally asked for; -1 for all of a token without experts."""
    key = "%s %s" % (seed, sorted((k, v) for k, v in case.items() if k != "name"))
    rng = np.random.default_rng(random.Random(key).getrandbits(63))
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    asked = rng.standard_normal((T, E), dtype=np.float32) + case["skew"] * rng.standard_normal(E, dtype=np.float32)
    idx = np.argsort(-asked, axis=1, kind="stable")[:, :k].astype(np.int32)
    idx[rng.random(T) < case["idle"]] = -1
    return idx


def _max_rows(case):
    pairs = case["tokens"] * case["top_k"]
    return (pairs + (TILE - 1) * min(case["experts"], pairs)) // TILE * TILE


def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (seed + 1) + salt)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _e2m1(v):
    a = v.abs()
    a = torch.where(a < 2, torch.round(a * 2) * 0.5, torch.where(a < 4, torch.round(a), torch.round(a * 0.5) * 2))
    return torch.copysign(a.clamp(max=6.0), v)


def _nvfp4(x, g):
    """(elements [..., blocks, 16], E4M3 block scales [..., blocks, 1]) of x under the tensor scale g, in 32 bits."""
    b = x.float().unflatten(-1, (-1, 16))
    s = (b.abs().amax(-1, keepdim=True) / (g * 6)).clamp(max=448.0).to(torch.float8_e4m3fn).float()
    return _e2m1(b * torch.where(s > 0, torch.reciprocal(s * g), torch.zeros_like(s))), s


def _mxfp4(x):
    """(elements [..., blocks, 32], power-of-two scales [..., blocks, 1]) of x, in 32 bits."""
    b = x.float().unflatten(-1, (-1, 32))
    e = torch.frexp(b.abs().amax(-1, keepdim=True))[1] - 3  # floor(log2 amax) - 2
    s = torch.ldexp(torch.ones_like(b[..., :1]), e.clamp(min=-126))
    return _e2m1(b / s), s


def _codes(e):
    """Packed E2M1 bytes of elements [..., blocks, block]."""
    e = e.flatten(-2)
    a = e.abs()
    code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a * 0.5 + 4)).to(torch.uint8) | (torch.signbit(e).to(torch.uint8) << 3)
    code = code.unflatten(-1, (-1, 2))
    return code[..., 0] | (code[..., 1] << 4)


def _tensor_core_order(b):
    """Block scale bytes [experts, rows, blocks], one for 16 elements, in the order that the linears read."""
    E, N, B = b.shape
    b = torch.nn.functional.pad(b, (0, 0, 0, -N % TILE))
    return b.view(E, -1, 4, 32, B // 4, 4).permute(0, 1, 4, 3, 2, 5).reshape(E, -1).contiguous()


def _weight(seed, salt, E, N, K, fmt):
    """Experts' weights as a checkpoint holds them: codes [E, N, K/2], block scales, tensor scales [E]."""
    codes, scales, gs = [], [], []
    for i in range(E):
        w = (_normal(_gen(seed, salt + i), N, K) / math.sqrt(K)).to(BF)
        if fmt == "nvfp4":
            g = w.abs().amax().float() / 2688
            e, s = _nvfp4(w, g)
            scales.append(s.squeeze(-1).to(torch.float8_e4m3fn).view(torch.uint8))
        else:
            g = torch.ones((), device=DEV)
            e, s = _mxfp4(w)
            scales.append((torch.frexp(s)[1] + 126).squeeze(-1).to(torch.uint8))
        codes.append(_codes(e))
        gs.append(g)
    c = dict(codes=torch.stack(codes), scales=torch.stack(scales), g=torch.stack(gs).view(E))
    c["ordered"] = _tensor_core_order(c["scales"] if fmt == "nvfp4" else c["scales"].repeat_interleave(2, -1))
    return c


def prepare(case, seed):
    kind, T, E, k = case["kind"], case["tokens"], case["experts"], case["top_k"]
    s = dict(case=case)
    if kind == "route":
        logits = 1.5 * _normal(_gen(seed, 1), T, E) + _normal(_gen(seed, 2), E)
        s["logits"] = logits.to(BF) if case["bf16"] else logits
        s["idx"] = torch.sort(s["logits"], dim=1, descending=True, stable=True)[1][:, :k].int().contiguous()
        s["bias"] = 0.1 * _normal(_gen(seed, 3), E) if case["bias"] else None
        s["d_weights"] = _normal(_gen(seed, 4), T, k)
        s["out_idx"], s["out_weights"] = torch.empty_like(s["idx"]), torch.empty(T, k, device=DEV)
        s["d_logits"] = torch.empty_like(s["logits"])
    else:
        idx = _choices(case, seed)
        s["idx"] = torch.as_tensor(idx, device=DEV)
        H, R = case["hidden"], _max_rows(case)
        s["weights"] = torch.softmax(_normal(_gen(seed, 5), T, k), -1) * (s["idx"] >= 0)
        spread = torch.exp(0.5 * _normal(_gen(seed, 6), H))  # channels of different sizes
        s["x"] = (_normal(_gen(seed, 7), T, H) * spread).to(BF)
        s["base"] = _normal(_gen(seed, 8), T, H).to(BF) if case.get("base") else None
        s["out"] = torch.empty_like(s["x"])
    if kind == "tokens":
        s["y"] = _normal(_gen(seed, 9), R, H).to(BF)  # what the experts gave, or the gradient of what they took
        s["rows"] = torch.zeros(R, H, dtype=BF, device=DEV)  # rows between the experts' stay as they are
        s["d_y"], s["d_x"] = torch.zeros_like(s["rows"]), torch.empty_like(s["x"])
        s["d_rows"] = _normal(_gen(seed, 10), R, H).to(BF)
        s["d_weights"] = torch.empty(T, k, device=DEV)
    if kind == "experts":
        I = case["inner"]
        s["cap"] = max(1, int(np.bincount(idx[idx >= 0], minlength=E).max()))
        # gate and up rows in turn, 16 of each
        s["gate_up"] = _weight(seed, 1000, E, 2 * I, H, case["fmt"])
        s["down"] = _weight(seed, 5000, E, H, I, case["fmt"])
        # Static scales, as a calibration on other tokens gives them.
        s["g_x"] = 1.07 * s["x"].abs().amax().float().view(1) / 2688
        s["g_h"] = torch.full((E,), 20.0 / 2688, device=DEV) * torch.exp(0.2 * _normal(_gen(seed, 11), E))
    if own:
        from paper_2606_15682_gb300 import nvfp4 as N
        s["plan"] = N.MoEPlan(T, k, E)
        if kind != "route":
            N.moe_sort(s["plan"], s["idx"])
        if kind == "experts":
            sizes = N.nvfp4_scales_bytes if case["fmt"] == "nvfp4" else N.mxfp4_scales_bytes
            for name, cols in (("a", H), ("h", I)):
                s[name + "_codes"] = torch.empty(R, cols // 2, dtype=torch.uint8, device=DEV)
                s[name + "_scales"] = torch.empty(sizes(R, cols, N.SCALES_MMA), dtype=torch.uint8, device=DEV)
            s["y"] = torch.empty(R, H, dtype=BF, device=DEV)
    return s


# -------------------------------------------------------------------- run ---

def run(state):
    case = state["case"]
    if case["kind"] == "route":
        return (_own_route if own else _plain_route)(state, case)
    if case["kind"] == "tokens":
        return (_own_tokens if own else _plain_tokens)(state, case)
    return (_own_experts if own else _plain_experts)(state, case)


def _own_route(s, case):
    from paper_2606_15682_gb300 import nvfp4 as N
    score = N.MOE_SIGMOID if case["score"] == "sigmoid" else N.MOE_SOFTMAX
    if case["grad"]:
        N.moe_route_backward(s["logits"], s["idx"], s["d_weights"], s["d_logits"], score=score,
                             renormalize=case["renormalize"])
        return dict(d_logits=s["d_logits"])
    N.moe_route(s["logits"], s["out_idx"], s["out_weights"], score=score, renormalize=case["renormalize"], bias=s["bias"])
    N.moe_sort(s["plan"], s["out_idx"])
    p = s["plan"]
    return dict(idx=s["out_idx"], weights=s["out_weights"], row_of=p.row_of, rows=p.rows, row_start=p.row_start)


def _own_tokens(s, case):
    from paper_2606_15682_gb300 import nvfp4 as N
    p = s["plan"]
    if case["grad"]:
        N.moe_combine_backward(p, s["x"], s["y"], s["weights"], s["d_y"], s["d_weights"])
        N.moe_combine(p, s["d_rows"], s["d_x"])
        return dict(d_y=s["d_y"], d_weights=s["d_weights"], d_x=s["d_x"])
    N.moe_dispatch(p, s["x"], s["rows"])
    N.moe_combine(p, s["y"], s["out"], weights=s["weights"], base=s["base"])
    return dict(rows=s["rows"], out=s["out"])


def _own_experts(s, case):
    from paper_2606_15682_gb300 import nvfp4 as N
    p, H, I, up, down = s["plan"], case["hidden"], case["inner"], s["gate_up"], s["down"]
    N.moe_sort(p, s["idx"])
    if case["fmt"] == "nvfp4":
        N.moe_dispatch_nvfp4(p, s["x"], s["g_x"], s["a_codes"], s["a_scales"])
        N.nvfp4_linear_grouped_swiglu_quantize(p, s["a_codes"], s["a_scales"], s["g_x"], up["codes"], up["ordered"],
                                               up["g"], I, H, s["g_h"], s["h_codes"], s["h_scales"])
        N.nvfp4_linear_grouped(p, s["h_codes"], s["h_scales"], s["g_h"], down["codes"], down["ordered"], down["g"],
                               s["y"], H, I)
    else:
        N.moe_dispatch_mxfp4(p, s["x"], s["a_codes"], s["a_scales"])
        N.mxfp4_linear_grouped_swiglu_quantize(p, s["a_codes"], s["a_scales"], up["codes"], up["ordered"], I, H,
                                               s["h_codes"], s["h_scales"])
        N.mxfp4_linear_grouped(p, s["h_codes"], s["h_scales"], down["codes"], down["ordered"], s["y"], H, I)
    N.moe_combine(p, s["y"], s["out"], weights=s["weights"], base=s["base"])
    return dict(out=s["out"])


def _plain_scores(l, score):
    if score == "sigmoid":
        return torch.reciprocal(1 + torch.exp(-l))
    e = torch.exp(l - l.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_rows(idx, experts):
    """(row of each choice or -1, rows of each expert, first row of each expert and the end)."""
    flat = idx.flatten()
    rows = (flat[:, None] == torch.arange(experts, device=DEV)).sum(0)
    tiles = torch.div(rows + TILE - 1, TILE, rounding_mode="floor")
    start = torch.nn.functional.pad(torch.cumsum(tiles * TILE, 0), (1, 0))
    order = torch.argsort(torch.where(flat < 0, experts, flat), stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(len(flat), device=DEV)
    before = torch.nn.functional.pad(torch.cumsum(rows, 0), (1, 0))[:-1]
    e = flat.clamp(min=0).long()
    row_of = torch.where(flat < 0, -1, start[e] + place - before[e])
    return row_of.view(idx.shape).int(), rows.int(), start.int()


def _plain_route(s, case):
    l, k = s["logits"].float(), case["top_k"]
    p = _plain_scores(l, case["score"])
    if case["grad"]:
        at = s["idx"].long()
        chosen = torch.zeros_like(l).scatter_(1, at, 1.0)
        dw = torch.zeros_like(l).scatter_(1, at, s["d_weights"])
        if case["renormalize"]:
            total = (p * chosen).sum(1, keepdim=True)
            dp = chosen * (dw - (dw * p).sum(1, keepdim=True) / total) / total
        else:
            dp = dw
        if case["score"] == "sigmoid":
            d = dp * p * (1 - p)
        else:
            d = p * (dp - (dp * p).sum(1, keepdim=True))
        return dict(d_logits=d.to(s["logits"].dtype))
    key = l if s["bias"] is None else p + s["bias"]
    idx = torch.sort(key, dim=1, descending=True, stable=True)[1][:, :k]
    w = p.gather(1, idx)
    if case["renormalize"]:
        w = w / w.sum(1, keepdim=True)
    idx = idx.int()
    row_of, rows, start = _plain_rows(idx, case["experts"])
    return dict(idx=idx, weights=w, row_of=row_of, rows=rows, row_start=start)


def _plain_tokens(s, case):
    row_of, _, _ = _plain_rows(s["idx"], case["experts"])
    live = row_of >= 0
    at = row_of.long().clamp(min=0)
    if case["grad"]:
        g = s["x"].float()
        d_w = (g[:, None] * s["y"][at].float()).sum(-1) * live
        d_y = torch.zeros_like(s["rows"])
        d_y[at[live]] = (s["weights"][..., None] * g[:, None])[live].to(BF)
        d_x = (s["d_rows"][at].float() * live[..., None]).sum(1)
        return dict(d_y=d_y, d_weights=d_w, d_x=d_x.to(BF))
    rows = torch.zeros_like(s["rows"])
    rows[at[live]] = s["x"][:, None].expand(-1, case["top_k"], -1)[live]
    out = (s["y"][at].float() * (s["weights"] * live)[..., None]).sum(1)
    if s["base"] is not None:
        out = out + s["base"].float()
    return dict(rows=rows, out=out.to(BF))


def _plain_weight(w, fmt):
    """Elements times block scales [E, N, K] (without the tensor scale)."""
    pairs = torch.tensor([[0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6][n] for b in range(256)
                          for n in (b & 15, b >> 4)], device=DEV).view(256, 2)
    e = pairs[w["codes"].int()].flatten(-2)
    if fmt == "nvfp4":
        return (e.unflatten(-1, (-1, 16)) * w["scales"].view(torch.float8_e4m3fn).float()[..., None]).flatten(-2)
    return (e.unflatten(-1, (-1, 32)) * torch.exp2(w["scales"].float() - 127)[..., None]).flatten(-2)


def _plain_operand(x, fmt, g):
    e, sc = _nvfp4(x, g) if fmt == "nvfp4" else _mxfp4(x)
    return (e * sc).flatten(-2)


def _plain_experts(s, case):
    E, k, cap, fmt = case["experts"], case["top_k"], s["cap"], case["fmt"]
    flat = s["idx"].flatten().long()
    row_of, _, start = _plain_rows(s["idx"], E)
    live = flat >= 0
    slot = (flat.clamp(min=0) * cap + row_of.flatten().long() - start[flat.clamp(min=0)].long())[live]
    token = torch.div(torch.arange(len(flat), device=DEV), k, rounding_mode="floor")[live]
    one = torch.ones(E, device=DEV)
    g_x, g_h = (s["g_x"], s["g_h"]) if fmt == "nvfp4" else (one[:1], one)
    a = torch.zeros(E * cap, case["hidden"], device=DEV)
    a[slot] = _plain_operand(s["x"], fmt, g_x)[token]
    gu = torch.matmul(a.view(E, cap, -1), _plain_weight(s["gate_up"], fmt).transpose(1, 2))
    gu = (gu * (g_x * s["gate_up"]["g"])[:, None, None]).unflatten(-1, (-1, 2, 16))
    gate, up = gu[..., 0, :].flatten(-2), gu[..., 1, :].flatten(-2)
    h = _plain_operand(gate / (1 + torch.exp(-gate)) * up, fmt, g_h[:, None, None, None])
    y = torch.matmul(h, _plain_weight(s["down"], fmt).transpose(1, 2)) * (g_h * s["down"]["g"])[:, None, None]
    out = torch.zeros(len(flat), case["hidden"], device=DEV)
    out[live] = y.view(E * cap, -1)[slot] * s["weights"].flatten()[live, None]
    out = out.view(-1, k, case["hidden"]).sum(1)
    if s["base"] is not None:
        out = out + s["base"].float()
    return dict(out=out.to(BF))


# ------------------------------------------------------------------- work ---

@functools.lru_cache(maxsize=64)
def _asked(items):
    """(choices, experts that have any) of a case's inputs with seed 0."""
    idx = _choices(dict(items), 0)
    return int((idx >= 0).sum()), int(len(np.unique(idx[idx >= 0])))


def work(case):
    T, E, k = case["tokens"], case["experts"], case["top_k"]
    if case["kind"] == "route":
        size = 2 if case["bf16"] else 4
        if case["grad"]:
            return dict(bytes=T * (2 * E * size + 8 * k), flops=0)
        return dict(bytes=T * (E * size + 12 * k) + 8 * E + 4 * E * case["bias"], flops=0)
    pairs, touched = _asked(tuple(sorted((a, b) for a, b in case.items() if a != "name")))
    H = case["hidden"]
    if case["kind"] == "tokens":
        if case["grad"]:
            return dict(bytes=2 * H * (2 * T + 3 * pairs) + 12 * T * k, flops=0)
        return dict(bytes=2 * H * (T * (2 + case["base"]) + 2 * pairs) + 8 * T * k, flops=0)
    I = case["inner"]
    scale = 1 / 16 if case["fmt"] == "nvfp4" else 1 / 32
    return dict(bytes=int(touched * 3 * H * I * (0.5 + scale)) + 2 * H * T * (2 + case["base"]) + 8 * T * k,
                flops=6 * pairs * H * I)


# ------------------------------------------------------- the same in 64 bits ---

def _exact_route(s, case):
    T, k = case["tokens"], case["top_k"]
    l = s["logits"].double()
    top = l.max(1, keepdim=True)[0]
    soft = torch.exp(l - top)
    p = torch.sigmoid(l) if case["score"] == "sigmoid" else soft / soft.sum(1, keepdim=True)
    if case["grad"]:
        idx = s["idx"].long()
        row = torch.arange(T, device=DEV)[:, None].expand(-1, k)
        w, d = p[row, idx], s["d_weights"].double()
        if case["renormalize"]:
            total = w.sum(1, keepdim=True)
            d = d / total - (d * w).sum(1, keepdim=True) / total ** 2
        out = torch.zeros_like(l)
        if case["score"] == "sigmoid":
            out[row, idx] = d * w * (1 - w)
        else:
            out -= p * (d * w).sum(1, keepdim=True)
            out[row, idx] += d * w
        return dict(d_logits=out)
    # Scores next to each other are told apart in 32 bits: that is the choice's definition.
    key = l.clone() if s["bias"] is None else ((1 / (1 + torch.exp(-s["logits"].float()))) + s["bias"]).double()
    w = torch.empty(T, k, dtype=torch.float64, device=DEV)
    for j in range(k):
        best = (key == key.max(1, keepdim=True)[0]).int().argmax(1)  # the first of equal ones
        w[:, j] = p[torch.arange(T, device=DEV), best]
        key[torch.arange(T, device=DEV), best] = -math.inf
    if case["renormalize"]:
        w = w / w.sum(1, keepdim=True)
    return dict(idx=None, weights=w, row_of=None, rows=None, row_start=None)


def _exact_places(idx, experts):
    """Per expert: (tokens, choices, first row) of its rows in order."""
    places, first = [], 0
    for e in range(experts):
        t, j = np.nonzero(idx == e)
        places.append((t, j, first))
        first += -(-len(t) // TILE) * TILE
    return places


def _exact_operand(x, fmt, g):
    """Elements times block scales of x, in 64 bits."""
    n = 16 if fmt == "nvfp4" else 32
    b = x.reshape(*x.shape[:-1], -1, n)
    top = b.abs().max(-1, keepdim=True)[0]
    if fmt == "nvfp4":
        sc = (top / (6 * g)).clamp(max=448)
        step = torch.exp2(torch.floor(torch.log2(sc.clamp(min=2.0 ** -6))) - 3)
        sc = torch.round(sc / step) * step
        a = b.abs() / (sc * g).clamp(min=1e-300)
    else:
        sc = torch.exp2(torch.frexp(top)[1].double() - 3)
        a = b.abs() / sc
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    a = (torch.round(a / step) * step).clamp(max=6)
    return (torch.where(sc > 0, a, torch.zeros_like(a)) * torch.sign(b) * sc).reshape(x.shape)


def _exact_weight(w, e, fmt):
    c = w["codes"][e].long()
    nib = torch.stack([c & 15, c >> 4], -1).flatten(1)
    m = nib & 7
    v = torch.where(m < 2, m.double() / 2, torch.ldexp(1 + (m & 1).double() / 2, (m >> 1) - 1))
    v = torch.where(nib > 7, -v, v)
    b = w["scales"][e].long()
    if fmt == "nvfp4":
        x, f = b >> 3, (b & 7).double()
        sc, n = torch.where(x == 0, f / 512, torch.ldexp(1 + f / 8, x - 7)), 16
    else:
        sc, n = torch.ldexp(torch.ones_like(b, dtype=torch.float64), b - 127), 32
    return v * sc.repeat_interleave(n, 1)


def exact(case, seed):
    if case["kind"] == "experts" and 6 * case["tokens"] * case["top_k"] * case["hidden"] * case["inner"] > 4e12:
        return None
    s = prepare(case, seed)
    if case["kind"] == "route":
        return _exact_route(s, case)
    places = _exact_places(s["idx"].cpu().numpy(), case["experts"])
    w = s["weights"].double()
    x = s["x"].double()
    out = torch.zeros_like(x) if s["base"] is None else s["base"].double()
    if case["kind"] == "tokens":
        rows, d_y = (torch.zeros(s["rows"].shape, dtype=torch.float64, device=DEV) for _ in range(2))
        d_x, d_w = torch.zeros_like(x), torch.zeros_like(w)
        for t, j, first in places:
            t, j = torch.as_tensor(t, device=DEV), torch.as_tensor(j, device=DEV)
            at = slice(first, first + len(t))
            rows[at] = x[t]
            out.index_put_((t,), w[t, j, None] * s["y"][at].double(), accumulate=True)
            d_y[at] = w[t, j, None] * x[t]
            d_w[t, j] = (x[t] * s["y"][at].double()).sum(1)
            d_x.index_put_((t,), s["d_rows"][at].double(), accumulate=True)
        return dict(d_y=d_y, d_weights=d_w, d_x=d_x) if case["grad"] else dict(rows=rows, out=out)
    fmt = case["fmt"]
    scaled = fmt == "nvfp4"
    g_x = float(s["g_x"]) if scaled else 1.0
    xq = _exact_operand(x, fmt, g_x)
    for e, (t, j, _) in enumerate(places):
        if not len(t):
            continue
        t, j = torch.as_tensor(t, device=DEV), torch.as_tensor(j, device=DEV)
        gu = xq[t] @ _exact_weight(s["gate_up"], e, fmt).T * (g_x * float(s["gate_up"]["g"][e]) if scaled else 1.0)
        gu = gu.view(len(t), -1, 32)
        gate, up = gu[..., :16].reshape(len(t), -1), gu[..., 16:].reshape(len(t), -1)
        g_h = float(s["g_h"][e]) if scaled else 1.0
        h = _exact_operand(gate * torch.sigmoid(gate) * up, fmt, g_h)
        y = h @ _exact_weight(s["down"], e, fmt).T * (g_h * float(s["down"]["g"][e]) if scaled else 1.0)
        out.index_put_((t,), w[t, j, None] * y, accumulate=True)
    return dict(out=out)
