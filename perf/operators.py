"""The operators around a W4A4KV4 layer's linears, as a server calls them, and the same in plain torch.

  attention   extend_attention_nvfp4: new tokens (one, a few, a chunk, a whole prompt) over the 4-bit cache,
              contiguous or paged, with a logit cap, a distance bias, a window, documents or a prefix
  append      kv_append_rope_axes_nvfp4: rotary positions with several axes on Q and K, K and V quantized
              into the cache; the rows are then read back with kv_read_nvfp4
  read        kv_read_nvfp4: cached rows as bf16
  norm        residual_norm_nvfp4: norm of a block's output, gate, residual add, norm of the next block's input

listed() names twelve cases, draw() gives more of the same ranges.  Head layouts and widths are those of
paper_2606_15682_gb300/synth.py (12 on 2, 40 on 8, 64 on 8 heads; 1536 and 5120 channels).  `run` computes the
plain form in 32 bits, or calls the framework where `own` is true.
"""
import math
import random

import numpy as np
import torch

own = False
DEV = "cuda"
D = 128
SOFTMAX = 1.0 / math.sqrt(D)
GK, GV = 0.02, 0.015  # static scales of the cache
EPS = 1e-6


# ------------------------------------------------------------------ cases ---

def _attention(name, batch, heads, kv_heads, context, new, page=0, kv="e2m1", ragged=False, cap=0.0, window=0,
               bias=False, prefix=0, docs=0):
    return dict(name=name, kind="attention", batch=batch, heads=heads, kv_heads=kv_heads, context=context, new=new,
                page=page, kv=kv, ragged=ragged, cap=cap, window=window, bias=bias, prefix=prefix, docs=docs)


def listed():
    return [
        # One short sequence on a small model, one new token: latency only.
        _attention("attn_one_token_t700", 1, 12, 2, 700, 1, page=16),
        # The decode batch of a reasoning server: 64 ragged sequences of up to 16384 tokens in a paged cache.
        _attention("attn_decode_b64_t16384", 64, 40, 8, 16384, 1, page=64, ragged=True),
        # Four drafted tokens verified per sequence, E1M2 cache, scores with a distance bias.
        _attention("attn_verify_b32_n4", 32, 40, 8, 4001, 4, page=128, kv="e1m2", bias=True),
        # A whole prompt, causal.
        _attention("attn_prompt_n4096", 1, 40, 8, 4096, 4096),
        # A chunk of a long prompt on the largest head layout, capped scores, paged cache.
        _attention("attn_chunk_n2048_t16384", 1, 64, 8, 16384, 2048, page=64, cap=50.0),
        # Ragged prompts of packed documents with a sliding window and a shared prefix.
        _attention("attn_documents_b6_n1500", 6, 12, 2, 1500, 1500, page=48, ragged=True, window=512, prefix=64, docs=4),
        # A decode step's rotation and append for 64 sequences.
        dict(name="append_decode_b64", kind="append", batch=64, heads=40, kv_heads=8, new=1, context=2048, axes=1,
             page=64, kv="e2m1", shift=True),
        # A prompt with images: three rotary axes, Q, K and V cut from one projection's output.
        dict(name="append_images_n8192", kind="append", batch=1, heads=64, kv_heads=8, new=8192, context=8192, axes=3,
             page=0, kv="e2m1", shift=False),
        # One sequence's cache read back.
        dict(name="read_b1_t1000", kind="read", batch=1, kv_heads=2, context=1000, page=16, kv="e1m2"),
        # A batch's cache read back, for a transfer or a re-quantization.
        dict(name="read_b32_t4096", kind="read", batch=32, kv_heads=8, context=4096, page=64, kv="e2m1"),
        # Between two blocks of a decode step.
        dict(name="norm_m32_h5120", kind="norm", rows=32, hidden=5120, post=False, gate=0, alpha=1.0),
        # Between two blocks of a long prompt, norms on both sides, a gate per sequence, a residual scale.
        dict(name="norm_m8192_h5120", kind="norm", rows=8192, hidden=5120, post=True, gate=2048, alpha=0.5),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = ((12, 2), (40, 8), (64, 8), (8, 8), (16, 2))


def draw(rng):
    kind = rng.choice(["attention", "attention", "attention", "append", "read", "norm"])
    heads, kv_heads = rng.choice(HEADS)
    page = rng.choice([0, 16, 37, 64, 128])
    kv = rng.choice(["e2m1", "e2m1", "e1m2"])
    if kind == "attention":
        form = rng.choice(["decode", "few", "chunk", "prompt"])
        if form == "decode":
            batch, context, new = _log(rng, 1, 64), _log(rng, 20, 12000), 1
        elif form == "few":
            batch, context, new = _log(rng, 1, 32), _log(rng, 50, 6000), rng.randint(2, 16)
        elif form == "chunk":
            batch, context, new = rng.randint(1, 3), _log(rng, 500, 6000), _log(rng, 17, 500)
        else:
            batch, context, new = rng.randint(1, 4), _log(rng, 20, 2500), 0
            new = context
        c = _attention("", batch, heads, kv_heads, context, new, page=page, kv=kv, ragged=rng.random() < 0.6,
                       cap=rng.choice([0.0, 0.0, 30.0]), window=rng.choice([0, 0, _log(rng, 16, 2000)]),
                       bias=rng.random() < 0.3, prefix=rng.choice([0, 0, _log(rng, 4, 400)]),
                       docs=rng.choice([0, 0, rng.randint(2, 5)]))
        del c["name"]
        return c
    if kind == "append":
        new = rng.choice([1, _log(rng, 2, 6000)])
        return dict(kind="append", batch=_log(rng, 1, 64) if new == 1 else 1, heads=heads, kv_heads=kv_heads, new=new,
                    context=new + rng.randint(0, 500), axes=rng.randint(1, 3), page=page, kv=kv,
                    shift=rng.random() < 0.5)
    if kind == "read":
        return dict(kind="read", batch=_log(rng, 1, 32), kv_heads=kv_heads, context=_log(rng, 1, 4000), page=page, kv=kv)
    return dict(kind="norm", rows=_log(rng, 1, 8000), hidden=rng.choice([512, 1536, 2048, 5120, 8192]),
                post=rng.random() < 0.5, gate=rng.choice([0, 1, _log(rng, 1, 3000)]), alpha=rng.choice([1.0, 0.22]))


def _rng(case, salt):
    return random.Random("%s %s" % (salt, sorted((k, v) for k, v in case.items() if k != "name")))


def _lens(case):
    """Cached tokens of each sequence, the new ones among them."""
    if not case.get("ragged"):
        return [case["context"]] * case["batch"]
    rng = _rng(case, "lens")
    return [case["context"]] + [_log(rng, max(1, case["context"] // 8), case["context"]) for _ in range(case["batch"] - 1)]


def _news(case):
    """New tokens of each sequence: whole prompts, chunks of different sizes, or the same few for each."""
    lens = _lens(case)
    if case["new"] == case["context"]:
        return lens
    if not case["ragged"] or case["new"] <= 16:
        return [min(case["new"], min(lens))] * case["batch"]
    rng = _rng(case, "news")
    return [min(n, case["new"] if b == 0 else rng.randint(1, case["new"])) for b, n in enumerate(lens)]


def _visible(case):
    """(sequence, position, lo, hi) arrays of the query tokens: query i sees cached tokens lo..hi-1."""
    rng = _rng(case, "docs")
    seq, pos, doc = [], [], []
    for b, (n, new) in enumerate(zip(_lens(case), _news(case))):
        p = np.arange(n - new, n)
        cuts = np.array([0] + sorted(rng.randint(0, n) for _ in range(case["docs"] - 1))) if case["docs"] else np.array([0])
        seq.append(np.full(new, b))
        pos.append(p)
        doc.append(cuts[np.searchsorted(cuts, p, side="right") - 1])
    seq, pos, doc = (np.concatenate(v) for v in (seq, pos, doc))
    lo = np.maximum(doc, pos + 1 - case["window"]) if case["window"] else doc
    lo = np.maximum(lo, 0)
    hi = np.maximum(pos + 1, np.minimum(case["prefix"], np.array(_lens(case))[seq]))
    return seq, pos, doc, lo, np.maximum(hi, lo)


# ---------------------------------------------------------------- prepare ---

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * (seed + 1) + salt)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _keys(seed, salt, n, heads, spread):
    """bf16 [n, heads, 128], N(0, 1) times a lognormal factor of the head's channel."""
    f = torch.exp(spread * _normal(_gen(0, salt), heads, D))
    return (_normal(_gen(seed, salt), n, heads, D) * f).to(torch.bfloat16)


def _e4m3(s):
    return s.clamp(max=448.0).to(torch.float8_e4m3fn)


def _quantized(x, g, kv):
    """(element values, E4M3 block scales, both fp32) of x [..., 128] along its last axis, blocks of 16, in 32 bits."""
    b = x.float().unflatten(-1, (-1, 16))
    top = 3.5 if kv == "e1m2" else 6.0
    g = torch.tensor(g, dtype=torch.float32, device=x.device)
    s = _e4m3(b.abs().amax(-1, keepdim=True) / (g * top)).float()
    v = b * torch.where(s > 0, torch.reciprocal(s * g), torch.zeros_like(s))
    a = v.abs()
    if kv == "e1m2":
        a = torch.round(a * 2).clamp(max=7.0) * 0.5
    else:
        a = torch.where(a < 2, torch.round(a * 2) * 0.5, torch.where(a < 4, torch.round(a), torch.round(a * 0.5) * 2)).clamp(max=6.0)
    return torch.copysign(a, v), s


def _bytes(x, g, kv):
    """Cache bytes of x [..., 128]: (codes [..., 64], scales [..., 8])."""
    e, s = _quantized(x, g, kv)
    e = e.flatten(-2)
    if kv == "e1m2":
        nib = (e * 2).to(torch.int32) & 15
    else:
        a = e.abs()
        code = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a * 0.5 + 4))
        nib = code.to(torch.int32) | (torch.signbit(e).to(torch.int32) << 3)
    nib = nib.to(torch.uint8).unflatten(-1, (-1, 2))
    return nib[..., 0] | (nib[..., 1] << 4), s.squeeze(-1).to(torch.float8_e4m3fn).view(torch.uint8)


def _cache(case, seed, fill):
    """The cache's buffers [pages or sequences, heads, tokens, ...], its page table, lengths and slots by token."""
    B, HK, T, page = case["batch"], case["kv_heads"], case["context"], case["page"]
    per = -(-T // page) if page else 1
    size = page or T
    rows = B * per
    c = dict(kv=case["kv"], size=size, rows=rows, per=per)
    for i, (name, g) in enumerate((("k", GK), ("v", GV))):
        if fill:
            parts = [_bytes(_keys(seed, 10 * r + i + 1, n * size, HK, 1.0 if name == "k" else 0.5).unflatten(0, (n, size)).transpose(1, 2),
                            g, case["kv"])
                     for r in range(0, rows, max(1, (1 << 20) // (size * HK)))
                     for n in [min(rows - r, max(1, (1 << 20) // (size * HK)))]]
            c[name + "_codes"], c[name + "_scales"] = (torch.cat(p).contiguous() for p in zip(*parts))
        else:
            c[name + "_codes"] = torch.zeros(rows, HK, size, D // 2, dtype=torch.uint8, device=DEV)
            c[name + "_scales"] = torch.zeros(rows, HK, size, D // 16, dtype=torch.uint8, device=DEV)
    c["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device=DEV)
    if page:
        order = torch.randperm(rows, generator=_gen(seed, 7), device=DEV)
        c["table"] = order.to(torch.int32).view(B, per)
    else:
        c["table"] = None
    if own:  # the framework's handles on the same buffers
        from paper_2606_15682_gb300 import nvfp4 as N
        h = N.KVCache(1, HK, 2, GK, GV, kv_format=N.KV_E1M2 if case["kv"] == "e1m2" else N.KV_E2M1)
        h.batch, h.capacity, h.seq_lens = rows, size, c["lens"]
        h.k_codes, h.k_scales, h.v_codes, h.v_scales = c["k_codes"], c["k_scales"], c["v_codes"], c["v_scales"]
        c["handle"] = h
        c["pages"] = N.KVPages(c["table"], c["lens"]) if page else None
    return c


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), device=DEV).to(torch.int32)


def _rope_table(n):
    inv = torch.pow(torch.tensor(1e6, dtype=torch.float64, device=DEV), -torch.arange(64, device=DEV, dtype=torch.float64) / 64)
    a = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * inv
    return torch.stack([a.cos(), a.sin()], -1).float()


def _axis_of_pair(axes):
    """The rotary axis of each of the 64 channel pairs: 16 of time, then 24 of height and 24 of width."""
    return [0] * 64 if axes == 1 else [0] * 40 + [1] * 24 if axes == 2 else [0] * 16 + [1] * 24 + [2] * 24


def prepare(case, seed):
    kind = case["kind"]
    s = dict(case=case)
    bf = torch.bfloat16
    if kind == "norm":
        R, H = case["rows"], case["hidden"]
        g = _gen(seed, 1)
        spread = torch.exp(0.7 * _normal(g, H))  # channels of different sizes, as residual streams have
        s["x"] = (_normal(g, R, H) * spread * 4).to(bf)
        s["y"] = (_normal(g, R, H) * spread).to(bf)
        s["w"], s["w_post"] = ((1 + 0.2 * _normal(g, H)).to(bf) for _ in range(2))
        s["gate"] = (1 + 0.3 * _normal(g, -(-R // case["gate"]), H)).to(bf) if case["gate"] else None
        s["r"], s["h"] = torch.empty_like(s["x"]), torch.empty_like(s["x"])
        return s
    if kind == "read":
        s["cache"] = _cache(case, seed, True)
        t = np.arange(case["context"])
        s["seq"], s["pos"] = _i32(np.repeat(np.arange(case["batch"]), len(t))), _i32(np.tile(t, case["batch"]))
        s["k"] = torch.empty(len(s["seq"]), case["kv_heads"], D, dtype=bf, device=DEV)
        s["v"] = torch.empty_like(s["k"])
        return s
    H, HK, B = case["heads"], case["kv_heads"], case["batch"]
    if kind == "append":
        n, T = case["new"], case["context"]
        s["cache"] = _cache(case, seed, False)
        qkv = torch.cat([_keys(seed, 1, B * n, H, 0.2), _keys(seed, 2, B * n, HK, 1.0), _keys(seed, 3, B * n, HK, 0.5)], 1)
        s["qkv"] = qkv.view(B * n, -1)
        t = np.tile(np.arange(T - n, T), B)
        s["seq"], s["pos"] = _i32(np.repeat(np.arange(B), n)), _i32(t)
        # Images of 32 x 32 patches: one time step each, rows and columns counted from it.
        base = t // 1024 * 32
        r = np.stack([base if case["axes"] > 1 else t, base + t // 32 % 32, base + t % 32], 1)[:, :case["axes"]]
        s["rope_pos"] = _i32(r)
        s["axis_of_pair"] = _axis_of_pair(case["axes"])
        s["axis"] = torch.tensor(s["axis_of_pair"], device=DEV)
        s["table"] = _rope_table(max(T, int(r.max()) + 1))
        s["shift"] = 0.5 * _normal(_gen(0, 5), HK, D) if case["shift"] else None
        s["q_out"] = torch.empty(B * n, H, D, dtype=bf, device=DEV)
        s["k"] = torch.empty(B * n, HK, D, dtype=bf, device=DEV)
        s["v"] = torch.empty_like(s["k"])
        return s
    s["cache"] = _cache(case, seed, True)
    seq, pos, doc, _, _ = _visible(case)
    s["q"] = _keys(seed, 4, len(seq), H, 0.1)
    s["seq"], s["pos"] = _i32(seq).long(), _i32(pos)
    news = _news(case)
    s["q_start"] = _i32(np.concatenate([[0], np.cumsum(news)])) if len(set(news)) > 1 else None
    s["doc_start"] = _i32(doc) if case["docs"] else None
    s["prefix"] = torch.full((B,), case["prefix"], dtype=torch.int32, device=DEV) if case["prefix"] else None
    s["slopes"] = torch.pow(2.0, -8.0 * torch.arange(1, H + 1, device=DEV, dtype=torch.float32) / H) if case["bias"] else None
    s["out"] = torch.empty_like(s["q"])
    if own:
        from paper_2606_15682_gb300 import nvfp4 as N
        c = s["cache"]
        nbytes = N.extend_attention_nvfp4_workspace_size(B, len(seq), H, HK, c["per"] * c["size"])
        s["ws"] = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    return s


# -------------------------------------------------------------------- run ---

def run(state):
    return (_run_own if own else _run_plain)(state)


def _qkv(s, case):
    return s["qkv"].view(-1, case["heads"] + 2 * case["kv_heads"], D).split([case["heads"], case["kv_heads"], case["kv_heads"]], 1)


def _run_own(s):
    from paper_2606_15682_gb300 import nvfp4 as N
    case = s["case"]
    if case["kind"] == "norm":
        N.residual_norm_nvfp4(s["x"], s["y"], s["r"], s["h"], s["w"], eps=EPS, w_post=s["w_post"] if case["post"] else None,
                              gate=s["gate"], rows_per_gate=case["gate"], alpha=case["alpha"])
        return dict(r=s["r"], h=s["h"])
    c = s["cache"]
    if case["kind"] == "read":
        N.kv_read_nvfp4(c["handle"], s["seq"], s["pos"], s["k"], s["v"], pages=c["pages"])
        return dict(k=s["k"], v=s["v"])
    if case["kind"] == "append":
        q, k, v = _qkv(s, case)
        N.kv_append_rope_axes_nvfp4(c["handle"], q, k, v, s["seq"], s["pos"], s["rope_pos"], s["axis_of_pair"], s["table"],
                                    s["q_out"], k_shift=s["shift"], pages=c["pages"])
        N.kv_read_nvfp4(c["handle"], s["seq"], s["pos"], s["k"], s["v"], pages=c["pages"])
        return dict(q=s["q_out"], k=s["k"], v=s["v"])
    N.extend_attention_nvfp4(c["handle"], s["q"], SOFTMAX, s["out"], s["ws"], q_start=s["q_start"], pages=c["pages"],
                             logit_cap=case["cap"], window=case["window"], slopes=s["slopes"], prefix_lens=s["prefix"],
                             doc_start=s["doc_start"])
    return dict(out=s["out"])


def _values(c, name, g, seq=None, pos=None):
    """fp32 values of the cache: [B, HK, T, 128] of all of it, or [n, HK, 128] of the rows (seq, pos)."""
    codes, scales = c[name + "_codes"], c[name + "_scales"]
    if seq is not None:
        seq, pos = seq.long(), pos.long()
        row, at = (c["table"][seq, pos // c["size"]].long(), pos % c["size"]) if c["table"] is not None else (seq, pos)
        codes, scales = codes[row, :, at], scales[row, :, at]
    elif c["table"] is not None:
        codes, scales = (t[c["table"].long()].transpose(1, 2).flatten(2, 3) for t in (codes, scales))
    if c["kv"] == "e1m2":
        grid = [n / 2 - (8 if n > 7 else 0) for n in range(16)]
    else:
        grid = [0, .5, 1, 1.5, 2, 3, 4, 6]
        grid += [-v for v in grid]
    pairs = torch.tensor([[grid[b & 15], grid[b >> 4]] for b in range(256)], device=codes.device)
    e = pairs[codes.int()].flatten(-2).unflatten(-1, (-1, 16))
    return (e * scales.view(torch.float8_e4m3fn).float()[..., None] * g).flatten(-2)


def _rotated(x, s):
    cs = s["table"][s["rope_pos"].long()[:, s["axis"]], torch.arange(64, device=DEV)]  # [n, 64, 2]
    c, d = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = x[..., :64].float(), x[..., 64:].float()
    return torch.cat([a * c - b * d, a * d + b * c], -1)


def _run_plain(s):
    case, bf = s["case"], torch.bfloat16
    if case["kind"] == "norm":
        x, z = s["x"].float(), s["y"].float()
        if case["post"]:
            z = z * torch.rsqrt((z * z).mean(-1, keepdim=True) + EPS) * s["w_post"].float()
        if case["gate"]:
            z = z * s["gate"].float().repeat_interleave(case["gate"], 0)[:len(z)]
        r = x + case["alpha"] * z
        h = r * torch.rsqrt((r * r).mean(-1, keepdim=True) + EPS) * s["w"].float()
        return dict(r=r.to(bf), h=h.to(bf))
    if case["kind"] == "read":
        return {n: _values(s["cache"], n, g, s["seq"], s["pos"]).to(bf) for n, g in (("k", GK), ("v", GV))}
    if case["kind"] == "append":
        q, k, v = _qkv(s, case)
        k = _rotated(k, s)
        if case["shift"]:
            k = k - s["shift"]
        got = dict(q=_rotated(q, s).to(bf))
        for name, x, g in (("k", k, GK), ("v", v, GV)):
            e, sc = _quantized(x, g, case["kv"])
            got[name] = (e * sc * g).flatten(-2).to(bf)
        return got
    return dict(out=_plain_attention(s, case))


def _plain_attention(s, case):
    c, B, H, HK = s["cache"], case["batch"], case["heads"], case["kv_heads"]
    k, v = _values(c, "k", GK), _values(c, "v", GV)  # [B, HK, T, 128]
    T, G = k.shape[2], H // HK
    # Queries padded to the longest sequence's: [B, new, ...].
    n = max(_news(case))
    if s["q_start"] is None:
        at = torch.arange(B * n, device=DEV).view(B, n)
        live = torch.ones(B, n, dtype=torch.bool, device=DEV)
    else:
        start = s["q_start"].long()
        at = start[:-1, None] + torch.arange(n, device=DEV)
        live = at < start[1:, None]
        at = at.clamp(max=len(s["q"]) - 1)
    q = s["q"].float()[at].view(B, n, HK, G, D).permute(0, 2, 3, 1, 4).reshape(B, HK, G * n, D)
    w = torch.matmul(q, k.transpose(-1, -2)).view(B, HK, G, n, T).mul_(SOFTMAX)
    if case["cap"]:
        w.div_(case["cap"]).tanh_().mul_(case["cap"])
    t, p, lens = torch.arange(T, device=DEV), s["pos"].long()[at][..., None], c["lens"].long()[:, None, None]
    if case["bias"]:
        w -= s["slopes"].view(1, HK, G, 1, 1) * (p - t).abs().float()[:, None, None]
    hi = p + 1
    if case["prefix"]:
        hi = torch.maximum(hi, torch.minimum(s["prefix"].long()[:, None, None], lens))
    see = live[..., None] & (t < hi)
    if case["window"]:
        see = see & (t > p - case["window"])
    if case["docs"]:
        see = see & (t >= s["doc_start"].long()[at][..., None])
    see = see[:, None, None]
    w.masked_fill_(~see, -math.inf)
    w -= w.amax(-1, keepdim=True).clamp(min=-1e30)
    w.exp_()
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(B, HK, G * n, T), v).view(B, HK, G, n, D) / total.clamp(min=1e-30)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, H, D)
    out = torch.zeros(len(s["q"]), H, D, device=DEV)
    out[at[live]] = o[live]
    return out.to(torch.bfloat16)


# ------------------------------------------------------------------- work ---

ROW = D // 2 + D // 16  # cache bytes of a row


def work(case):
    kind = case["kind"]
    if kind == "norm":
        n = case["rows"] * case["hidden"]
        gate = -(-case["rows"] // case["gate"]) if case["gate"] else 0
        return dict(bytes=8 * n + 2 * case["hidden"] * (1 + case["post"] + gate), flops=0)
    if kind == "read":
        rows = case["batch"] * case["context"]
        return dict(bytes=rows * (2 * case["kv_heads"] * (ROW + 2 * D) + 8), flops=0)
    if kind == "append":
        n, HK = case["batch"] * case["new"], case["kv_heads"]
        append = n * (4 * case["heads"] * D + 2 * HK * (2 * D + ROW) + 8 + 4 * case["axes"])
        return dict(bytes=append + n * 2 * HK * (ROW + 2 * D), flops=0)
    seq, _, _, lo, hi = _visible(case)
    read = 0
    for b in range(case["batch"]):
        edge = np.zeros(case["context"] + 1, dtype=np.int64)
        np.add.at(edge, lo[seq == b], 1)
        np.add.at(edge, hi[seq == b], -1)
        read += int((np.cumsum(edge) > 0).sum())
    return dict(bytes=2 * read * case["kv_heads"] * ROW + 4 * len(seq) * case["heads"] * D,
                flops=4 * D * case["heads"] * int((hi - lo).sum()))


# ------------------------------------------------------- the same in 64 bits ---

def _exact_rows(c, name, b, head, g):
    """Sequence b's cached rows of one head, [T, 128] in 64 bits."""
    if c["table"] is None:
        codes, scales = c[name + "_codes"][b, head], c[name + "_scales"][b, head]
    else:
        pages = c["table"][b].long()
        codes = c[name + "_codes"][pages, head].reshape(-1, D // 2)
        scales = c[name + "_scales"][pages, head].reshape(-1, D // 16)
    nib = torch.stack([codes & 15, codes >> 4], -1).flatten(1).long()
    if c["kv"] == "e1m2":
        e = torch.where(nib > 7, nib - 16, nib).double() / 2
    else:
        m, sign = nib & 7, torch.where(nib > 7, -1.0, 1.0).double()
        # exponent (m >> 1) with bias 1, one bit of fraction; exponent 0 is m / 2
        e = sign * torch.where(m < 2, m.double() / 2, torch.ldexp(1 + (m & 1).double() / 2, (m >> 1) - 1))
    b8 = scales.long()
    x, f = b8 >> 3, (b8 & 7).double()
    sc = torch.where(x == 0, f / 512, torch.ldexp(1 + f / 8, x - 7))
    return e * sc.repeat_interleave(16, 1) * float(np.float32(g))


def _exact_quantized(x, g, kv):
    """x [n, heads, 128] in 64 bits -> the values that its codes and scales stand for."""
    g, top = float(np.float32(g)), 3.5 if kv == "e1m2" else 6.0
    b = x.reshape(*x.shape[:-1], 8, 16)
    s = (b.abs().amax(-1, keepdim=True) / (g * top)).clamp(max=448)
    step = torch.ldexp(torch.ones_like(s), torch.floor(torch.log2(s.clamp(min=2.0 ** -6))).long() - 3)
    s = torch.round(s / step) * step
    a = b.abs() / (s * g).clamp(min=1e-300)
    if kv == "e1m2":
        a = torch.round(2 * a).clamp(max=7) / 2
    else:
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
        a = (torch.round(a / step) * step).clamp(max=6)
    a = torch.where(s > 0, a, torch.zeros_like(a))
    return (a * torch.sign(b) * s * g).reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        R = case["rows"]
        x, z = s["x"].double(), s["y"].double()
        if case["post"]:
            z = z / torch.sqrt(z.square().sum(1, keepdim=True) / case["hidden"] + EPS) * s["w_post"].double()
        if case["gate"]:
            z = z * s["gate"].double()[torch.arange(R, device=DEV) // case["gate"]]
        r = x + case["alpha"] * z
        return dict(r=r, h=r / torch.sqrt(r.square().sum(1, keepdim=True) / case["hidden"] + EPS) * s["w"].double())
    if kind == "read":
        B, HK, T = case["batch"], case["kv_heads"], case["context"]
        got = {}
        for name, g in (("k", GK), ("v", GV)):
            out = torch.empty(B, T, HK, D, dtype=torch.float64, device=DEV)
            for b in range(B):
                for h in range(HK):
                    out[b, :, h] = _exact_rows(s["cache"], name, b, h, g)[:T]
            got[name] = out.view(B * T, HK, D)
        return got
    if kind == "append":
        H, HK = case["heads"], case["kv_heads"]
        x = s["qkv"].double().view(-1, H + 2 * HK, D)
        C, S = (torch.empty(len(x), 64, dtype=torch.float64, device=DEV) for _ in range(2))
        for pair in range(64):
            row = s["table"][s["rope_pos"][:, s["axis_of_pair"][pair]].long(), pair].double()
            C[:, pair], S[:, pair] = row[:, 0], row[:, 1]
        lo, hi = x[:, :H + HK, :64], x[:, :H + HK, 64:]
        y = torch.cat([lo * C[:, None] - hi * S[:, None], hi * C[:, None] + lo * S[:, None]], 2)
        k = y[:, H:] - (s["shift"].double() if case["shift"] else 0)
        return dict(q=y[:, :H], k=_exact_quantized(k, GK, case["kv"]), v=_exact_quantized(x[:, H + HK:], GV, case["kv"]))
    if 4 * D * case["heads"] * case["batch"] * max(_news(case)) * case["context"] > 4e12:
        return None
    seq, pos, _, lo, hi = _visible(case)
    B, H, HK = case["batch"], case["heads"], case["kv_heads"]
    G = H // HK
    out = torch.zeros(len(seq), H, D, dtype=torch.float64, device=DEV)
    for b in range(B):
        rows = np.nonzero(seq == b)[0]
        for head in range(HK):
            k, v = (_exact_rows(s["cache"], n, b, head, g) for n, g in (("k", GK), ("v", GV)))
            for at in np.array_split(rows, -(-len(rows) // 512)):
                i = torch.as_tensor(at, device=DEV)
                left, right, p = (torch.as_tensor(a[at], device=DEV)[:, None] for a in (lo, hi, pos))
                t = torch.arange(len(k), device=DEV)
                hide = (t < left) | (t >= right)
                for gq in range(G):
                    h = head * G + gq
                    z = s["q"][i, h].double() @ k.T / math.sqrt(D)
                    if case["cap"]:
                        z = case["cap"] * torch.tanh(z / case["cap"])
                    if case["bias"]:
                        z = z - s["slopes"][h].double() * (t - p).abs()
                    z = z.masked_fill(hide, -math.inf)
                    z = torch.exp(z - z.amax(1, keepdim=True).clamp(min=-1e300))
                    out[i, h] = z @ v / z.sum(1, keepdim=True).clamp(min=1e-300)
    return dict(out=out)
