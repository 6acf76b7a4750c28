"""W4A4KV4 layers that serve sequences from a paged 4-bit cache: prompts, chunks of prompts, drafted tokens and
single tokens all take the same path.

    python -m paper_2606_15682_gb300.serve --batch 8 --prompt 1500 --chunk 512 --steps 32

A layer's step for n new tokens, every line one call of the library:

    residual_norm_nvfp4           x (+ the last layer's output) and the norm, as qkv's NVFP4 input
    nvfp4_linear                  qkv
    kv_append_rope_axes_nvfp4     rotated Q, quantized K and V into the sequences' pages
    extend_attention_nvfp4        the new tokens over their sequences' caches
    nvfp4_quantize, nvfp4_linear  o
    residual_norm_nvfp4           the residual sum and the norm, as gate_up's NVFP4 input
    nvfp4_linear_swiglu_quantize  gate_up, SwiGLU, down's NVFP4 input
    nvfp4_linear                  down

or, in a layer of experts (--experts 64 --top-k 8), in place of the last two:

    nvfp4_linear, moe_route       the router's logits; each token's experts and their weights
    moe_sort, moe_dispatch_nvfp4  the tokens' rows by expert, and the norm's output quantized into them
    nvfp4_linear_grouped_swiglu_quantize, nvfp4_linear_grouped  the experts' gate_up and down
    moe_combine                   the rows back to their tokens, weighted and summed

Buffers are allocated for a Batch of `n_new` tokens per sequence once and reused by all its steps; a step
reads nothing back, so a decode step is captured in a CUDA graph and replayed.  Weights here are seeded random
ones; the static activation scales are arguments, as a calibration would give them.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import build as _build

_build.build()
from . import nvfp4 as N  # noqa: E402

D = 128


def _quantize_weight(w, codes, scales, g):
    N.nvfp4_tensor_scale(w, g)
    N.nvfp4_quantize(w, g, codes, scales, N.SCALES_MMA)


def _quantized_weight(w):
    g = torch.empty(1, dtype=torch.float32, device=w.device)
    codes = torch.empty(w.shape[0], w.shape[1] // 2, dtype=torch.uint8, device=w.device)
    scales = torch.empty(N.nvfp4_scales_bytes(*w.shape, N.SCALES_MMA), dtype=torch.uint8, device=w.device)
    _quantize_weight(w, codes, scales, g)
    return codes, scales, g


def _gate_up(gate, up):
    both = torch.empty(2 * gate.shape[0], gate.shape[1], dtype=torch.bfloat16, device=gate.device)
    N.nvfp4_interleave_gate_up(gate, up, both)
    return both


def _quantized_experts(experts, rows, cols, device):
    """Codes, scales and tensor scales of the experts' weights [rows, cols], one after another."""
    E = len(experts)
    codes = torch.empty(E, rows, cols // 2, dtype=torch.uint8, device=device)
    scales = torch.empty(E, N.nvfp4_scales_bytes(rows, cols, N.SCALES_MMA), dtype=torch.uint8, device=device)
    g = torch.empty(E, dtype=torch.float32, device=device)
    for e, w in enumerate(experts):
        _quantize_weight(w, codes[e], scales[e], g[e:e + 1])
    return codes, scales, g


class Layer:
    """One layer's weights, quantized once, and its paged cache.

    weights: bf16 "qkv" [(hq + 2 hkv) * 128, H], "o" [H, hq * 128], "gate" and "up" [I, H], "down" [H, I], "norm1" and
    "norm2" [H]; act_scales: the static NVFP4 scales of the inputs of qkv, o, gate_up and down.  With "router" [E, H] (E a
    multiple of 16) gate, up and down have an expert as their first axis, and a token goes through top_k of them.
    """

    def __init__(self, weights, heads, kv_heads, pages, page, kv_scales, act_scales, kv_format=N.KV_E2M1, k_shift=None,
                 top_k=0):
        self.heads, self.kv_heads, self.top_k = heads, kv_heads, top_k
        self.hidden, self.inner = weights["o"].shape[0], weights["down"].shape[-1]
        dev = weights["gate"].device
        self.qkv, self.o = (_quantized_weight(weights[n]) for n in ("qkv", "o"))
        self.experts = weights["router"].shape[0] if "router" in weights else 0
        if not self.experts and top_k:
            raise ValueError("top_k without a router")
        if self.experts:
            if self.experts % 16 or not 1 <= top_k <= min(self.experts, 32):
                raise ValueError("experts must be a multiple of 16, top_k 1 to 32 of them")
            self.router = _quantized_weight(weights["router"])
            self.gate_up = _quantized_experts([_gate_up(*w) for w in zip(weights["gate"], weights["up"])],
                                              2 * self.inner, self.hidden, dev)
            self.down = _quantized_experts(weights["down"], self.hidden, self.inner, dev)
        else:
            self.gate_up, self.down = _quantized_weight(_gate_up(weights["gate"], weights["up"])), _quantized_weight(weights["down"])
        self.norm1, self.norm2, self.k_shift = weights["norm1"], weights["norm2"], k_shift
        self.cache = N.KVCache(pages, kv_heads, page, *kv_scales, device=dev, kv_format=kv_format)
        self.g = [torch.tensor([g], dtype=torch.float32, device=dev) for g in act_scales]


def _experts(layer):
    """(experts, top_k) of a layer; of one with an MLP, which need not know of experts, (0, 0)."""
    return getattr(layer, "experts", 0), getattr(layer, "top_k", 0)


class Batch:
    """n_new tokens of each of `batch` sequences on their way through the layers, and the buffers they need.

    table: int32 [batch, pages_per_seq], seq_lens: int32 [batch], both on the device and shared with other Batches of the
    same sequences; axis_of_pair: the rotary axis of each channel pair.
    """

    def __init__(self, layer, table, seq_lens, n_new, rope_table, axis_of_pair=bytes(64)):
        dev, n = table.device, table.shape[0] * n_new
        H, I, hq, hkv = layer.hidden, layer.inner, layer.heads, layer.kv_heads
        self.n, self.n_new = n, n_new
        self.pages = N.KVPages(table, seq_lens)
        self.rope_table, self.axis_of_pair = rope_table, axis_of_pair
        self.seq = torch.arange(table.shape[0], dtype=torch.int32, device=dev).repeat_interleave(n_new)
        self.step = torch.arange(n_new, dtype=torch.int32, device=dev).repeat(table.shape[0])
        self.pos = torch.zeros(n, dtype=torch.int32, device=dev)

        def bf16(*shape):
            return torch.empty(*shape, dtype=torch.bfloat16, device=dev)

        def fp4(rows, cols):
            return (torch.empty(rows, cols // 2, dtype=torch.uint8, device=dev),
                    torch.empty(N.nvfp4_scales_bytes(rows, cols, N.SCALES_MMA), dtype=torch.uint8, device=dev))

        self.qkv, self.q, self.attn = bf16(n, (hq + 2 * hkv) * D), bf16(n, hq, D), bf16(n, hq, D)
        self.r, self.o, self.y, self.h = bf16(n, H), bf16(n, H), bf16(n, H), bf16(n, H)
        self.a_qkv, self.a_o, self.a_gu = fp4(n, H), fp4(n, hq * D), fp4(n, H)
        self.experts = _experts(layer)
        if self.experts[0]:
            self.plan = N.MoEPlan(n, layer.top_k, layer.experts, device=dev)
            rows = self.plan.max_rows
            self.logits, self.h2 = bf16(n, layer.experts), bf16(n, H)
            self.expert_idx = torch.empty(n, layer.top_k, dtype=torch.int32, device=dev)
            self.expert_weights = torch.empty(n, layer.top_k, dtype=torch.float32, device=dev)
            self.a_rows, self.a_down, self.y_rows = fp4(rows, H), fp4(rows, I), bf16(rows, H)
        else:
            self.a_down = fp4(n, I)
        size = N.extend_attention_nvfp4_workspace_size(table.shape[0], n, hq, hkv,
                                                       table.shape[1] * layer.cache.capacity)
        self.workspace = torch.empty(size, dtype=torch.uint8, device=dev) if size else None

    def begin(self):
        """The new tokens join their sequences."""
        lens = self.pages.seq_lens
        torch.add(lens.repeat_interleave(self.n_new, output_size=self.n), self.step, out=self.pos)
        lens += self.n_new

    def run(self, layers, x, norm_out, rope_pos=None, logit_cap=0.0, window=0):
        """x [n, H] bf16 -> the last norm's output [n, H]; rope_pos [n, axes] int32 (None: the place in the sequence).

        A cap and a key shift exclude each other: the cache holds K - m, whose scores differ from K's by q.m.  A softmax
        does not see that, a cap does.
        """
        if logit_cap and any(w.k_shift is not None for w in layers):
            raise ValueError("logit_cap needs the keys themselves: a layer with k_shift caches K - m")
        if any(_experts(w) != self.experts for w in layers):
            raise ValueError("a Batch runs layers with the experts and top_k of the one that it was made for")
        self.begin()
        rope_pos = self.pos[:, None] if rope_pos is None else rope_pos
        r, y = x, None
        for w in layers:
            n, H, I, hq, hkv = self.n, w.hidden, w.inner, w.heads, w.kv_heads
            # y None: the first layer, whose residual stream is x itself.
            N.residual_norm_nvfp4(r, y, None if y is None else self.r, None, w.norm1, g_out=w.g[0], codes=self.a_qkv[0],
                                  scales=self.a_qkv[1])
            r = x if y is None else self.r
            N.nvfp4_linear(*self.a_qkv, w.g[0], *w.qkv, self.qkv, n, (hq + 2 * hkv) * D, H)
            q, k, v = self.qkv.view(n, hq + 2 * hkv, D).split([hq, hkv, hkv], 1)
            N.kv_append_rope_axes_nvfp4(w.cache, q, k, v, self.seq, self.pos, rope_pos, self.axis_of_pair,
                                        self.rope_table, self.q, k_shift=w.k_shift, pages=self.pages)
            N.extend_attention_nvfp4(w.cache, self.q, 1.0 / math.sqrt(D), self.attn, self.workspace, pages=self.pages,
                                     logit_cap=logit_cap, window=window)
            N.nvfp4_quantize(self.attn.view(n, hq * D), w.g[1], *self.a_o, N.SCALES_MMA)
            N.nvfp4_linear(*self.a_o, w.g[1], *w.o, self.o, n, H, hq * D)
            N.residual_norm_nvfp4(r, self.o, self.r, self.h2 if self.experts[0] else None, w.norm2, g_out=w.g[2],
                                  codes=self.a_gu[0], scales=self.a_gu[1])
            r = self.r
            if self.experts[0]:
                self.run_experts(w)
            else:
                N.nvfp4_linear_swiglu_quantize(*self.a_gu, w.g[2], *w.gate_up, n, I, H, w.g[3], *self.a_down)
                N.nvfp4_linear(*self.a_down, w.g[3], *w.down, self.y, n, H, I)
            y = self.y
        N.residual_norm_nvfp4(r, y, self.r, self.h, norm_out)
        return self.h

    def run_experts(self, w):
        """The norm's output (self.h2, and self.a_gu as NVFP4) through each token's experts -> self.y."""
        plan, I, H = self.plan, w.inner, w.hidden
        N.nvfp4_linear(*self.a_gu, w.g[2], *w.router, self.logits, self.n, w.experts, H)
        N.moe_route(self.logits, self.expert_idx, self.expert_weights)
        N.moe_sort(plan, self.expert_idx)
        N.moe_dispatch_nvfp4(plan, self.h2, w.g[2], *self.a_rows)
        N.nvfp4_linear_grouped_swiglu_quantize(plan, *self.a_rows, w.g[2], *w.gate_up, I, H, w.g[3], *self.a_down)
        N.nvfp4_linear_grouped(plan, *self.a_down, w.g[3], *w.down, self.y_rows, H, I)
        N.moe_combine(plan, self.y_rows, self.y, weights=self.expert_weights)

    def cached(self, layer, sequence, start, stop):
        """A layer's cached K and V of a sequence's tokens start .. stop-1, as bf16 [stop - start, kv heads, 128]."""
        dev = self.seq.device
        pos = torch.arange(start, stop, dtype=torch.int32, device=dev)
        k = torch.empty(stop - start, layer.kv_heads, D, dtype=torch.bfloat16, device=dev)
        v = torch.empty_like(k)
        N.kv_read_nvfp4(layer.cache, torch.full_like(pos, sequence), pos, k, v, pages=self.pages)
        return k, v


def random_layer(hidden, inner, heads, kv_heads, pages, page, seed, device="cuda", kv_format=N.KV_E2M1, experts=0,
                 top_k=0):
    """A layer of seeded random weights whose static scales fit inputs of unit size."""
    gen = torch.Generator(device=device).manual_seed(seed)

    def w(rows, cols):
        return (torch.randn(rows, cols, generator=gen, device=device) / math.sqrt(cols)).to(torch.bfloat16)

    def each(rows, cols):
        return [w(rows, cols) for _ in range(experts)]
    if experts:
        mlp = dict(router=w(experts, hidden) * 2, gate=torch.stack(each(inner, hidden)), up=torch.stack(each(inner, hidden)),
                   down=torch.stack(each(hidden, inner)))
    else:
        mlp = None
    weights = dict(qkv=w((heads + 2 * kv_heads) * D, hidden), o=w(hidden, heads * D),
                   **(mlp or dict(gate=w(inner, hidden), up=w(inner, hidden), down=w(hidden, inner))),
                   norm1=torch.ones(hidden, dtype=torch.bfloat16, device=device),
                   norm2=torch.ones(hidden, dtype=torch.bfloat16, device=device))
    # amax / (the format's largest element * 448) of a Gaussian activation, with room for its tail.
    unit, kv = 6.0 / (6 * 448), 6.0 / ((3.5 if kv_format == N.KV_E1M2 else 6) * 448)
    return weights, Layer(weights, heads, kv_heads, pages, page, (kv, kv), (unit, unit, unit, unit), kv_format,
                          top_k=top_k)


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=1500)
    ap.add_argument("--chunk", type=int, default=512)
    ap.add_argument("--steps", type=int, default=32)
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--page", type=int, default=64)
    ap.add_argument("--hidden", type=int, default=1536)
    ap.add_argument("--inner", type=int, default=8960)
    ap.add_argument("--heads", type=int, default=12)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--experts", type=int, default=0, help="experts a layer, a multiple of 16; 0: one MLP")
    ap.add_argument("--top-k", type=int, default=8, help="experts of a token")
    a = ap.parse_args()
    dev = torch.device("cuda", 0)
    torch.cuda.set_device(dev)
    top = a.prompt + a.steps + 2
    per = -(-top // a.page)
    layers = [random_layer(a.hidden, a.inner, a.heads, a.kv_heads, a.batch * per, a.page, seed, experts=a.experts,
                           top_k=min(a.top_k, a.experts))[1] for seed in range(a.layers)]
    gen = torch.Generator(device=dev).manual_seed(99)
    table = torch.randperm(a.batch * per, generator=gen, device=dev).to(torch.int32).view(a.batch, per)
    lens = torch.zeros(a.batch, dtype=torch.int32, device=dev)
    rope = torch.empty(top, D // 2, 2, dtype=torch.float32, device=dev)
    N.nvfp4_rope_table(rope)
    norm = torch.ones(a.hidden, dtype=torch.bfloat16, device=dev)
    prompt = torch.randn(a.batch, a.prompt, a.hidden, generator=gen, device=dev).to(torch.bfloat16)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))

    def prefill():
        lens.zero_()
        for t in range(0, a.prompt, a.chunk):
            x = prompt[:, t:t + a.chunk].reshape(-1, a.hidden)
            h = batches[x.shape[0] // a.batch].run(layers, x, norm)
        return h
    batches = {n: Batch(layers[0], table, lens, n, rope) for n in {min(a.chunk, a.prompt), a.prompt % a.chunk or 1, 1}}
    prefill()  # warm-up
    torch.cuda.synchronize()
    start.record()
    h = prefill()
    end.record()
    torch.cuda.synchronize()
    ms = start.elapsed_time(end)
    print(f"prompts: {a.batch} x {a.prompt} tokens in chunks of {a.chunk}, {a.layers} layers: {ms:.2f} ms, "
          f"{a.batch * a.prompt / ms * 1e3:.0f} tokens/s")

    one = batches[1]
    x = h.view(a.batch, -1, a.hidden)[:, -1].contiguous()  # in place of an embedding
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        one.run(layers, x, norm)  # warm-up: one token, taken back below
        lens -= 1
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.copy_(one.run(layers, x, norm))
    torch.cuda.synchronize()
    start.record()
    for _ in range(a.steps):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    us = start.elapsed_time(end) * 1e3 / a.steps
    print(f"decode: {a.batch} sequences, {a.steps} steps: {us:.1f} us a step, {us / a.layers:.1f} us a layer")
    k, v = one.cached(layers[0], 0, 0, int(lens[0]))
    print(f"cache of sequence 0: {k.shape[0]} tokens, rms of K {k.float().pow(2).mean().sqrt():.3f}, "
          f"of V {v.float().pow(2).mean().sqrt():.3f}, rms of the last norm {x.float().pow(2).mean().sqrt():.3f}")
    assert N.nvfp4_get_device_status() == 0


if __name__ == "__main__":
    main()
