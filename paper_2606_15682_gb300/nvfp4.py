"""Thin ctypes binding of libnvfp4.so (include/nvfp4.h).

Argument marshalling only: every function takes torch CUDA tensors (or plain
integers for scalars), passes their device pointers and the current CUDA
stream to the C entry point of the same name, and raises ``NVFP4Error`` on a
non-OK status.  No computation happens here, and there is no CPU fallback:
if the library is missing, importing this module fails.
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
# NVFP4_DEBUG=1 selects the bounds-checked build, NVFP4_TIMELINE=1 the
# timeline build (paper_2606_15682_gb300.build).
LIB_PATH = os.path.join(_PKG, "_build_debug" if os.environ.get("NVFP4_DEBUG") == "1" else
                        ("_build_timeline" if os.environ.get("NVFP4_TIMELINE") == "1" else "_build"), "libnvfp4.so")

SCALES_ROWMAJOR = 0
SCALES_MMA = 1

STATUS = {0: "ok", 1: "invalid argument", 2: "shape", 3: "alignment", 4: "unsupported", 5: "cuda",
          6: "timeout", 7: "capacity"}


class NVFP4Error(RuntimeError):
    def __init__(self, fn, code):
        self.code = code
        super().__init__(f"{fn} failed: {STATUS.get(code, code)} ({code})")


if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is missing: run paper_2606_15682_gb300.build.build() first")
_lib = ctypes.CDLL(LIB_PATH)

_p, _i64, _i32, _f32, _sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t


class KVCacheStruct(ctypes.Structure):
    _fields_ = [("k_codes", _p), ("k_scales", _p), ("v_codes", _p), ("v_scales", _p), ("seq_lens", _p),
                ("batch", _i32), ("num_kv_heads", _i32), ("head_dim", _i32), ("capacity", _i32),
                ("k_gscale", _f32), ("v_gscale", _f32), ("kv_format", _i32)]


class KVPagesStruct(ctypes.Structure):
    _fields_ = [("table", _p), ("seq_lens", _p), ("batch", _i32), ("pages_per_seq", _i32)]


class AttentionOptionsStruct(ctypes.Structure):
    _fields_ = [("softmax_scale", _f32), ("logit_cap", _f32), ("slopes", _p), ("window", _i32),
                ("prefix_lens", _p), ("doc_start", _p)]


class MoEPlanStruct(ctypes.Structure):
    _fields_ = [("row_start", _p), ("rows", _p), ("row_of", _p), ("n_tokens", _i64), ("top_k", _i32),
                ("num_experts", _i32)]


class MoERouteOptionsStruct(ctypes.Structure):
    _fields_ = [("score", _i32), ("renormalize", _i32), ("scale", _f32), ("bias", _p)]


# The same structs as bytes: one call makes them.
_PLAN, _ROUTE = struct.Struct("PPPqii"), struct.Struct("iif4xP")
assert (_PLAN.size, _ROUTE.size) == (ctypes.sizeof(MoEPlanStruct), ctypes.sizeof(MoERouteOptionsStruct))
_CACHE, _PAGES, _OPTIONS = struct.Struct("PPPPPiiiiffi4x"), struct.Struct("PPii"), struct.Struct("ffPi4xPP")
assert (_CACHE.size, _PAGES.size, _OPTIONS.size) == tuple(
    ctypes.sizeof(t) for t in (KVCacheStruct, KVPagesStruct, AttentionOptionsStruct))


def _sig(name, args, res=ctypes.c_int):
    f = getattr(_lib, name)
    f.argtypes = args
    f.restype = res
    return f


_tensor_scale = _sig("nvfp4_tensor_scale", [_p, _i64, _i64, _i64, _p, _p])
_quantize = _sig("nvfp4_quantize", [_p, _i64, _i64, _i64, _p, _p, _p, ctypes.c_int, _p])
_quantize_dynamic = _sig("nvfp4_quantize_dynamic", [_p, _i64, _i64, _i64, _p, _p, _p, _p, ctypes.c_int, _p])
_relayout = _sig("nvfp4_scales_relayout", [_p, _p, _i64, _i64, ctypes.c_int, ctypes.c_int, _p])
_linear = _sig("nvfp4_linear", [_p, _p, _p, _p, _p, _p, _i64, _i64, _i64, _p, _i64, _p])
_linear_dynamic = _sig("nvfp4_linear_dynamic", [_p, _i64, _i64, _i64, _p, _p, _p, _i64, _p, _i64, _p, _p])
_linear_swiglu = _sig("nvfp4_linear_swiglu_quantize", [_p, _p, _p, _p, _p, _p, _i64, _i64, _i64, _p, _p, _p, _p])
_interleave = _sig("nvfp4_interleave_gate_up", [_p, _p, _i64, _i64, _p, _p])
_kv_append = _sig("kv_append_nvfp4", [ctypes.POINTER(KVCacheStruct), _p, _p, _p, _p, _i64, _p, _p])
_kv_append_rope = _sig("kv_append_rope_nvfp4",
                       [ctypes.POINTER(KVCacheStruct), _p, _p, _p, _p, _i64, _p, _i64, _p, _p])
_rope_table = _sig("nvfp4_rope_table", [_p, _i64, _i32, _f32, _p])
_attn_ws = _sig("decode_attention_nvfp4_workspace_size", [_i32, _i32, _i32], _sz)
_attn = _sig("decode_attention_nvfp4", [ctypes.POINTER(KVCacheStruct), _p, _i32, _f32, _p, _p, _sz, _p])
_attn_quant = _sig("decode_attention_nvfp4_quantize",
                   [ctypes.POINTER(KVCacheStruct), _p, _i32, _f32, _p, _p, _p, _p, _sz, _p])
_attn_static = _sig("decode_attention_nvfp4_static_scratch", [ctypes.POINTER(KVCacheStruct), _p, _i32, _f32, _p, _p])
_qfit_ws = _sig("nvfp4_qfit_workspace_size", [_i32, _i32, _i32, _i32, _i32, _i32], _sz)
_qfit = _sig("nvfp4_qfit_calibrate", [_p, _p, _p, _i32, _i32, _i32, _i32, _i32, _p, _i64, _i32, _i32,
                                      ctypes.c_double, _i32, _p, _p, _p, _p, _p, _sz, _p])
_append_axes = _sig("kv_append_rope_axes_nvfp4",
                    [_p, _p, _p, _i64, _i32, _p, _i64, _p, _i64, _p, _p, _p, _i32, _p, _i64, _p, _i64, _p, _p, _p])
_kv_read = _sig("kv_read_nvfp4", [_p, _p, _p, _p, _i64, _p, _p, _p])
_extend_ws = _sig("extend_attention_nvfp4_workspace_size", [_i32, _i64, _i32, _i32, _i64], _sz)
_extend = _sig("extend_attention_nvfp4",
               [_p, _p, _p, _i64, _i64, _i32, _p, _p, _p, _p, _sz, _p])
_residual_norm = _sig("residual_norm_nvfp4", [_p, _i64, _p, _i64, _i64, _i64, _p, _p, _i64, _f32, _p, _f32, _p, _p, _p,
                                              _p, _p, _p])
_moe_max_rows = _sig("moe_max_rows", [_i64, _i32, _i32], _i64)
_moe_sort_ws = _sig("moe_sort_workspace_size", [_i64, _i32, _i32], _sz)
_moe_route = _sig("moe_route", [_p, _i32, _i64, _i64, _i32, _i32, _p, _p, _p, _p])
_moe_route_backward = _sig("moe_route_backward", [_p, _i32, _i64, _i64, _i32, _i32, _p, _p, _p, _p, _p])
_moe_sort = _sig("moe_sort", [_p, _p, _p, _sz, _p])
_moe_dispatch = _sig("moe_dispatch", [_p, _p, _i64, _i64, _p, _p, _p])
_moe_dispatch_nvfp4 = _sig("moe_dispatch_nvfp4", [_p, _p, _i64, _i64, _p, _p, _p, _p])
_moe_dispatch_mxfp4 = _sig("moe_dispatch_mxfp4", [_p, _p, _i64, _i64, ctypes.c_int, _p, _p, _p])
_moe_combine = _sig("moe_combine", [_p, _p, _i64, _p, _p, _i64, _p, _i64, _p])
_moe_combine_backward = _sig("moe_combine_backward", [_p, _p, _i64, _p, _i64, _p, _p, _p, _p])
_linear_grouped = _sig("nvfp4_linear_grouped", [_p, _p, _p, _p, _i32, _p, _p, _p, _i64, _i64, _p, _i64, _p])
_mx_linear_grouped = _sig("mxfp4_linear_grouped", [_p, _p, _p, _p, _p, _i64, _i64, _p, _i64, _p])
_linear_grouped_swiglu = _sig("nvfp4_linear_grouped_swiglu_quantize",
                              [_p, _p, _p, _p, _i32, _p, _p, _p, _i64, _i64, _p, _i32, _p, _p, _p])
_mx_linear_grouped_swiglu = _sig("mxfp4_linear_grouped_swiglu_quantize",
                                 [_p, _p, _p, _p, _p, _i64, _i64, ctypes.c_int, _p, _p, _p])
_get_status = _sig("nvfp4_get_device_status", [ctypes.POINTER(_i32), _p])
_status_string = _sig("nvfp4_status_string", [ctypes.c_int], ctypes.c_char_p)
_launch_count = _sig("nvfp4_launch_count", [], ctypes.c_uint64)
_scales_bytes = _sig("nvfp4_scales_bytes", [_i64, _i64, ctypes.c_int], _sz)
_mx_scales_bytes = _sig("mxfp4_scales_bytes", [_i64, _i64, ctypes.c_int], _sz)
_inject_fault = _sig("nvfp4_debug_inject_fault", [ctypes.c_int])
FAULT_NONE, FAULT_ATTN_SKIP_STAGE, FAULT_GEMM_SKIP_STAGE, FAULT_GROUPED_REVERSED = 0, 1, 2, 3


def nvfp4_debug_inject_fault(what):
    """Test-only: arm one injected fault for the next call of its kind (see include/nvfp4.h)."""
    _check("nvfp4_debug_inject_fault", _inject_fault(what))
_mx_quantize = _sig("mxfp4_quantize", [_p, _i64, _i64, _i64, ctypes.c_int, _p, _p, ctypes.c_int, _p])
_mx_linear = _sig("mxfp4_linear", [_p, _p, _p, _p, _i64, _i64, _i64, _p, _i64, _p])
_mx_linear_swiglu = _sig("mxfp4_linear_swiglu_quantize", [_p, _p, _p, _p, _i64, _i64, _i64, ctypes.c_int, _p, _p, _p])


# The current stream's raw handle without building a torch.cuda.Stream object
# (0.1 us instead of ~3 us per call); the public calls where these are absent.
_raw_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _handle(stream):
    """A stream's handle as an integer; None: the current one's."""
    if stream is None:
        if _raw_current_stream is not None:
            return _raw_current_stream(_raw_current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _stream(stream):
    return ctypes.c_void_p(_handle(stream))


def _ptr(t):
    """Device pointer of a dense tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensor arguments must be contiguous (row-padded 2-D inputs go through the ld argument)")
    return ctypes.c_void_p(t.data_ptr())


def _mat(x):
    """(pointer, rows, cols, ld) of a 2-D row-major tensor whose rows may be padded."""
    if x.dim() != 2 or (x.shape[1] > 1 and x.stride(1) != 1):
        raise ValueError("expected a 2-D row-major tensor")
    rows, cols = x.shape
    ld = x.stride(0) if rows > 1 else cols
    if rows > 1 and ld < cols:
        raise ValueError("rows overlap")
    return ctypes.c_void_p(x.data_ptr()), rows, cols, ld


def _check(fn, code):
    if code != 0:
        raise NVFP4Error(fn, code)


# ----------------------------------------------------------------- calls ---

def nvfp4_scales_bytes(rows, cols, layout):
    return int(_scales_bytes(rows, cols, layout))


def nvfp4_tensor_scale(x, g, stream=None):
    """g[0] <- amax(|x|) / (6*448) (device)."""
    _check("nvfp4_tensor_scale", _tensor_scale(*_mat(x), _ptr(g), _stream(stream)))


def nvfp4_quantize(x, g, codes, scales, layout=SCALES_MMA, stream=None):
    _check("nvfp4_quantize", _quantize(*_mat(x), _ptr(g), _ptr(codes), _ptr(scales), layout, _stream(stream)))


DYNAMIC_STATE_BYTES = 16
KV_E2M1, KV_E1M2 = 0, 1


def nvfp4_quantize_dynamic(x, state, g, codes, scales, layout=SCALES_MMA, stream=None):
    """Tensor scale + quantization in one launch; `state` is a zero-filled
    device buffer of DYNAMIC_STATE_BYTES bytes owned by the caller."""
    _check("nvfp4_quantize_dynamic",
           _quantize_dynamic(*_mat(x), _ptr(state), _ptr(g), _ptr(codes), _ptr(scales), layout, _stream(stream)))


def nvfp4_scales_relayout(src, dst, rows, cols, from_layout, to_layout, stream=None):
    _check("nvfp4_scales_relayout", _relayout(_ptr(src), _ptr(dst), rows, cols, from_layout, to_layout,
                                              _stream(stream)))


def nvfp4_linear(a_codes, a_scales, g_a, w_codes, w_scales, g_w, out, M, N, K, ldo=None, stream=None):
    _check("nvfp4_linear", _linear(_ptr(a_codes), _ptr(a_scales), _ptr(g_a), _ptr(w_codes), _ptr(w_scales),
                                   _ptr(g_w), M, N, K, _ptr(out), N if ldo is None else ldo, _stream(stream)))


def nvfp4_linear_dynamic(x, w_codes, w_scales, g_w, out, N, ldo=None, g_a=None, stream=None):
    """Tensor scale, quantization of the bf16 activation x [M, K] (M <= 32,
    K <= 1536) and the linear layer with W in one launch; g_a (optional
    device float) receives the tensor scale."""
    ptr, M, K, ld = _mat(x)
    _check("nvfp4_linear_dynamic", _linear_dynamic(ptr, M, K, ld, _ptr(w_codes), _ptr(w_scales), _ptr(g_w), N,
                                                   _ptr(out), N if ldo is None else ldo, _ptr(g_a),
                                                   _stream(stream)))


def mxfp4_scales_bytes(rows, cols, layout):
    return int(_mx_scales_bytes(rows, cols, layout))


def mxfp4_quantize(x, codes, scales, layout=SCALES_MMA, rotate=False, stream=None):
    """MXFP4 codes and E8M0 block scales of a bf16 [rows, cols] tensor
    (optionally after the 32-element block rotation)."""
    _check("mxfp4_quantize", _mx_quantize(*_mat(x), int(bool(rotate)), _ptr(codes), _ptr(scales), layout,
                                          _stream(stream)))


def mxfp4_linear(a_codes, a_scales, w_codes, w_scales, out, M, N, K, ldo=None, stream=None):
    _check("mxfp4_linear", _mx_linear(_ptr(a_codes), _ptr(a_scales), _ptr(w_codes), _ptr(w_scales), M, N, K,
                                      _ptr(out), N if ldo is None else ldo, _stream(stream)))


def mxfp4_linear_swiglu_quantize(a_codes, a_scales, w_codes, w_scales, M, I, K, out_codes, out_scales,
                                  rotate=False, stream=None):
    _check("mxfp4_linear_swiglu_quantize",
           _mx_linear_swiglu(_ptr(a_codes), _ptr(a_scales), _ptr(w_codes), _ptr(w_scales), M, I, K,
                             int(bool(rotate)), _ptr(out_codes), _ptr(out_scales), _stream(stream)))


def nvfp4_linear_swiglu_quantize(a_codes, a_scales, g_a, w_codes, w_scales, g_w, M, I, K, g_out,
                                 out_codes, out_scales, stream=None):
    _check("nvfp4_linear_swiglu_quantize",
           _linear_swiglu(_ptr(a_codes), _ptr(a_scales), _ptr(g_a), _ptr(w_codes), _ptr(w_scales), _ptr(g_w),
                          M, I, K, _ptr(g_out), _ptr(out_codes), _ptr(out_scales), _stream(stream)))


def nvfp4_interleave_gate_up(w_gate, w_up, w_out, stream=None):
    _check("nvfp4_interleave_gate_up",
           _interleave(_ptr(w_gate), _ptr(w_up), w_gate.shape[0], w_gate.shape[1] * w_gate.element_size(),
                       _ptr(w_out), _stream(stream)))


def kv_append_nvfp4(cache, k, v, seq_idx, pos, k_shift=None, stream=None):
    s = cache.struct()
    _check("kv_append_nvfp4", _kv_append(ctypes.byref(s), _ptr(k), _ptr(v), _ptr(seq_idx), _ptr(pos), k.shape[0],
                                         _ptr(k_shift), _stream(stream)))


def kv_append_rope_nvfp4(cache, k_pre, v, seq_idx, pos, rope_table, k_shift=None, stream=None):
    """rope_table: float32 [n_pos, 64, 2] (see nvfp4_rope_table), n_pos >= cache.capacity."""
    s = cache.struct()
    _check("kv_append_rope_nvfp4",
           _kv_append_rope(ctypes.byref(s), _ptr(k_pre), _ptr(v), _ptr(seq_idx), _ptr(pos), k_pre.shape[0],
                           _ptr(rope_table), rope_table.shape[0], _ptr(k_shift), _stream(stream)))


def nvfp4_rope_table(table, theta=1.0e6, stream=None):
    """Fill table (float32 [n_pos, head_dim/2, 2]) with (cos, sin) of p * theta^(-2i/head_dim)."""
    _check("nvfp4_rope_table", _rope_table(_ptr(table), table.shape[0], 2 * table.shape[1], theta, _stream(stream)))


def decode_attention_nvfp4_workspace_size(batch, num_q_heads, capacity):
    return int(_attn_ws(batch, num_q_heads, capacity))


def decode_attention_nvfp4(cache, q, softmax_scale, out, workspace, stream=None):
    s = cache.struct()
    _check("decode_attention_nvfp4", _attn(ctypes.byref(s), _ptr(q), q.shape[1], softmax_scale, _ptr(out),
                                           _ptr(workspace), workspace.numel() * workspace.element_size(),
                                           _stream(stream)))


ATTN_STATIC_SCRATCH_BYTES = 24 << 20


def decode_attention_nvfp4_quantize(cache, q, softmax_scale, g_out, out_codes, out_scales, workspace, stream=None):
    """out_codes [batch, H_q*64] uint8, out_scales MMA layout for [batch, H_q*128]."""
    s = cache.struct()
    _check("decode_attention_nvfp4_quantize",
           _attn_quant(ctypes.byref(s), _ptr(q), q.shape[1], softmax_scale, _ptr(g_out), _ptr(out_codes),
                       _ptr(out_scales), _ptr(workspace), workspace.numel() * workspace.element_size(),
                       _stream(stream)))


def decode_attention_nvfp4_static_scratch(cache, q, softmax_scale, out, stream=None):
    """Decode attention whose partials live in the library's own device scratch (no workspace)."""
    s = cache.struct()
    _check("decode_attention_nvfp4_static_scratch", _attn_static(ctypes.byref(s), _ptr(q), q.shape[1], softmax_scale,
                                                                 _ptr(out), _stream(stream)))


# The calls of a decode step are short, and so is their marshalling: plain integers for
# pointers, each tensor looked at once, the structs packed (include/nvfp4.h's layout).
_bf16, _int32, _float32, _uint8 = torch.bfloat16, torch.int32, torch.float32, torch.uint8


def _rows3(x, what):
    """(pointer, tokens, heads, elements between tokens) of a bf16 [tokens, heads, 128] tensor that may be a slice of
    a wider projection output."""
    n, h, d = x.shape
    between, head, last = x.stride()
    if d != 128 or last != 1 or (h > 1 and head != 128) or x.dtype is not _bf16:
        raise ValueError(f"{what} must be a bfloat16 [tokens, heads, 128] tensor with dense heads")
    return x.data_ptr(), n, h, between if n > 1 else h * 128


def _typed(t, dtype, what, numel=None):
    """Device pointer of a dense argument whose element type the call fixes; None -> NULL."""
    if t is None:
        return None
    if t.dtype is not dtype or (numel is not None and t.numel() != numel) or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous {dtype}" + ("" if numel is None else f" with {numel} elements"))
    return t.data_ptr()


def kv_append_rope_axes_nvfp4(cache, q, k, v, seq_idx, pos, rope_pos, axis_of_pair, rope_table, q_out, k_shift=None,
                              pages=None, stream=None):
    """Rotate q (-> q_out) and k by rotary positions rope_pos [n, axes] and append k and v to the (paged) cache.

    q, k, v: [n, heads, 128] bf16, may be slices of one projection output; q and q_out may be None.
    axis_of_pair: 64 integers (a bytes object is taken as it is), the axis that rotates each channel pair (c, c + 64).
    """
    kp, n, hk, ld_k = _rows3(k, "k")
    vp, nv, hv, ld_v = _rows3(v, "v")
    qp, nq, hq, ld_q = _rows3(q, "q") if q is not None else (None, n, 0, 0)
    n_rope, axes = rope_pos.shape
    if not (n == nv == nq == n_rope) or hk != cache.num_kv_heads or hv != hk:
        raise ValueError("q, k, v and rope_pos must have the same tokens, k and v the cache's heads")
    if q is not None and q_out is None:
        raise ValueError("q_out must hold the rotated queries")
    if type(axis_of_pair) is not bytes:
        axis_of_pair = bytes(axis_of_pair)
    if len(axis_of_pair) != 64:
        raise ValueError("axis_of_pair must have 64 entries")
    _check("kv_append_rope_axes_nvfp4",
           _append_axes(cache.packed(), None if pages is None else pages.packed(), qp, ld_q, hq, kp, ld_k, vp, ld_v,
                        _typed(seq_idx, _int32, "seq_idx", n), _typed(pos, _int32, "pos", n),
                        _typed(rope_pos, _int32, "rope_pos"), axes, axis_of_pair, n,
                        _typed(rope_table, _float32, "rope_table", len(rope_table) * 128), len(rope_table),
                        None if k_shift is None else _typed(k_shift, _float32, "k_shift", hk * 128),
                        None if q is None else _typed(q_out, _bf16, "q_out", n * hq * 128), _stream(stream)))


def kv_read_nvfp4(cache, seq_idx, pos, k_out, v_out, pages=None, stream=None):
    """Cached rows (seq_idx[i], pos[i]) as bf16 [n, kv heads, 128]; k_out or v_out may be None."""
    n = seq_idx.numel()
    size = n * cache.num_kv_heads * 128
    _check("kv_read_nvfp4",
           _kv_read(cache.packed(), None if pages is None else pages.packed(), _typed(seq_idx, _int32, "seq_idx"),
                    _typed(pos, _int32, "pos", n), n, _typed(k_out, _bf16, "k_out", size),
                    _typed(v_out, _bf16, "v_out", size), _stream(stream)))


def extend_attention_nvfp4_workspace_size(batch, n_tokens, num_q_heads, num_kv_heads, context):
    """context: the cache's capacity, or pages_per_seq * page tokens."""
    return int(_extend_ws(batch, n_tokens, num_q_heads, num_kv_heads, context))


def extend_attention_nvfp4(cache, q, softmax_scale, out, workspace, q_start=None, pages=None, logit_cap=0.0, window=0,
                           slopes=None, prefix_lens=None, doc_start=None, stream=None):
    """Attention of the new tokens q [n_tokens, heads, 128] over the cache that holds them (see include/nvfp4.h)."""
    qp, n, hq, ld_q = _rows3(q, "q")
    batch = cache.batch if pages is None else pages.batch
    options = _OPTIONS.pack(softmax_scale, logit_cap, _typed(slopes, _float32, "slopes", hq) or 0, window,
                            _typed(prefix_lens, _int32, "prefix_lens", batch) or 0,
                            _typed(doc_start, _int32, "doc_start", n) or 0)
    _check("extend_attention_nvfp4",
           _extend(cache.packed(), None if pages is None else pages.packed(), qp, ld_q, n, hq,
                   _typed(q_start, _int32, "q_start", batch + 1), options, _typed(out, _bf16, "out", n * hq * 128),
                   *((None, 0) if workspace is None else (workspace.data_ptr(), workspace.nbytes)), _stream(stream)))


def residual_norm_nvfp4(x, y, r_out, h_out, w_norm, eps=1e-6, w_post=None, gate=None, rows_per_gate=1, alpha=1.0,
                        g_out=None, codes=None, scales=None, stream=None):
    """r = x + alpha * (y, normed by w_post, gated); h = norm of r: bf16 (h_out) and / or NVFP4 (codes, scales, g_out).
    y, r_out, h_out, w_norm may be None."""
    rows, cols = x.shape
    ld_x, step = x.stride()
    ld_y, yp = 0, None
    if x.dtype is not _bf16 or (cols > 1 and step != 1):
        raise ValueError("x must be row-major bfloat16")
    if y is not None:
        ld_y, step = y.stride()
        yp = y.data_ptr()
        if y.dtype is not _bf16 or y.shape != x.shape or (cols > 1 and step != 1):
            raise ValueError("y must be row-major bfloat16 of x's shape")
    if rows == 1:
        ld_x, ld_y = cols, cols
    if gate is None:
        rows_per_gate = 1
    elif rows_per_gate < 1 or gate.shape[-1] != cols or gate.numel() != -(-rows // rows_per_gate) * cols:
        raise ValueError("gate must be [ceil(rows / rows_per_gate), cols]")
    n = rows * cols
    if codes is not None and (codes.numel() != n // 2 or scales is None or g_out is None or
                              scales.numel() != _scales_bytes(rows, cols, SCALES_MMA)):
        raise ValueError("codes [rows, cols/2] come with g_out and MMA-layout scales")
    _check("residual_norm_nvfp4",
           _residual_norm(x.data_ptr(), ld_x, yp, ld_y, rows, cols, _typed(w_post, _bf16, "w_post", cols),
                          _typed(gate, _bf16, "gate"), rows_per_gate, alpha, _typed(w_norm, _bf16, "w_norm", cols), eps,
                          _typed(r_out, _bf16, "r_out", n), _typed(h_out, _bf16, "h_out", n),
                          _typed(g_out, _float32, "g_out"), _typed(codes, torch.uint8, "codes"),
                          _typed(scales, torch.uint8, "scales"), _stream(stream)))


# ------------------------------------------------- mixture of experts ---

MOE_SOFTMAX, MOE_SIGMOID = 0, 1


def moe_max_rows(n_tokens, top_k, num_experts):
    """Rows of a plan's buffers (include/nvfp4.h)."""
    return int(_moe_max_rows(n_tokens, top_k, num_experts))


def moe_sort_workspace_size(n_tokens, top_k, num_experts):
    return int(_moe_sort_ws(n_tokens, top_k, num_experts))


# Each tensor is looked at once: these calls are a few microseconds of a decode step whose kernels are no longer.

def _matrix(x, rows, what):
    """(pointer, elements between rows, cols) of a bf16 [rows, cols] argument whose rows may be padded."""
    n, cols = x.shape
    between, step = x.stride()
    if x.dtype is not _bf16 or n != rows or (step != 1 and cols > 1):
        raise ValueError(f"{what} must be row-major bfloat16 [{rows}, cols]")
    return x.data_ptr(), between if rows > 1 else cols, cols


def _bytes(t, numel, what):
    """Device pointer of a dense uint8 argument of `numel` bytes."""
    if t.dtype is not _uint8 or t.numel() != numel or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous uint8 with {numel} elements")
    return t.data_ptr()


def _floats(t, numel, what):
    """Device pointer of a dense float32 argument of `numel` numbers."""
    if t.dtype is not _float32 or t.numel() != numel or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous float32 with {numel} elements")
    return t.data_ptr()


def _rows(t, numel, what):
    """Device pointer of a plan's dense bf16 rows."""
    if t.dtype is not _bf16 or t.numel() != numel or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous bfloat16 with {numel} elements")
    return t.data_ptr()


def _logits(logits, tokens):
    """(pointer, nvfp4_float_type, elements between rows, experts) of a router's [tokens, experts]."""
    n, experts = logits.shape
    between, step = logits.stride()
    dtype = logits.dtype
    if (dtype is not _float32 and dtype is not _bf16) or (step != 1 and experts > 1) or n != tokens:
        raise ValueError("logits must be row-major float32 or bfloat16 [tokens, experts] of expert_idx's tokens")
    return logits.data_ptr(), 1 if dtype is _bf16 else 0, between if n > 1 else experts, experts


def moe_route(logits, expert_idx, weights, score=MOE_SOFTMAX, renormalize=True, scale=1.0, bias=None, stream=None):
    """The experts expert_idx [tokens, top_k] (int32) of each token and their weights (float32) from logits [tokens,
    experts]; bias (with MOE_SIGMOID) moves the choice alone."""
    n, k = expert_idx.shape
    lp, kind, ld, experts = _logits(logits, n)
    _check("moe_route",
           _moe_route(lp, kind, ld, n, experts, k,
                      _ROUTE.pack(score, renormalize, scale, 0 if bias is None else _floats(bias, experts, "bias")),
                      _typed(expert_idx, _int32, "expert_idx"), _floats(weights, n * k, "weights"), _handle(stream)))


def moe_route_backward(logits, expert_idx, d_weights, d_logits, score=MOE_SOFTMAX, renormalize=True, scale=1.0,
                       stream=None):
    """The logits' gradient (dense, of their type) from that of moe_route's weights."""
    n, k = expert_idx.shape
    lp, kind, ld, experts = _logits(logits, n)
    _check("moe_route_backward",
           _moe_route_backward(lp, kind, ld, n, experts, k, _ROUTE.pack(score, renormalize, scale, 0),
                               _typed(expert_idx, _int32, "expert_idx"), _floats(d_weights, n * k, "d_weights"),
                               _typed(d_logits, logits.dtype, "d_logits", n * experts), _handle(stream)))


def moe_sort(plan, expert_idx, stream=None):
    """The plan's rows for expert_idx int32 [n_tokens, top_k]; a negative entry is a choice without an expert."""
    ws = plan.workspace
    _check("moe_sort", _moe_sort(plan.packed(), _typed(expert_idx, _int32, "expert_idx", plan.choices),
                                 *((None, 0) if ws is None else (ws.data_ptr(), ws.nbytes)), _handle(stream)))


def moe_dispatch(plan, x, rows, weights=None, stream=None):
    """x [n_tokens, cols] bf16 to its experts' rows [plan.max_rows, cols], times weights [n_tokens, top_k] if given."""
    xp, ld, cols = _matrix(x, plan.n_tokens, "x")
    _check("moe_dispatch",
           _moe_dispatch(plan.packed(), xp, ld, cols, None if weights is None else _floats(weights, plan.choices, "weights"),
                         _rows(rows, plan.max_rows * cols, "rows"), _handle(stream)))


def moe_dispatch_nvfp4(plan, x, g, codes, scales, stream=None):
    """x [n_tokens, cols] bf16, NVFP4-quantized with the scale g, to its experts' rows: codes [plan.max_rows, cols/2] and
    MMA-layout scales."""
    xp, ld, cols = _matrix(x, plan.n_tokens, "x")
    n = plan.max_rows * cols
    _check("moe_dispatch_nvfp4",
           _moe_dispatch_nvfp4(plan.packed(), xp, ld, cols, _floats(g, 1, "g"), _bytes(codes, n // 2, "codes"),
                               _bytes(scales, n // 16, "scales"), _handle(stream)))


def moe_dispatch_mxfp4(plan, x, codes, scales, rotate=False, stream=None):
    """The same as MXFP4, optionally after the 32-element block rotation."""
    xp, ld, cols = _matrix(x, plan.n_tokens, "x")
    n = plan.max_rows * cols
    _check("moe_dispatch_mxfp4",
           _moe_dispatch_mxfp4(plan.packed(), xp, ld, cols, int(bool(rotate)), _bytes(codes, n // 2, "codes"),
                               _bytes(scales, n // 16, "scales"), _handle(stream)))


def moe_combine(plan, y, out, weights=None, base=None, stream=None):
    """out [n_tokens, cols] = base + the sum of weights * y over each token's rows; also the gradient of moe_dispatch's x
    from that of its rows, y, with the weights that it had or without."""
    op, ld, cols = _matrix(out, plan.n_tokens, "out")
    bp, ld_base, base_cols = (None, 0, cols) if base is None else _matrix(base, plan.n_tokens, "base")
    if base_cols != cols:
        raise ValueError("base must have out's shape")
    _check("moe_combine",
           _moe_combine(plan.packed(), _rows(y, plan.max_rows * cols, "y"), cols,
                        None if weights is None else _floats(weights, plan.choices, "weights"), bp, ld_base, op, ld,
                        _handle(stream)))


def moe_combine_backward(plan, d_out, y, weights, d_y, d_weights, stream=None):
    """moe_combine's gradients: d_y [max_rows, cols] and d_weights [n_tokens, top_k]; one of them may be None.  With x in place
    of d_out and the rows' gradient in place of y, d_weights is that of a weighted moe_dispatch."""
    gp, ld, cols = _matrix(d_out, plan.n_tokens, "d_out")
    n = plan.max_rows * cols
    _check("moe_combine_backward",
           _moe_combine_backward(plan.packed(), gp, ld, _rows(y, n, "y"), cols, _floats(weights, plan.choices, "weights"),
                                 None if d_y is None else _rows(d_y, n, "d_y"),
                                 None if d_weights is None else _floats(d_weights, plan.choices, "d_weights"),
                                 _handle(stream)))


def _per_expert(g, plan, what):
    """(pointer, step) of a tensor scale: one for all, or one an expert."""
    n = g.numel()
    if n != 1 and n != plan.num_experts:
        raise ValueError(f"{what} must have one element or one an expert")
    return _floats(g, n, what), 0 if n == 1 else 1


def nvfp4_linear_grouped(plan, a_codes, a_scales, g_a, w_codes, w_scales, g_w, out, N, K, stream=None):
    """out [plan.max_rows, N]: each expert's rows [.., K] times its weight [N, K]; g_a: one or one an expert."""
    E, R = plan.num_experts, plan.max_rows
    op, ldo, cols = _matrix(out, R, "out")
    if cols != N:
        raise ValueError("out must be [plan.max_rows, N]")
    ga, ga_step = _per_expert(g_a, plan, "g_a")
    _check("nvfp4_linear_grouped",
           _linear_grouped(plan.packed(), _bytes(a_codes, R * K // 2, "a_codes"), _bytes(a_scales, R * K // 16, "a_scales"),
                           ga, ga_step, _bytes(w_codes, E * N * K // 2, "w_codes"),
                           _bytes(w_scales, E * ((N + 127) // 128 * 128) * (K // 16), "w_scales"), _floats(g_w, E, "g_w"),
                           N, K, op, ldo, _handle(stream)))


def mxfp4_linear_grouped(plan, a_codes, a_scales, w_codes, w_scales, out, N, K, stream=None):
    E, R = plan.num_experts, plan.max_rows
    op, ldo, cols = _matrix(out, R, "out")
    if cols != N:
        raise ValueError("out must be [plan.max_rows, N]")
    _check("mxfp4_linear_grouped",
           _mx_linear_grouped(plan.packed(), _bytes(a_codes, R * K // 2, "a_codes"),
                              _bytes(a_scales, R * K // 16, "a_scales"), _bytes(w_codes, E * N * K // 2, "w_codes"),
                              _bytes(w_scales, E * ((N + 127) // 128 * 128) * (K // 16), "w_scales"), N, K, op, ldo,
                              _handle(stream)))


def nvfp4_linear_grouped_swiglu_quantize(plan, a_codes, a_scales, g_a, w_codes, w_scales, g_w, I, K, g_out, out_codes,
                                         out_scales, stream=None):
    """h = SiLU(gate) * up of each expert's rows, NVFP4-quantized with g_out (one or one an expert)."""
    E, R, N = plan.num_experts, plan.max_rows, 2 * I
    ga, ga_step = _per_expert(g_a, plan, "g_a")
    go, go_step = _per_expert(g_out, plan, "g_out")
    _check("nvfp4_linear_grouped_swiglu_quantize",
           _linear_grouped_swiglu(plan.packed(), _bytes(a_codes, R * K // 2, "a_codes"),
                                  _bytes(a_scales, R * K // 16, "a_scales"), ga, ga_step,
                                  _bytes(w_codes, E * N * K // 2, "w_codes"),
                                  _bytes(w_scales, E * ((N + 127) // 128 * 128) * (K // 16), "w_scales"),
                                  _floats(g_w, E, "g_w"), I, K, go, go_step, _bytes(out_codes, R * I // 2, "out_codes"),
                                  _bytes(out_scales, R * I // 16, "out_scales"), _handle(stream)))


def mxfp4_linear_grouped_swiglu_quantize(plan, a_codes, a_scales, w_codes, w_scales, I, K, out_codes, out_scales,
                                         rotate=False, stream=None):
    E, R, N = plan.num_experts, plan.max_rows, 2 * I
    _check("mxfp4_linear_grouped_swiglu_quantize",
           _mx_linear_grouped_swiglu(plan.packed(), _bytes(a_codes, R * K // 2, "a_codes"),
                                     _bytes(a_scales, R * K // 16, "a_scales"), _bytes(w_codes, E * N * K // 2, "w_codes"),
                                     _bytes(w_scales, E * ((N + 127) // 128 * 128) * (K // 16), "w_scales"), I, K,
                                     int(bool(rotate)), _bytes(out_codes, R * I // 2, "out_codes"),
                                     _bytes(out_scales, R * I // 16, "out_scales"), _handle(stream)))


def nvfp4_qfit_workspace_size(batch, tokens, num_q_heads, num_kv_heads, grid_s, grid_m):
    return int(_qfit_ws(batch, tokens, num_q_heads, num_kv_heads, grid_s, grid_m))


def nvfp4_qfit_calibrate(q_pre, k_pre, v, rope_table, grid_s, grid_m, eps, kv_format, s_q, s_k, m, errors,
                         workspace, stream=None):
    """q_pre [B, T, H_q, 128], k_pre and v [B, T, H_kv, 128] bf16; rope_table fp32 [n, 64, 2];
    s_q, s_k, m fp32 device outputs; errors: a host (CPU) float64 tensor of grid_s * grid_m, or None."""
    B, T, hq, d = q_pre.shape
    hkv = k_pre.shape[2]
    if errors is not None and (errors.device.type != "cpu" or errors.dtype != torch.float64 or
                               not errors.is_contiguous() or errors.numel() != grid_s * grid_m):
        raise ValueError("errors must be a contiguous CPU float64 tensor of grid_s * grid_m")
    _check("nvfp4_qfit_calibrate",
           _qfit(_ptr(q_pre), _ptr(k_pre), _ptr(v), B, T, hq, hkv, d, _ptr(rope_table), rope_table.shape[0], grid_s,
                 grid_m, float(eps), kv_format, _ptr(s_q), _ptr(s_k), _ptr(m),
                 None if errors is None else ctypes.c_void_p(errors.data_ptr()), _ptr(workspace),
                 workspace.numel() * workspace.element_size(), _stream(stream)))


def nvfp4_get_device_status(stream=None):
    v = _i32(0)
    _check("nvfp4_get_device_status", _get_status(ctypes.byref(v), _stream(stream)))
    return int(v.value)


def nvfp4_status_string(code):
    return _status_string(code).decode()


def nvfp4_launch_count():
    return int(_launch_count())


# ------------------------------------------------------------- KV cache ---

class KVCache:
    """Caller-owned NVFP4 KV cache buffers (layout of include/nvfp4.h)."""

    def __init__(self, batch, num_kv_heads, capacity, k_gscale, v_gscale, head_dim=128, device="cuda", kv_format=0):
        self.batch, self.num_kv_heads, self.capacity, self.head_dim = batch, num_kv_heads, capacity, head_dim
        self.kv_format = kv_format  # KV_E2M1 or KV_E1M2
        self.k_gscale, self.v_gscale = float(k_gscale), float(v_gscale)
        shape = (batch, num_kv_heads, capacity)
        self.k_codes = torch.zeros(shape + (head_dim // 2,), dtype=torch.uint8, device=device)
        self.v_codes = torch.zeros_like(self.k_codes)
        self.k_scales = torch.zeros(shape + (head_dim // 16,), dtype=torch.uint8, device=device)
        self.v_scales = torch.zeros_like(self.k_scales)
        self.seq_lens = torch.zeros(batch, dtype=torch.int32, device=device)

    def packed(self):
        """The nvfp4_kv_cache's bytes, for the calls that take it packed."""
        return _CACHE.pack(self.k_codes.data_ptr(), self.k_scales.data_ptr(), self.v_codes.data_ptr(),
                           self.v_scales.data_ptr(), self.seq_lens.data_ptr(), self.batch, self.num_kv_heads,
                           self.head_dim, self.capacity, self.k_gscale, self.v_gscale, self.kv_format)

    def struct(self):
        return KVCacheStruct(self.k_codes.data_ptr(), self.k_scales.data_ptr(), self.v_codes.data_ptr(),
                             self.v_scales.data_ptr(), self.seq_lens.data_ptr(), self.batch, self.num_kv_heads,
                             self.head_dim, self.capacity, self.k_gscale, self.v_gscale, self.kv_format)


class KVPages:
    """Sequences over a paged cache: `table` int32 [batch, pages_per_seq] of page indexes, `seq_lens` int32 [batch].
    The pool itself is a KVCache whose batch is the number of pages and whose capacity is the page's tokens."""

    def __init__(self, table, seq_lens):
        if table.dtype != torch.int32 or table.dim() != 2 or seq_lens.dtype != torch.int32 or \
                seq_lens.numel() != table.shape[0] or not table.is_contiguous() or not seq_lens.is_contiguous():
            raise ValueError("table must be int32 [batch, pages_per_seq], seq_lens int32 [batch], both contiguous")
        self.table, self.seq_lens = table, seq_lens
        self.batch, self.pages_per_seq = table.shape

    def packed(self):
        return _PAGES.pack(self.table.data_ptr(), self.seq_lens.data_ptr(), self.batch, self.pages_per_seq)


class MoEPlan:
    """Which rows of the sorted buffers n_tokens tokens with top_k choices among num_experts experts have (layout of
    include/nvfp4.h): written by moe_sort, read by the calls on rows.  Buffers of rows have max_rows of them."""

    def __init__(self, n_tokens, top_k, num_experts, device="cuda"):
        self.n_tokens, self.top_k, self.num_experts = n_tokens, top_k, num_experts
        self.max_rows, self.choices = moe_max_rows(n_tokens, top_k, num_experts), n_tokens * top_k
        if self.max_rows == 0 and n_tokens != 0:
            raise ValueError("n_tokens, top_k or num_experts out of range")
        self._arrays = (torch.zeros(num_experts + 1, dtype=torch.int32, device=device),
                        torch.zeros(num_experts, dtype=torch.int32, device=device),
                        torch.full((n_tokens, top_k), -1, dtype=torch.int32, device=device))
        size = moe_sort_workspace_size(n_tokens, top_k, num_experts)
        self.workspace = torch.empty(size, dtype=torch.uint8, device=device) if size else None
        self._packed = _PLAN.pack(*(t.data_ptr() for t in self._arrays), n_tokens, top_k, num_experts)

    # The arrays are the plan's own for its life: their addresses are packed once.
    row_start = property(lambda self: self._arrays[0])
    rows = property(lambda self: self._arrays[1])
    row_of = property(lambda self: self._arrays[2])

    def packed(self):
        """The moe_plan's bytes, for the calls that take it packed."""
        return self._packed


EXPORTED = ["nvfp4_scales_bytes", "nvfp4_tensor_scale", "nvfp4_quantize", "nvfp4_quantize_dynamic", "nvfp4_scales_relayout", "nvfp4_linear",
            "nvfp4_linear_dynamic",
            "nvfp4_linear_swiglu_quantize", "nvfp4_interleave_gate_up",
            "mxfp4_scales_bytes", "mxfp4_quantize", "mxfp4_linear", "mxfp4_linear_swiglu_quantize",
            "kv_append_nvfp4", "kv_append_rope_nvfp4", "nvfp4_rope_table", "decode_attention_nvfp4_workspace_size", "decode_attention_nvfp4",
            "decode_attention_nvfp4_quantize",
            "decode_attention_nvfp4_static_scratch", "nvfp4_qfit_workspace_size", "nvfp4_qfit_calibrate",
            "kv_append_rope_axes_nvfp4", "kv_read_nvfp4", "extend_attention_nvfp4_workspace_size",
            "extend_attention_nvfp4", "residual_norm_nvfp4",
            "moe_max_rows", "moe_route", "moe_route_backward", "moe_sort_workspace_size", "moe_sort", "moe_dispatch",
            "moe_dispatch_nvfp4", "moe_dispatch_mxfp4", "moe_combine", "moe_combine_backward", "nvfp4_linear_grouped",
            "mxfp4_linear_grouped", "nvfp4_linear_grouped_swiglu_quantize", "mxfp4_linear_grouped_swiglu_quantize",
            "nvfp4_get_device_status", "nvfp4_status_string", "nvfp4_launch_count", "nvfp4_debug_inject_fault"]
