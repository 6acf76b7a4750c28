// Rotary positions on several axes with the quantized append of K and V, and
// the cache read back, over a contiguous or a paged cache.
#include "kv_pages.cuh"

namespace nvfp4 {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxAxes = 4;

struct AppendArgs {
  KVMap map;
  uint8_t* kc;
  uint8_t* ks;
  uint8_t* vc;
  uint8_t* vs;
  const uint16_t* q;
  const uint16_t* k;
  const uint16_t* v;
  const int32_t* seq_idx;
  const int32_t* pos;
  const int32_t* rope_pos;
  const float2* rope;
  const float* k_shift;
  uint16_t* q_out;
  int64_t ld_q, ld_k, ld_v;
  uint32_t axes;
  uint32_t axis_bits[4];  // two bits per channel pair
  uint32_t n_new, hq, heads;  // heads: hq + 2 * hkv
  FastDiv split;              // lane groups of a token; a group takes heads g, g + split, ...
  uint32_t rope_positions;
  float gk, gv;
  int* status;
};

// Eight lanes hold one 128-channel row: lane c has channels 8c..8c+7 and
// 64+8c..64+8c+7, so a rotation needs no other lane's values, and a lane pair
// (2i, 2i+1) has the two 16-element blocks i and 4+i.  The lane group keeps the
// (cos, sin) of its token in registers for all heads that it takes.
//
// HBM-bound at prompt sizes: a token reads 256 bytes for each of its heads and writes
// 256 (Q) or 72 (K, V), and its table rows come from L2.  The next head's loads are
// issued before a head is rotated (8192 tokens of 64 + 2 x 8 heads 61 -> 55 us, 84 % of the
// measured copy rate; 64 us with the 70 registers that the compiler would take, three CTAs
// an SM instead of four).
template <bool kE1M2>
__global__ void __launch_bounds__(kThreads, 4) append_axes_kernel(const AppendArgs a) {
  griddep_wait_and_release();
  const uint32_t group = (blockIdx.x * kThreads + threadIdx.x) >> 3, c = threadIdx.x & 7;
  const uint32_t tok_raw = a.split.div(group);
  const bool live = tok_raw < a.n_new;
  const uint32_t tok = live ? tok_raw : 0;
  const uint32_t h0 = group - tok_raw * a.split.d;
  const int32_t b = __ldg(a.seq_idx + tok), p = __ldg(a.pos + tok);
  uint32_t rp[kMaxAxes];
  bool rotary_ok = true;
#pragma unroll
  for (int x = 0; x < kMaxAxes; ++x) {
    rp[x] = x < static_cast<int>(a.axes) ? static_cast<uint32_t>(__ldg(a.rope_pos + static_cast<uint64_t>(tok) * a.axes + x)) : 0u;
    rotary_ok = rotary_ok && rp[x] < a.rope_positions;
  }
  bool stored = live && static_cast<uint32_t>(b) < a.map.batch && static_cast<uint32_t>(p) < a.map.context;
  const int64_t row0 = stored ? a.map.row(b, p) : -1;
  stored = row0 >= 0 && rotary_ok;
  if (live && !stored && h0 == 0 && c == 0) set_status(a.status, NVFP4_ERR_CAPACITY);

  float2 cs[8];
  const uint32_t bits = a.axis_bits[c >> 1] >> ((c & 1) * 16);  // of pairs 8c..8c+7
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t x = (bits >> (2 * i)) & 3u;
    const uint32_t r = x == 0 ? rp[0] : x == 1 ? rp[1] : x == 2 ? rp[2] : rp[3];
    cs[i] = rotary_ok ? __ldg(a.rope + static_cast<uint64_t>(r) * 64 + 8 * c + i) : make_float2(0.0f, 0.0f);
  }
  const float qmax = kE1M2 ? 3.5f : 6.0f;
  const float max_k = __fmul_rn(qmax, a.gk), max_v = __fmul_rn(qmax, a.gv);

  // The lane's 2 x 16 bytes of head h; of a query off the rotary table zeros, whatever it holds.
  const auto load = [&](uint32_t h, uint4* lo, uint4* hi) {
    *lo = *hi = make_uint4(0, 0, 0, 0);
    if (!live || h >= a.heads || (!rotary_ok && h < a.hq)) return;
    const uint16_t* src = h < a.hq               ? a.q + tok * a.ld_q + h * 128u
                          : h < a.hq + a.map.hkv ? a.k + tok * a.ld_k + (h - a.hq) * 128u
                                                 : a.v + tok * a.ld_v + (h - a.hq - a.map.hkv) * 128u;
    *lo = __ldg(reinterpret_cast<const uint4*>(src) + c);
    *hi = __ldg(reinterpret_cast<const uint4*>(src) + 8 + c);
  };
  uint4 next_lo, next_hi;
  load(h0, &next_lo, &next_hi);
  // Every lane of the warp makes the same number of turns (the amax shuffles).
  for (uint32_t turn = 0; turn < a.heads; turn += a.split.d) {
    const uint32_t h = h0 + turn;
    const bool in = live && h < a.heads;
    const bool is_q = h < a.hq, is_k = !is_q && h < a.hq + a.map.hkv;
    const uint32_t kvh = is_q ? 0 : h - a.hq - (is_k ? 0 : a.map.hkv);
    const uint4 lo = next_lo, hi = next_hi;
    load(h + a.split.d, &next_lo, &next_hi);
    float x[8], y[8];
    unpack_bf16x8(lo, x);
    unpack_bf16x8(hi, y);
    if (is_q || is_k) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = __fsub_rn(__fmul_rn(x[i], cs[i].x), __fmul_rn(y[i], cs[i].y));
        y[i] = __fadd_rn(__fmul_rn(x[i], cs[i].y), __fmul_rn(y[i], cs[i].x));
        x[i] = u;
      }
    }
    if (in && is_q) {
      uint4* dst = reinterpret_cast<uint4*>(a.q_out + (static_cast<uint64_t>(tok) * a.hq + h) * 128);
      dst[c] = make_uint4(bf16x2_rn(x[0], x[1]), bf16x2_rn(x[2], x[3]), bf16x2_rn(x[4], x[5]), bf16x2_rn(x[6], x[7]));
      dst[8 + c] = make_uint4(bf16x2_rn(y[0], y[1]), bf16x2_rn(y[2], y[3]), bf16x2_rn(y[4], y[5]), bf16x2_rn(y[6], y[7]));
    }
    if (!__any_sync(0xffffffffu, in && !is_q)) continue;
    if (is_k && a.k_shift) {
      const float* m = a.k_shift + kvh * 128u + 8 * c;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = __fsub_rn(x[i], __ldg(m + i));
        y[i] = __fsub_rn(y[i], __ldg(m + 64 + i));
      }
    }
    float ax = 0.0f, ay = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      ax = fmaxf(ax, fabsf(x[i]));
      ay = fmaxf(ay, fabsf(y[i]));
    }
    const float g = is_k ? a.gk : a.gv, top = is_k ? max_k : max_v;
    uint32_t sx, sy;
    const uint32_t wx = quantize8_pair<kE1M2>(x, ax, g, top, &sx);
    const uint32_t wy = quantize8_pair<kE1M2>(y, ay, g, top, &sy);
    if (!in || is_q || !stored) continue;
    const uint64_t row = static_cast<uint64_t>(row0) + static_cast<uint64_t>(kvh) * a.map.size.d;
    if (!in_bounds(a.status, row < static_cast<uint64_t>(a.map.pages) * a.map.hkv * a.map.size.d)) continue;
    uint32_t* codes = reinterpret_cast<uint32_t*>((is_k ? a.kc : a.vc) + row * 64);
    codes[c] = wx;
    codes[8 + c] = wy;
    if ((c & 1) == 0) {
      uint8_t* scales = (is_k ? a.ks : a.vs) + row * 8;
      scales[c >> 1] = static_cast<uint8_t>(sx);
      scales[4 + (c >> 1)] = static_cast<uint8_t>(sy);
    }
  }
}

struct ReadArgs {
  KVMap map;
  const int32_t* seq_idx;
  const int32_t* pos;
  uint4* k_out;
  uint4* v_out;
  uint64_t items;  // (token, head) rows
  FastDiv heads;
  float gk, gv;
  int* status;
};

template <bool kE1M2>
__device__ __forceinline__ uint4 read8(uint32_t codes, uint32_t scale, float g) {
  uint32_t e[4];
  elements8<kE1M2>(codes, e);
  // e2m1 * e4m3 is exact in fp32; one rounding with g, one to bf16.
  const float s = kE1M2 ? e4m3_value(scale) * 0.5f : e4m3_value(scale);
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    o[i] = bf16x2_rn(__fmul_rn(__fmul_rn(f16_lo(e[i]), s), g), __fmul_rn(__fmul_rn(f16_hi(e[i]), s), g));
  return make_uint4(o[0], o[1], o[2], o[3]);
}

// Sixteen lanes hold one 128-channel row, eight elements each: 4 bytes of codes
// and a scale byte in, 16 bytes out, for K and V; kRowsAtOnce rows a lane group and
// turn, whose loads are in flight together.  HBM-bound: 72 bytes read and 256
// written per row (32 x 4096 tokens x 8 heads, K and V: 124 us, 82 % of the measured
// copy rate).
template <bool kE1M2, int kRowsAtOnce>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(const ReadArgs a) {
  griddep_wait_and_release();
  const uint32_t c = threadIdx.x & 15;
  constexpr uint64_t kRows = kThreads / 16 * kRowsAtOnce;  // of a CTA's turn
  for (uint64_t i0 = blockIdx.x * kRows + (threadIdx.x >> 4); i0 < a.items; i0 += gridDim.x * kRows) {
    int64_t row[kRowsAtOnce];
    uint32_t head[kRowsAtOnce];
#pragma unroll
    for (int u = 0; u < kRowsAtOnce; ++u) {
      const uint64_t i = i0 + u * (kThreads / 16);
      const bool in = i < a.items;
      const uint32_t tok = in ? a.heads.div(static_cast<uint32_t>(i)) : 0;
      head[u] = static_cast<uint32_t>(i) - tok * a.heads.d;
      const int32_t b = __ldg(a.seq_idx + tok), p = __ldg(a.pos + tok);
      row[u] = in && static_cast<uint32_t>(b) < a.map.batch && static_cast<uint32_t>(p) < a.map.context ? a.map.row(b, p) : -1;
      if (in && row[u] < 0 && head[u] == 0 && c == 0) set_status(a.status, NVFP4_ERR_CAPACITY);
    }
    uint32_t kc[kRowsAtOnce], ks[kRowsAtOnce], vc[kRowsAtOnce], vs[kRowsAtOnce];
#pragma unroll
    for (int u = 0; u < kRowsAtOnce; ++u) {
      const uint64_t r = static_cast<uint64_t>(row[u]) + static_cast<uint64_t>(head[u]) * a.map.size.d;
      const bool there = row[u] >= 0;
      kc[u] = there && a.k_out ? __ldg(reinterpret_cast<const uint32_t*>(a.map.k_codes + r * 64) + c) : 0u;
      ks[u] = there && a.k_out ? __ldg(a.map.k_scales + r * 8 + (c >> 1)) : 0u;
      vc[u] = there && a.v_out ? __ldg(reinterpret_cast<const uint32_t*>(a.map.v_codes + r * 64) + c) : 0u;
      vs[u] = there && a.v_out ? __ldg(a.map.v_scales + r * 8 + (c >> 1)) : 0u;
    }
#pragma unroll
    for (int u = 0; u < kRowsAtOnce; ++u) {
      const uint64_t i = i0 + u * (kThreads / 16);
      if (i >= a.items) break;
      const uint4 none = make_uint4(0, 0, 0, 0);
      if (a.k_out) a.k_out[i * 16 + c] = row[u] < 0 ? none : read8<kE1M2>(kc[u], ks[u], a.gk);
      if (a.v_out) a.v_out[i * 16 + c] = row[u] < 0 ? none : read8<kE1M2>(vc[u], vs[u], a.gv);
    }
  }
}

}  // namespace
}  // namespace nvfp4

using namespace nvfp4;

NVFP4_API nvfp4_status kv_append_rope_axes_nvfp4(const nvfp4_kv_cache* cache, const nvfp4_kv_pages* pages,
                                                 const void* q_bf16, int64_t ld_q, int32_t num_q_heads,
                                                 const void* k_bf16, int64_t ld_k, const void* v_bf16, int64_t ld_v,
                                                 const int32_t* seq_idx, const int32_t* pos, const int32_t* rope_pos,
                                                 int32_t n_axes, const uint8_t* axis_of_pair, int64_t n_new,
                                                 const float* rope_table, int64_t rope_positions,
                                                 const float* k_shift, void* q_out, void* stream) {
  NVFP4_TRACE("kv_append_rope_axes_nvfp4");
  AppendArgs a;
  const nvfp4_status st = kv_map(cache, pages, &a.map);
  if (st != NVFP4_OK) return st;
  if (n_new < 0) return NVFP4_ERR_SHAPE;
  if (n_new == 0) return NVFP4_OK;
  if (!k_bf16 || !v_bf16 || !seq_idx || !pos || !rope_pos || !axis_of_pair || !rope_table || (q_bf16 && !q_out))
    return NVFP4_ERR_INVALID_ARG;
  const int64_t hq = q_bf16 ? num_q_heads : 0, hkv = cache->num_kv_heads;
  if ((q_bf16 && num_q_heads < 1) || n_axes < 1 || n_axes > kMaxAxes || rope_positions < 1 ||
      rope_positions >= (1ll << 31) || hq > (1 << 20) || hkv > (1 << 20))
    return NVFP4_ERR_SHAPE;
  if (n_new > 1 && ((q_bf16 && ld_q < hq * 128) || ld_k < hkv * 128 || ld_v < hkv * 128)) return NVFP4_ERR_SHAPE;
  for (int i = 0; i < 4; ++i) a.axis_bits[i] = 0;
  for (int i = 0; i < 64; ++i) {
    if (axis_of_pair[i] >= n_axes) return NVFP4_ERR_INVALID_ARG;
    a.axis_bits[i >> 4] |= static_cast<uint32_t>(axis_of_pair[i]) << (2 * (i & 15));
  }
  if (!aligned(q_bf16, 16) || !aligned(k_bf16, 16) || !aligned(v_bf16, 16) || !aligned(rope_table, 16) ||
      !aligned(k_shift, 16) || (q_bf16 && !aligned(q_out, 16)) || !aligned(seq_idx, 4) || !aligned(pos, 4) ||
      !aligned(rope_pos, 4) || (q_bf16 && ld_q % 8) || ld_k % 8 || ld_v % 8)
    return NVFP4_ERR_ALIGN;
  a.kc = cache->k_codes;
  a.ks = cache->k_scales;
  a.vc = cache->v_codes;
  a.vs = cache->v_scales;
  a.q = static_cast<const uint16_t*>(q_bf16);
  a.k = static_cast<const uint16_t*>(k_bf16);
  a.v = static_cast<const uint16_t*>(v_bf16);
  a.seq_idx = seq_idx;
  a.pos = pos;
  a.rope_pos = rope_pos;
  a.rope = reinterpret_cast<const float2*>(rope_table);
  a.k_shift = k_shift;
  a.q_out = static_cast<uint16_t*>(q_out);
  a.ld_q = ld_q;
  a.ld_k = ld_k;
  a.ld_v = ld_v;
  a.axes = static_cast<uint32_t>(n_axes);
  a.hq = static_cast<uint32_t>(hq);
  a.heads = static_cast<uint32_t>(hq + 2 * hkv);
  a.rope_positions = static_cast<uint32_t>(rope_positions);
  a.gk = cache->k_gscale;
  a.gv = cache->v_gscale;
  a.status = status_word_dev();
  // Lane groups per token: one head each while that leaves SMs without work, else
  // four, which then share the token's table rows over several heads (8192 tokens of
  // 64 + 2 x 8 heads: 2 groups 55.2, 4 groups 54.6, 8 groups 56.8, 20 groups 71.7 us).
  const uint64_t one_each = static_cast<uint64_t>(n_new) * a.heads * 8;
  const uint32_t split = one_each <= static_cast<uint64_t>(sm_count()) * 2048 || a.heads < 4 ? a.heads : 4;
  const uint64_t groups = static_cast<uint64_t>(n_new) * split;
  if (n_new >= (1ll << 31) || groups >= (1ull << 29)) return NVFP4_ERR_SHAPE;
  a.n_new = static_cast<uint32_t>(n_new);
  a.split = FastDiv(split);
  const uint32_t grid = static_cast<uint32_t>((groups * 8 + kThreads - 1) / kThreads);
  const auto kernel = cache->kv_format == NVFP4_KV_E1M2 ? append_axes_kernel<true> : append_axes_kernel<false>;
  if (launch_pdl(kernel, dim3(grid), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), a) != cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}

NVFP4_API nvfp4_status kv_read_nvfp4(const nvfp4_kv_cache* cache, const nvfp4_kv_pages* pages, const int32_t* seq_idx,
                                     const int32_t* pos, int64_t n, void* k_out, void* v_out, void* stream) {
  NVFP4_TRACE("kv_read_nvfp4");
  ReadArgs a;
  const nvfp4_status st = kv_map(cache, pages, &a.map);
  if (st != NVFP4_OK) return st;
  if (n < 0) return NVFP4_ERR_SHAPE;
  if (n == 0) return NVFP4_OK;
  if (!seq_idx || !pos || (!k_out && !v_out)) return NVFP4_ERR_INVALID_ARG;
  if (n >= (1ll << 31) || n * cache->num_kv_heads >= (1ll << 31)) return NVFP4_ERR_SHAPE;
  if (!aligned(seq_idx, 4) || !aligned(pos, 4) || !aligned(k_out, 16) || !aligned(v_out, 16)) return NVFP4_ERR_ALIGN;
  a.seq_idx = seq_idx;
  a.pos = pos;
  a.k_out = static_cast<uint4*>(k_out);
  a.v_out = static_cast<uint4*>(v_out);
  a.items = static_cast<uint64_t>(n) * cache->num_kv_heads;
  a.heads = FastDiv(static_cast<uint32_t>(cache->num_kv_heads));
  a.gk = cache->k_gscale;
  a.gv = cache->v_gscale;
  a.status = status_word_dev();
  // Four rows at once where there are enough for every SM (32 x 4096 tokens x 8 heads
  // 144 -> 124 us), one where the latency of few is the time (1000 x 2: 3.6 -> 2.1 us).
  const bool e1m2 = cache->kv_format == NVFP4_KV_E1M2, many = a.items >= static_cast<uint64_t>(sm_count()) * 256;
  const uint64_t kRows = kThreads / 16 * (many ? 4 : 1);
  const uint64_t grid = (a.items + kRows - 1) / kRows;
  const auto kernel = many ? (e1m2 ? kv_read_kernel<true, 4> : kv_read_kernel<false, 4>)
                           : (e1m2 ? kv_read_kernel<true, 1> : kv_read_kernel<false, 1>);
  if (launch_pdl(kernel, dim3(static_cast<uint32_t>(grid)), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), a) !=
      cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}
