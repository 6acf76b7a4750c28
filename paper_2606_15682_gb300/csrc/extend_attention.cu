// Attention of new tokens (one, a few, a chunk, a whole prompt) over the 4-bit
// cache that already holds them, contiguous or paged: scores optionally capped
// and biased by distance, keys limited by causality, window, prefix, document.
#include "kv_pages.cuh"

namespace nvfp4 {
namespace {

constexpr int kD = 128;
constexpr float kLog2e = 1.4426950408889634f;

struct ExtendArgs {
  KVMap map;
  const uint16_t* q;
  uint16_t* out;
  const int32_t* q_start;  // null: `uniform` tokens per sequence
  const float* slopes;
  const int32_t* prefix_lens;
  const int32_t* doc_start;
  int64_t ld_q;
  uint32_t n_tokens, uniform, hq;
  FastDiv group;
  int window;
  float scale;  // softmax_scale * g_K
  float cap;
  float gv;
  int* status;
};

// Tokens of sequence b: its first query, how many, and its cached length.
struct Seq {
  uint32_t first, n;
  int len;
};
__device__ __forceinline__ Seq sequence(const ExtendArgs& a, uint32_t b) {
  Seq s;
  bool bad = false;
  if (a.q_start) {
    const int32_t lo = __ldg(a.q_start + b), hi = __ldg(a.q_start + b + 1), n = static_cast<int32_t>(a.n_tokens);
    const int32_t l = max(0, min(lo, n)), h = max(l, min(hi, n));
    bad = l != lo || h != hi;
    s.first = static_cast<uint32_t>(l);
    s.n = static_cast<uint32_t>(h - l);
  } else {
    s.first = b * a.uniform;
    s.n = a.uniform;
  }
  const int32_t len = __ldg(a.map.seq_lens + b);
  s.len = max(0, min(len, static_cast<int32_t>(a.map.context)));
  if (bad || s.len != len) set_status(a.status, NVFP4_ERR_CAPACITY);
  return s;
}

// Keys that the query at position p sees: [lo, hi).
__device__ __forceinline__ int2 visible(const ExtendArgs& a, int p, int len, int prefix, int doc) {
  int lo = max(doc, 0);
  if (a.window) lo = max(lo, p - a.window + 1);
  return make_int2(lo, min(len, max(p + 1, prefix)));
}

// One CTA per (token, query head): scores of 128 keys, a thread each, then the
// weighted sum of V, a channel per thread.
template <bool kE1M2>
__global__ void __launch_bounds__(kD) extend_simple_kernel(const ExtendArgs a) {
  __shared__ float q_sh[kD], p_sh[kD], red[4];
  __shared__ int64_t row_sh[kD];
  griddep_wait_and_release();
  const uint32_t tok = blockIdx.x, h = blockIdx.y, kvh = a.group.div(h);
  uint32_t b = 0;
  Seq s = sequence(a, 0);
  while (tok >= s.first + s.n && b + 1 < a.map.batch) s = sequence(a, ++b);
  const bool mine = tok >= s.first && tok < s.first + s.n;
  const int p = s.len - static_cast<int>(s.n) + static_cast<int>(tok - s.first);
  const int2 v = visible(a, p, s.len, a.prefix_lens ? __ldg(a.prefix_lens + b) : 0, a.doc_start ? __ldg(a.doc_start + tok) : 0);
  const int c = threadIdx.x, lane = c & 31, warp = c >> 5;
  q_sh[c] = __uint_as_float(static_cast<uint32_t>(a.q[tok * a.ld_q + h * kD + c]) << 16);
  const float slope = a.slopes ? __ldg(a.slopes + h) : 0.0f;
  float m = -INFINITY, l = 0.0f, o = 0.0f;
  const int end = mine && p >= 0 ? v.y : 0;
  for (int t0 = v.x; t0 < end; t0 += kD) {
    __syncthreads();
    const int t = t0 + c;
    float x = -INFINITY;
    int64_t row = -1;
    if (t < end) row = a.map.row(b, t);
    if (row >= 0) {
      row += static_cast<int64_t>(kvh) * a.map.size.d;
      x = 0.0f;
      for (int i = 0; i < 16; ++i) {
        uint32_t e[4];
        elements8<kE1M2>(__ldg(reinterpret_cast<const uint32_t*>(a.map.k_codes + row * 64) + i), e);
        const float sc = e4m3_value(__ldg(a.map.k_scales + row * 8 + (i >> 1))) * (kE1M2 ? 0.5f : 1.0f);
        float part = 0.0f;
        for (int k = 0; k < 4; ++k) part += f16_lo(e[k]) * q_sh[8 * i + 2 * k] + f16_hi(e[k]) * q_sh[8 * i + 2 * k + 1];
        x += part * sc;
      }
      x *= a.scale;
      if (a.cap > 0.0f) x = a.cap * tanhf(x / a.cap);
      x -= slope * static_cast<float>(abs(p - t));
    }
    float mx = x;
    for (int sh = 16; sh; sh >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, sh));
    if (lane == 0) red[warp] = mx;
    row_sh[c] = row;
    __syncthreads();
    const float m_new = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    p_sh[c] = row >= 0 ? exp2f((x - m_new) * kLog2e) : 0.0f;
    __syncthreads();
    const float shrink = m_new == -INFINITY ? 1.0f : exp2f((m - m_new) * kLog2e);
    m = m_new;
    o *= shrink;
    l *= shrink;
    for (int k = 0; k < min(kD, end - t0); ++k) {
      const int64_t r = row_sh[k];
      if (r < 0) continue;
      uint32_t e[4];
      elements8<kE1M2>(__ldg(a.map.v_codes + r * 64 + (c >> 1)), e);
      const float sc = e4m3_value(__ldg(a.map.v_scales + r * 8 + (c >> 4))) * (kE1M2 ? 0.5f : 1.0f);
      o += p_sh[k] * ((c & 1) ? f16_hi(e[0]) : f16_lo(e[0])) * sc;
      l += p_sh[k];
    }
  }
  const uint32_t bits = bf16x2_rn(l > 0.0f ? o / l * a.gv : 0.0f, 0.0f);
  a.out[(static_cast<uint64_t>(tok) * a.hq + h) * kD + c] = static_cast<uint16_t>(bits);
}

}  // namespace
}  // namespace nvfp4

using namespace nvfp4;

NVFP4_API size_t extend_attention_nvfp4_workspace_size(int32_t batch, int64_t n_tokens, int32_t num_q_heads,
                                                       int32_t num_kv_heads, int64_t context) {
  (void)batch, (void)n_tokens, (void)num_q_heads, (void)num_kv_heads, (void)context;
  return 0;
}

NVFP4_API nvfp4_status extend_attention_nvfp4(const nvfp4_kv_cache* cache, const nvfp4_kv_pages* pages,
                                              const void* q_bf16, int64_t ld_q, int64_t n_tokens, int32_t num_q_heads,
                                              const int32_t* q_start, const nvfp4_attention_options* options,
                                              void* out_bf16, void* workspace, size_t workspace_bytes, void* stream) {
  NVFP4_TRACE("extend_attention_nvfp4");
  ExtendArgs a;
  const nvfp4_status st = kv_map(cache, pages, &a.map);
  if (st != NVFP4_OK) return st;
  if (!options || !a.map.seq_lens) return NVFP4_ERR_INVALID_ARG;
  if (!(options->softmax_scale > 0.0f && options->softmax_scale <= FLT_MAX) ||
      !(options->logit_cap >= 0.0f && options->logit_cap <= FLT_MAX) || options->window < 0)
    return NVFP4_ERR_INVALID_ARG;
  if (n_tokens < 0 || n_tokens >= (1ll << 31) || num_q_heads <= 0 || num_q_heads > 65535 ||
      num_q_heads % cache->num_kv_heads || (!q_start && n_tokens % a.map.batch))
    return NVFP4_ERR_SHAPE;
  if (n_tokens == 0) return NVFP4_OK;
  if (!q_bf16 || !out_bf16) return NVFP4_ERR_INVALID_ARG;
  if (n_tokens > 1 && ld_q < static_cast<int64_t>(num_q_heads) * kD) return NVFP4_ERR_SHAPE;
  const size_t need = extend_attention_nvfp4_workspace_size(static_cast<int32_t>(a.map.batch), n_tokens, num_q_heads,
                                                            cache->num_kv_heads, a.map.context);
  if (need && !workspace) return NVFP4_ERR_INVALID_ARG;
  if (workspace_bytes < need) return NVFP4_ERR_SHAPE;
  if (!aligned(q_bf16, 16) || !aligned(out_bf16, 16) || ld_q % 8 || (need && !aligned(workspace, 16)) ||
      !aligned(a.map.seq_lens, 4) || !aligned(q_start, 4) || !aligned(options->slopes, 4) ||
      !aligned(options->prefix_lens, 4) || !aligned(options->doc_start, 4))
    return NVFP4_ERR_ALIGN;
  a.q = static_cast<const uint16_t*>(q_bf16);
  a.out = static_cast<uint16_t*>(out_bf16);
  a.q_start = q_start;
  a.slopes = options->slopes;
  a.prefix_lens = options->prefix_lens;
  a.doc_start = options->doc_start;
  a.ld_q = ld_q;
  a.n_tokens = static_cast<uint32_t>(n_tokens);
  a.uniform = static_cast<uint32_t>(n_tokens / a.map.batch);
  a.hq = static_cast<uint32_t>(num_q_heads);
  a.group = FastDiv(static_cast<uint32_t>(num_q_heads / cache->num_kv_heads));
  a.window = options->window;
  a.scale = options->softmax_scale * cache->k_gscale;
  a.cap = options->logit_cap;
  a.gv = cache->v_gscale;
  a.status = status_word_dev();
  const auto kernel = cache->kv_format == NVFP4_KV_E1M2 ? extend_simple_kernel<true> : extend_simple_kernel<false>;
  if (launch_pdl(kernel, dim3(a.n_tokens, a.hq), dim3(kD), 0, static_cast<cudaStream_t>(stream), a) != cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}
