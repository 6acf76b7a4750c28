// Addressing of a KV cache that may be paged, and its element grids, shared by
// the calls that take nvfp4_kv_pages.
#pragma once

#include <cfloat>

#include "common.cuh"
#include "nvfp4_quant.cuh"

namespace nvfp4 {

// Where token t of sequence b is: row t % size of page table[b, t / size]; a
// contiguous cache is one page per sequence, table[b, 0] = b.
struct KVMap {
  const uint8_t* k_codes;
  const uint8_t* k_scales;
  const uint8_t* v_codes;
  const uint8_t* v_scales;
  const int32_t* table;  // null: contiguous
  const int32_t* seq_lens;
  uint32_t batch, hkv, pages, per_seq;
  uint32_t context;  // tokens that a sequence can hold
  FastDiv size;      // tokens of a page

  // Row index (of the [page, head, token] rows) of head 0's token t, or -1
  // where the page is absent; head h's row is `size.d` rows times h further.
  // b < batch and t < context are the caller's checks.
  __device__ __forceinline__ int64_t row(uint32_t b, uint32_t t) const {
    if (!table) return static_cast<int64_t>(b) * hkv * size.d + t;
    const uint32_t i = size.div(t);
    const int32_t page = __ldg(table + static_cast<uint64_t>(b) * per_seq + i);
    if (static_cast<uint32_t>(page) >= pages) return -1;
    return static_cast<int64_t>(page) * hkv * size.d + (t - i * size.d);
  }
};

// Checks of the cache and its pages that every such call makes, and the map.
inline nvfp4_status kv_map(const nvfp4_kv_cache* cache, const nvfp4_kv_pages* pages, KVMap* m) {
  if (!cache || !cache->k_codes || !cache->k_scales || !cache->v_codes || !cache->v_scales ||
      (pages && !pages->table))
    return NVFP4_ERR_INVALID_ARG;
  if (!(cache->k_gscale > 0.0f && cache->k_gscale <= FLT_MAX) || !(cache->v_gscale > 0.0f && cache->v_gscale <= FLT_MAX))
    return NVFP4_ERR_INVALID_ARG;
  if (cache->kv_format != NVFP4_KV_E2M1 && cache->kv_format != NVFP4_KV_E1M2) return NVFP4_ERR_INVALID_ARG;
  if (cache->head_dim != 128 || cache->batch <= 0 || cache->num_kv_heads <= 0 || cache->capacity <= 0 ||
      (pages && (pages->batch <= 0 || pages->pages_per_seq <= 0)))
    return NVFP4_ERR_SHAPE;
  const int64_t context = static_cast<int64_t>(cache->capacity) * (pages ? pages->pages_per_seq : 1);
  if (context >= (1ll << 31) - 512) return NVFP4_ERR_SHAPE;  // block ends stay within 32 bits
  if (!aligned(cache->k_codes, 16) || !aligned(cache->v_codes, 16) || !aligned(cache->k_scales, 8) ||
      !aligned(cache->v_scales, 8) || (pages && !aligned(pages->table, 4)))
    return NVFP4_ERR_ALIGN;
  m->k_codes = cache->k_codes;
  m->k_scales = cache->k_scales;
  m->v_codes = cache->v_codes;
  m->v_scales = cache->v_scales;
  m->table = pages ? pages->table : nullptr;
  m->seq_lens = pages ? pages->seq_lens : cache->seq_lens;
  m->batch = static_cast<uint32_t>(pages ? pages->batch : cache->batch);
  m->hkv = static_cast<uint32_t>(cache->num_kv_heads);
  m->pages = static_cast<uint32_t>(cache->batch);
  m->per_seq = static_cast<uint32_t>(pages ? pages->pages_per_seq : 1);
  m->context = static_cast<uint32_t>(context);
  m->size = FastDiv(static_cast<uint32_t>(cache->capacity));
  return NVFP4_OK;
}

// Two E4M3 bytes (low byte -> low half) -> f16x2, exact.
__device__ __forceinline__ uint32_t e4m3x2_f16x2(uint32_t two_bytes) {
  uint32_t h;
  asm("{\n .reg .b16 s;\n cvt.u16.u32 s, %1;\n cvt.rn.f16x2.e4m3x2 %0, s;\n}" : "=r"(h) : "r"(two_bytes));
  return h;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ uint32_t sub_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// The eight elements of a code word as four f16x2 in order: e[i] = (2i, 2i+1).
// E2M1: the values.  E1M2 (two's-complement nibble n, value n / 2): n; a byte's
// two nibbles n ^ 8 are set into the low mantissa bits of 1024, from which 1032
// is taken away.  The missing 1/2 goes into the block scale (kv_scale16).
template <bool kE1M2>
__device__ __forceinline__ void elements8(uint32_t w, uint32_t e[4]) {
  if (kE1M2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t b = (w >> (8 * i)) & 0xFFu;
      e[i] = sub_f16x2(((b & 0xFu) | (b & 0xF0u) << 12) ^ 0x64086408u, 0x64086408u);
    }
  } else {
    asm("{\n .reg .b8 b0, b1, b2, b3;\n mov.b32 {b0, b1, b2, b3}, %4;\n"
        " cvt.rn.f16x2.e2m1x2 %0, b0;\n cvt.rn.f16x2.e2m1x2 %1, b1;\n"
        " cvt.rn.f16x2.e2m1x2 %2, b2;\n cvt.rn.f16x2.e2m1x2 %3, b3;\n}"
        : "=r"(e[0]), "=r"(e[1]), "=r"(e[2]), "=r"(e[3])
        : "r"(w));
  }
}
// The f16 factor of elements8's results for a pair of scale bytes: e4m3, or
// e4m3 / 2 (exact: the smallest E4M3 scale is 2^-9) for E1M2.
template <bool kE1M2>
__device__ __forceinline__ uint32_t kv_scales16(uint32_t two_bytes) {
  const uint32_t s = e4m3x2_f16x2(two_bytes);
  return kE1M2 ? mul_f16x2(s, 0x38003800u) : s;
}

__device__ __forceinline__ float f16_lo(uint32_t h) {
  float f;
  asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.f32.f16 %0, lo;\n}" : "=f"(f) : "r"(h));
  return f;
}
__device__ __forceinline__ float f16_hi(uint32_t h) {
  float f;
  asm("{\n .reg .b16 lo, hi;\n mov.b32 {lo, hi}, %1;\n cvt.f32.f16 %0, hi;\n}" : "=f"(f) : "r"(h));
  return f;
}
__device__ __forceinline__ uint32_t bf16x2_rn(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

}  // namespace nvfp4
