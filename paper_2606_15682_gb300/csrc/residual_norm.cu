// The norms around a block's residual sum in one pass over the row:
//   z = y [rms-normed * w_post] [* gate];  r = x + alpha z;  h = rms(r) * w_norm
// and h quantized to NVFP4 where the next linear reads it so.
//
// One CTA per row; the row stays in registers as fp32 between the two norms
// (each thread holds kVec groups of 8 channels), so every input is read once
// and every output written once.  HBM-bound at prompt sizes: 8 bytes per
// element with bf16 outputs (r, h), 6.56 with h in NVFP4 only: 8192 x 5120 with a
// post-norm and a gate, 62 us, 0.80 of the measured copy rate, and without them but with h
// in NVFP4 alone 56 us, 0.73; 32 rows 2.1 us (NVFP4 3.2), a launch's latency.  (Persistent CTAs that load the next row early: 133 us; w_post,
// gate and w_norm loaded with the row: 64 to 82 us, by their registers.)
#include "common.cuh"
#include "nvfp4_quant.cuh"

#include <cfloat>

namespace nvfp4 {
namespace {

struct NormArgs {
  const uint16_t* x;
  const uint16_t* y;
  const uint16_t* w_post;
  const uint16_t* gate;
  const uint16_t* w_norm;
  uint16_t* r_out;
  uint16_t* h_out;
  const float* g_out;
  uint8_t* codes;
  uint8_t* scales;
  int64_t ld_x, ld_y, rows, rows_per_gate;
  uint32_t cols;
  float alpha, eps;
  int* status;
};

__device__ __forceinline__ uint32_t pack_rn(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// Sum over the CTA's threads; every thread gets it.  sh: one float per warp,
// for this sum alone.
__device__ __forceinline__ float block_sum(float v, float* sh, int warps) {
#pragma unroll
  for (int s = 16; s; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
  if (warps == 1) return v;
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  float t = static_cast<int>(threadIdx.x & 31) < warps ? sh[threadIdx.x & 31] : 0.0f;
#pragma unroll
  for (int s = 16; s; s >>= 1) t += __shfl_xor_sync(0xffffffffu, t, s);
  return t;
}

template <int kVec>
__global__ void __launch_bounds__(1024) residual_norm_kernel(const NormArgs a) {
  __shared__ float sh[2][32];
  griddep_wait_and_release();
  const int warps = blockDim.x >> 5;
  const uint32_t vecs = a.cols >> 3;  // groups of 8 channels
  const int64_t row = blockIdx.x;
  const uint4* x4 = reinterpret_cast<const uint4*>(a.x + row * a.ld_x);
  const uint4* y4 = reinterpret_cast<const uint4*>(a.y + row * a.ld_y);
  const uint4 zero = make_uint4(0, 0, 0, 0);
  uint4 xin[kVec], yin[kVec];
#pragma unroll
  for (int k = 0; k < kVec; ++k) {
    const uint32_t i = threadIdx.x + k * blockDim.x;
    xin[k] = i < vecs ? x4[i] : zero;  // not __ldg: r_out may be x
    yin[k] = a.y && i < vecs ? __ldg(y4 + i) : zero;
  }
  float r[kVec][8];
#pragma unroll
  for (int k = 0; k < kVec; ++k) unpack_bf16x8(yin[k], r[k]);
  if (a.w_post) {
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < kVec; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) s += r[k][e] * r[k][e];
    const float inv = rsqrtf(block_sum(s, sh[0], warps) / static_cast<float>(a.cols) + a.eps);
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const uint32_t i = threadIdx.x + k * blockDim.x;
      float w[8];
      unpack_bf16x8(i < vecs ? __ldg(reinterpret_cast<const uint4*>(a.w_post) + i) : zero, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) r[k][e] *= inv * w[e];
    }
  }
  if (a.gate) {
    const uint4* g4 = reinterpret_cast<const uint4*>(a.gate + row / a.rows_per_gate * a.cols);
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
      const uint32_t i = threadIdx.x + k * blockDim.x;
      float g[8];
      unpack_bf16x8(i < vecs ? __ldg(g4 + i) : zero, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) r[k][e] *= g[e];
    }
  }
#pragma unroll
  for (int k = 0; k < kVec; ++k) {
    const uint32_t i = threadIdx.x + k * blockDim.x;
    float x[8];
    unpack_bf16x8(xin[k], x);
#pragma unroll
    for (int e = 0; e < 8; ++e) r[k][e] = a.y ? fmaf(a.alpha, r[k][e], x[e]) : x[e];
    if (a.r_out && i < vecs)
      reinterpret_cast<uint4*>(a.r_out + row * a.cols)[i] =
          make_uint4(pack_rn(r[k][0], r[k][1]), pack_rn(r[k][2], r[k][3]), pack_rn(r[k][4], r[k][5]),
                     pack_rn(r[k][6], r[k][7]));
  }
  if (!a.w_norm) return;

  float s = 0.0f;
#pragma unroll
  for (int k = 0; k < kVec; ++k)
#pragma unroll
    for (int e = 0; e < 8; ++e) s += r[k][e] * r[k][e];
  const float inv = rsqrtf(block_sum(s, sh[1], warps) / static_cast<float>(a.cols) + a.eps);
  float g = 1.0f;
  bool g_ok = true;
  if (a.codes) {
    g = __ldg(a.g_out);
    g_ok = g > 0.0f && g <= FLT_MAX;
    if (!g_ok && row == 0 && threadIdx.x == 0) set_status(a.status, NVFP4_ERR_INVALID_ARG);
    if (!g_ok) g = 1.0f;
  }
#pragma unroll
  for (int k = 0; k < kVec; ++k) {
    const uint32_t i = threadIdx.x + k * blockDim.x;
    float w[8];
    unpack_bf16x8(i < vecs ? __ldg(reinterpret_cast<const uint4*>(a.w_norm) + i) : zero, w);
    const uint4 h = make_uint4(pack_rn(r[k][0] * inv * w[0], r[k][1] * inv * w[1]),
                               pack_rn(r[k][2] * inv * w[2], r[k][3] * inv * w[3]),
                               pack_rn(r[k][4] * inv * w[4], r[k][5] * inv * w[5]),
                               pack_rn(r[k][6] * inv * w[6], r[k][7] * inv * w[7]));
    if (a.h_out && i < vecs) reinterpret_cast<uint4*>(a.h_out + row * a.cols)[i] = h;
    if (a.codes) {  // whole warps: the lane pair (2j, 2j+1) has one 16-element block
      float v[8];
      unpack_bf16x8(h, v);
      uint32_t sc;
      const uint32_t codes =
          quantize8_pair(v, __uint_as_float(amax_bits_bf16x8(h) << 16), g, __fmul_rn(6.0f, g), &sc);
      // Scales of four blocks, 8 lanes, as the one word that the layout keeps together.
      uint32_t word = sc << (8 * ((threadIdx.x >> 1) & 3));
      word |= __shfl_xor_sync(0xffffffffu, word, 2);
      word |= __shfl_xor_sync(0xffffffffu, word, 4);
      if (i < vecs) {
        reinterpret_cast<uint32_t*>(a.codes + row * (a.cols >> 1))[i] = g_ok ? codes : 0;
        if ((i & 7) == 0) {
          const uint64_t off = mma_scale_offset(row, i >> 1, a.cols >> 6);
          if (in_bounds(a.status, off + 4 <= ((a.rows + 127) / 128) * 128 * (a.cols >> 4)))
            *reinterpret_cast<uint32_t*>(a.scales + off) = g_ok ? word : 0;
        }
      }
    }
  }
  if (a.codes) {
    // Padding rows of the last row tile hold zero scales; the last rows' CTAs share them.
    const int64_t padded = (a.rows + 127) / 128 * 128;
    for (int64_t pr = a.rows + row; pr < padded; pr += a.rows)
      for (uint32_t j = threadIdx.x; j < a.cols >> 6; j += blockDim.x)
        *reinterpret_cast<uint32_t*>(a.scales + mma_scale_offset(pr, 4 * j, a.cols >> 6)) = 0;
  }
}

}  // namespace
}  // namespace nvfp4

using namespace nvfp4;

NVFP4_API nvfp4_status residual_norm_nvfp4(const void* x_bf16, int64_t ld_x, const void* y_bf16, int64_t ld_y,
                                           int64_t rows, int64_t cols, const void* w_post, const void* gate,
                                           int64_t rows_per_gate, float alpha, const void* w_norm, float eps,
                                           void* r_out, void* h_out, const float* g_out, uint8_t* codes,
                                           uint8_t* scales, void* stream) {
  NVFP4_TRACE("residual_norm_nvfp4");
  const bool quant = codes || scales || g_out;
  if (!y_bf16) r_out = nullptr;
  if (rows < 0 || cols < 8 || cols > 32768 || cols % 8 || (quant && cols % 64) || (gate && y_bf16 && rows_per_gate < 1))
    return NVFP4_ERR_SHAPE;
  if (rows == 0) return NVFP4_OK;
  if (rows >= (1ll << 31)) return NVFP4_ERR_SHAPE;
  if (ld_x < cols || (y_bf16 && ld_y < cols)) return NVFP4_ERR_SHAPE;
  if (!x_bf16 || (quant && !(codes && scales && g_out)) || ((h_out || quant) && !w_norm) || (!r_out && !h_out && !quant))
    return NVFP4_ERR_INVALID_ARG;
  if (!(eps > 0.0f && eps <= FLT_MAX) || !(alpha >= -FLT_MAX && alpha <= FLT_MAX)) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(x_bf16, 16) || !aligned(y_bf16, 16) || !aligned(w_post, 16) || !aligned(gate, 16) ||
      !aligned(w_norm, 16) || !aligned(r_out, 16) || !aligned(h_out, 16) || !aligned(codes, 16) ||
      !aligned(scales, 4) || !aligned(g_out, 4) || ld_x % 8 || (y_bf16 && ld_y % 8))
    return NVFP4_ERR_ALIGN;
  NormArgs a;
  a.x = static_cast<const uint16_t*>(x_bf16);
  a.y = static_cast<const uint16_t*>(y_bf16);
  a.w_post = y_bf16 ? static_cast<const uint16_t*>(w_post) : nullptr;
  a.gate = y_bf16 ? static_cast<const uint16_t*>(gate) : nullptr;
  a.w_norm = h_out || quant ? static_cast<const uint16_t*>(w_norm) : nullptr;
  a.r_out = static_cast<uint16_t*>(r_out);
  a.h_out = static_cast<uint16_t*>(h_out);
  a.g_out = g_out;
  a.codes = codes;
  a.scales = scales;
  a.ld_x = ld_x;
  a.ld_y = ld_y;
  a.rows = rows;
  a.rows_per_gate = gate && y_bf16 ? rows_per_gate : 1;
  a.cols = static_cast<uint32_t>(cols);
  a.alpha = alpha;
  a.eps = eps;
  a.status = status_word_dev();
  const uint32_t vecs = a.cols / 8;
  const int vec = vecs <= 2048 ? 2 : 4;
  const uint32_t threads = ((vecs + vec - 1) / vec + 31) / 32 * 32;
  const auto kernel = vec == 2 ? residual_norm_kernel<2> : residual_norm_kernel<4>;
  if (launch_pdl(kernel, dim3(static_cast<uint32_t>(rows)), dim3(threads), 0, static_cast<cudaStream_t>(stream), a) !=
      cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}
