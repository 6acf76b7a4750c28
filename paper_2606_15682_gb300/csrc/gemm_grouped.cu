// The experts' linears: block-scaled FP4 x FP4 products of rows sorted by expert,
// each expert's rows with its own weight.
//   out[r, n] = bf16( g_a[e] g_w[e] sum_k a[r, k] w_e[n, k] ),  r among expert e's rows
// and the same for gate_up with h = SiLU(gate) up quantized in the epilogue.
//
// A 64 x 64 tile per CTA: both operands dequantized into shared memory as fp32,
// a thread has 4 x 4 sums.
#include <cfloat>

#include "moe_plan.cuh"
#include "nvfp4_quant.cuh"

namespace nvfp4 {
namespace {

constexpr int kTile = 64, kDepth = 32, kPitch = kTile + 4;

struct GroupedArgs {
  const int32_t* row_start;
  const int32_t* rows;
  const uint8_t* a_codes;
  const uint8_t* a_scales;
  const uint8_t* w_codes;
  const uint8_t* w_scales;
  const float* g_a;
  const float* g_w;
  const float* g_out;
  uint16_t* out;
  uint8_t* q_codes;
  uint8_t* q_scales;
  int64_t ldo;
  int experts, max_rows, N, K, g_a_step, g_out_step;
  bool mx;
  uint32_t q_mode;  // 0 NVFP4, 1 MXFP4, 2 MXFP4 after the block rotation
  int* status;
};

__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

__device__ __forceinline__ float e2m1_value(uint32_t c) {
  const uint32_t m = c & 7;
  const float v = m < 2 ? 0.5f * m : __uint_as_float((126 + (m >> 1)) << 23 | (m & 1) << 22);
  return c & 8 ? -v : v;
}

template <bool kSwiGLU>
__global__ void __launch_bounds__(256) grouped_simple_kernel(const GroupedArgs a) {
  __shared__ float sa[kDepth][kPitch], sw[kDepth][kPitch];
  __shared__ float tile[kTile][kTile + 1];
  griddep_wait_and_release();
  // The tile's expert: the last one that starts at or before it.
  const int r0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile;
  int lo = 0, hi = a.experts;  // row_start[lo] <= r0 < row_start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (__ldg(a.row_start + mid) <= r0) lo = mid; else hi = mid;
  }
  const ExpertRows er = expert_rows(a.row_start, a.rows, lo, a.max_rows);
  const int live = min(kTile, er.first + er.n - r0);
  if (r0 < er.first || live <= 0) return;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const uint32_t kgroups = a.K / 64;
  const uint64_t w_tile_bytes = static_cast<uint64_t>((a.N + 127) / 128) * 128 * (a.K / 16);
  const uint8_t* w_codes = a.w_codes + static_cast<uint64_t>(lo) * a.N * (a.K / 2);
  const uint8_t* w_scales = a.w_scales + lo * w_tile_bytes;
  auto scale = [&](uint32_t c) { return a.mx ? __uint_as_float(c ? c << 23 : 1u << 22) : e4m3_value(c); };
  float acc[4][4] = {};
  for (int k0 = 0; k0 < a.K; k0 += kDepth) {
    // 64 rows x 32 channels: 2 blocks of 16 a row; half of the threads load each operand.
    const int half = threadIdx.x >> 7, i = threadIdx.x & 127, r = i >> 1, b = i & 1;
    const int64_t row = half ? n0 + r : r0 + r;
    const bool ok = half ? row < a.N : r < live;
    uint2 c = make_uint2(0, 0);
    float s = 0.0f;
    if (ok) {
      c = *reinterpret_cast<const uint2*>((half ? w_codes : a.a_codes) + row * (a.K / 2) + (k0 + 16 * b) / 2);
      s = scale((half ? w_scales : a.a_scales)[mma_scale_offset(row, k0 / 16 + b, kgroups)]);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 16; ++e)
      (half ? sw : sa)[16 * b + e][r] = s * e2m1_value((e < 8 ? c.x >> (4 * e) : c.y >> (4 * (e - 8))) & 15);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDepth; ++k) {
      const float4 x = *reinterpret_cast<const float4*>(&sa[k][4 * ty]);
      const float4 w = *reinterpret_cast<const float4*>(&sw[k][4 * tx]);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[p][q] = fmaf(xs[p], ws[q], acc[p][q]);
    }
  }
  const float g = a.g_a ? __fmul_rn(__ldg(a.g_a + lo * a.g_a_step), __ldg(a.g_w + lo)) : 1.0f;
  if constexpr (!kSwiGLU) {
#pragma unroll
    for (int p = 0; p < 4; ++p)
      if (4 * ty + p < live && n0 + 4 * tx < a.N)
        *reinterpret_cast<uint2*>(a.out + static_cast<int64_t>(r0 + 4 * ty + p) * a.ldo + n0 + 4 * tx) =
            make_uint2(pack_pair(acc[p][0] * g, acc[p][1] * g), pack_pair(acc[p][2] * g, acc[p][3] * g));
  } else {
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
      for (int q = 0; q < 4; ++q) tile[4 * ty + p][4 * tx + q] = acc[p][q] * g;
    __syncthreads();
    if (static_cast<int>(threadIdx.x) >= live) return;
    // A thread has a row: 32 outputs of the tile's 16 gate, 16 up, 16 gate, 16 up rows.
    const int r = threadIdx.x;
    const uint32_t cols = a.N / 2, oc0 = n0 / 2;
    float h[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float gate = tile[r][32 * (i >> 4) + (i & 15)], up = tile[r][32 * (i >> 4) + 16 + (i & 15)];
      h[i] = gate / (1.0f + expf(-gate)) * up;
    }
    uint32_t code[2];
    if (a.q_mode == 0) {
      const float g_in = __ldg(a.g_out + lo * a.g_out_step);
      const bool g_ok = g_in > 0.0f && g_in <= FLT_MAX;
      if (!g_ok) set_status(a.status, NVFP4_ERR_INVALID_ARG);
      const float go = g_ok ? g_in : 1.0f;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float amax = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) amax = fmaxf(amax, fabsf(h[16 * b + i]));
        const BlockScale s = block_scale(amax, go, __fmul_rn(6.0f, go));
        code[b] = g_ok ? s.code : 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) h[16 * b + i] = g_ok ? __fmul_rn(h[16 * b + i], s.mult) : 0.0f;
      }
    } else {
      if (a.q_mode == 2) hadamard32(h);
      float amax = 0.0f;
#pragma unroll
      for (int i = 0; i < 32; ++i) amax = fmaxf(amax, fabsf(h[i]));
      code[0] = code[1] = mx_scale_code(amax);
#pragma unroll
      for (int i = 0; i < 32; ++i) h[i] = __fmul_rn(h[i], mx_inv_scale(code[0]));
    }
    const uint64_t row = r0 + r;
    *reinterpret_cast<uint4*>(a.q_codes + row * (cols / 2) + oc0 / 2) =
        make_uint4(e2m1x8(h), e2m1x8(h + 8), e2m1x8(h + 16), e2m1x8(h + 24));
    *reinterpret_cast<uint16_t*>(a.q_scales + mma_scale_offset(row, oc0 / 16, cols / 64)) =
        static_cast<uint16_t>(code[0] | code[1] << 8);
  }
}

nvfp4_status launch_grouped(const moe_plan* plan, GroupedArgs& a, bool swiglu, cudaStream_t s) {
  if (plan->n_tokens == 0) return NVFP4_OK;
  a.row_start = plan->row_start;
  a.rows = plan->rows;
  a.experts = plan->num_experts;
  a.max_rows = static_cast<int>(moe_rows_bound(plan->n_tokens, plan->top_k, plan->num_experts));
  a.status = status_word_dev();
  const dim3 grid((a.N + kTile - 1) / kTile, a.max_rows / kTile);
  if (launch_pdl(swiglu ? grouped_simple_kernel<true> : grouped_simple_kernel<false>, grid, dim3(256), 0, s, a) !=
      cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}

constexpr int64_t kMaxSide = 1ll << 20;  // N and K

// The operands' checks that all four calls share; g: whether there are tensor scales.
nvfp4_status check_operands(const moe_plan* plan, const GroupedArgs& a, int64_t N, int64_t K, bool g, int64_t n_step) {
  const nvfp4_status st = check_moe_plan(plan);
  if (st != NVFP4_OK) return st;
  if (!a.a_codes || !a.a_scales || !a.w_codes || !a.w_scales || (g && (!a.g_a || !a.g_w))) return NVFP4_ERR_INVALID_ARG;
  if ((a.g_a_step != 0 && a.g_a_step != 1) || (a.g_out_step != 0 && a.g_out_step != 1)) return NVFP4_ERR_INVALID_ARG;
  if (N <= 0 || K <= 0 || N > kMaxSide || K > kMaxSide || K % 256 || N % n_step) return NVFP4_ERR_SHAPE;
  if (plan->num_experts * ((N + 127) / 128) * (K / 32) >= (1ll << 31) || plan->num_experts * N >= (1ll << 31))
    return NVFP4_ERR_SHAPE;
  if (!aligned(a.a_codes, 16) || !aligned(a.a_scales, 16) || !aligned(a.w_codes, 16) || !aligned(a.w_scales, 16) ||
      !aligned(a.g_a, 4) || !aligned(a.g_w, 4))
    return NVFP4_ERR_ALIGN;
  return NVFP4_OK;
}

nvfp4_status linear(const moe_plan* plan, GroupedArgs a, int64_t N, int64_t K, void* out, int64_t ldo, void* stream) {
  const nvfp4_status st = check_operands(plan, a, N, K, !a.mx, 16);
  if (st != NVFP4_OK) return st;
  if (!out) return NVFP4_ERR_INVALID_ARG;
  if (ldo < N || ldo % 8) return NVFP4_ERR_SHAPE;
  if (!aligned(out, 16)) return NVFP4_ERR_ALIGN;
  a.out = static_cast<uint16_t*>(out);
  a.ldo = ldo;
  a.N = static_cast<int>(N);
  a.K = static_cast<int>(K);
  return launch_grouped(plan, a, false, static_cast<cudaStream_t>(stream));
}

nvfp4_status swiglu(const moe_plan* plan, GroupedArgs a, int64_t I, int64_t K, uint8_t* codes, uint8_t* scales,
                    void* stream) {
  const nvfp4_status st = check_operands(plan, a, 2 * I, K, !a.mx, 256);
  if (st != NVFP4_OK) return st;
  if (!codes || !scales || (!a.mx && !a.g_out)) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(codes, 16) || !aligned(scales, 4) || !aligned(a.g_out, 4)) return NVFP4_ERR_ALIGN;
  a.q_codes = codes;
  a.q_scales = scales;
  a.N = static_cast<int>(2 * I);
  a.K = static_cast<int>(K);
  return launch_grouped(plan, a, true, static_cast<cudaStream_t>(stream));
}

GroupedArgs operands(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* w_codes, const uint8_t* w_scales) {
  GroupedArgs a = {};
  a.a_codes = a_codes;
  a.a_scales = a_scales;
  a.w_codes = w_codes;
  a.w_scales = w_scales;
  return a;
}

}  // namespace
}  // namespace nvfp4

using namespace nvfp4;

NVFP4_API nvfp4_status nvfp4_linear_grouped(const moe_plan* plan, const uint8_t* a_codes, const uint8_t* a_scales,
                                            const float* g_a, int32_t g_a_step, const uint8_t* w_codes,
                                            const uint8_t* w_scales, const float* g_w, int64_t N, int64_t K,
                                            void* out_bf16, int64_t ldo, void* stream) {
  NVFP4_TRACE("nvfp4_linear_grouped");
  GroupedArgs a = operands(a_codes, a_scales, w_codes, w_scales);
  a.g_a = g_a;
  a.g_w = g_w;
  a.g_a_step = g_a_step;
  return linear(plan, a, N, K, out_bf16, ldo, stream);
}

NVFP4_API nvfp4_status mxfp4_linear_grouped(const moe_plan* plan, const uint8_t* a_codes, const uint8_t* a_scales,
                                            const uint8_t* w_codes, const uint8_t* w_scales, int64_t N, int64_t K,
                                            void* out_bf16, int64_t ldo, void* stream) {
  NVFP4_TRACE("mxfp4_linear_grouped");
  GroupedArgs a = operands(a_codes, a_scales, w_codes, w_scales);
  a.mx = true;
  return linear(plan, a, N, K, out_bf16, ldo, stream);
}

NVFP4_API nvfp4_status nvfp4_linear_grouped_swiglu_quantize(const moe_plan* plan, const uint8_t* a_codes,
                                                            const uint8_t* a_scales, const float* g_a,
                                                            int32_t g_a_step, const uint8_t* w_codes,
                                                            const uint8_t* w_scales, const float* g_w, int64_t I,
                                                            int64_t K, const float* g_out, int32_t g_out_step,
                                                            uint8_t* out_codes, uint8_t* out_scales, void* stream) {
  NVFP4_TRACE("nvfp4_linear_grouped_swiglu_quantize");
  GroupedArgs a = operands(a_codes, a_scales, w_codes, w_scales);
  a.g_a = g_a;
  a.g_w = g_w;
  a.g_a_step = g_a_step;
  a.g_out = g_out;
  a.g_out_step = g_out_step;
  return swiglu(plan, a, I, K, out_codes, out_scales, stream);
}

NVFP4_API nvfp4_status mxfp4_linear_grouped_swiglu_quantize(const moe_plan* plan, const uint8_t* a_codes,
                                                            const uint8_t* a_scales, const uint8_t* w_codes,
                                                            const uint8_t* w_scales, int64_t I, int64_t K, int rotate,
                                                            uint8_t* out_codes, uint8_t* out_scales, void* stream) {
  NVFP4_TRACE("mxfp4_linear_grouped_swiglu_quantize");
  if (rotate != 0 && rotate != 1) return NVFP4_ERR_INVALID_ARG;
  GroupedArgs a = operands(a_codes, a_scales, w_codes, w_scales);
  a.mx = true;
  a.q_mode = rotate ? 2u : 1u;
  return swiglu(plan, a, I, K, out_codes, out_scales, stream);
}
