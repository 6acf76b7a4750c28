// The router of a mixture-of-experts layer: each token's top_k experts and their
// weights from the logits, and the logits' gradient.
//   score   p = softmax(l) over the experts, or p = 1 / (1 + e^-l)
//   choice  the top_k largest l, or with a bias the largest fp32(p) + bias; the lowest
//           index among equal ones
//   weight  w = scale * p [/ sum of the chosen p]
//   gradient, D_j = scale * dL/dw_j, with the weights normed w' = p / sum and without:
//           dL/dp_i = (D_i - sum_j D_j w'_j) / sum on the chosen, or D_i;
//           softmax dl = p (dp - sum dp p), sigmoid dl = dp p (1 - p)
// A warp has a token, a lane every 32nd expert in registers: the logits are read
// once, the k-th choice is a maximum over the lane's registers and two reductions
// over the warp.  An expert whose logit is -inf or NaN is never chosen and has p = 0.
#include <cfloat>
#include <cmath>

#include "moe_plan.cuh"

namespace nvfp4 {
namespace {

constexpr int kRouteThreads = 128;
constexpr float kInf = INFINITY;

struct RouteArgs {
  const void* logits;
  const float* bias;
  int32_t* idx;
  float* weights;
  const float* d_weights;
  void* d_logits;
  int64_t ld, tokens;
  int experts, top_k;
  float scale;
  bool bf16, sigmoid, renormalize;
};

// A logit; -inf in place of NaN.
__device__ __forceinline__ float load_logit(const RouteArgs& a, int64_t at) {
  const float l = a.bf16 ? __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const uint16_t*>(a.logits) + at)) << 16)
                         : __ldg(static_cast<const float*>(a.logits) + at);
  return l == l ? l : -kInf;
}

// Each operation rounded to nearest: the choice under a bias is by these 32 bits.
__device__ __forceinline__ float sigmoid_rn(float l) { return __frcp_rn(__fadd_rn(1.0f, expf(-l))); }

// e^(l - m), also where both are infinite.
__device__ __forceinline__ float exp_below(float l, float m) { return l == m ? 1.0f : __expf(l - m); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int s = 16; s; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
  return v;
}

// Unsigned integers in the order of the floats, both zeros alike; 0 for -inf and NaN: no choice.
__device__ __forceinline__ uint32_t order_key(float f) {
  if (!(f > -kInf)) return 0;
  const uint32_t b = __float_as_uint(f + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <int kPer>
__global__ void __launch_bounds__(kRouteThreads) moe_route_kernel(const RouteArgs a) {
  griddep_wait_and_release();
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kRouteThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= a.tokens) return;
  float l[kPer];
  uint32_t key[kPer];
  float top = -kInf;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = i * 32 + lane;
    l[i] = e < a.experts ? load_logit(a, t * a.ld + e) : -kInf;
    key[i] = order_key(!a.bias || !(l[i] > -kInf) ? l[i] : __fadd_rn(sigmoid_rn(l[i]), __ldg(a.bias + e)));
    top = fmaxf(top, l[i]);
  }
  // Lane j: choice j and its logit.
  int chosen = -1;
  float chosen_l = -kInf;
  for (int j = 0; j < a.top_k; ++j) {
    uint32_t best = key[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) best = max(best, key[i]);
    const uint32_t all = __reduce_max_sync(0xffffffffu, best);
    if (all == 0) break;
    uint32_t at = 0xffffffffu;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) at = key[i] == all ? i * 32 + lane : at;
    const uint32_t e = __reduce_min_sync(0xffffffffu, at);
#pragma unroll
    for (int i = 0; i < kPer; ++i) key[i] = e == static_cast<uint32_t>(i * 32 + lane) ? 0u : key[i];
    if (lane == j) chosen = static_cast<int>(e);
  }
  if (chosen >= 0) chosen_l = load_logit(a, t * a.ld + chosen);
  float p;
  if (a.sigmoid) {
    p = chosen >= 0 ? sigmoid_rn(chosen_l) : 0.0f;
    if (a.renormalize) {
      const float total = warp_sum(p);
      p = total > 0.0f ? p / total : 0.0f;
    }
  } else {
#pragma unroll
    for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    p = chosen >= 0 ? exp_below(chosen_l, top) : 0.0f;
    float total = 0.0f;
    if (a.renormalize) {
      total = p;
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) total += l[i] > -kInf ? exp_below(l[i], top) : 0.0f;
    }
    total = warp_sum(total);
    p = total > 0.0f ? p / total : 0.0f;
  }
  if (lane < a.top_k) {
    a.idx[t * a.top_k + lane] = chosen;
    a.weights[t * a.top_k + lane] = p * a.scale;
  }
}

template <int kPer>
__global__ void __launch_bounds__(kRouteThreads) moe_route_backward_kernel(const RouteArgs a) {
  __shared__ float rows[kRouteThreads / 32][kPer * 32];
  griddep_wait_and_release();
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kRouteThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= a.tokens) return;
  float* row = rows[threadIdx.x >> 5];
  float l[kPer];
  float top = -kInf;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int e = i * 32 + lane;
    l[i] = e < a.experts ? load_logit(a, t * a.ld + e) : -kInf;
    top = fmaxf(top, l[i]);
    row[e] = l[i];
  }
  __syncwarp();
  // Lane j: choice j, its D and its logit.
  int e = lane < a.top_k ? __ldg(a.idx + t * a.top_k + lane) : -1;
  if (e >= a.experts) e = -1;
  const float le = e >= 0 ? row[e] : -kInf;
  float D = e >= 0 ? a.scale * __ldg(a.d_weights + t * a.top_k + lane) : 0.0f;
  if (!(le > -kInf)) {  // never chosen by the forward pass
    e = -1;
    D = 0.0f;
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kPer; ++i) row[i * 32 + lane] = 0.0f;
  __syncwarp();
  float p, spread = 0.0f;  // spread: what softmax without norming takes off all experts
  float total = 0.0f;
  if (a.sigmoid) {
    // 1 - p as the sigmoid of -l: no cancellation.
    const float q = e >= 0 ? sigmoid_rn(-le) : 0.0f;
    p = e >= 0 ? sigmoid_rn(le) : 0.0f;
    if (a.renormalize) {
      total = warp_sum(p);
      const float w = total > 0.0f ? p / total : 0.0f;
      D = w * (D - warp_sum(D * w)) * q;
    } else {
      D = D * p * q;
    }
  } else {
#pragma unroll
    for (int s = 16; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
    p = e >= 0 ? exp_below(le, top) : 0.0f;
    if (a.renormalize) {
      total = warp_sum(p);
      const float w = total > 0.0f ? p / total : 0.0f;
      D = w * (D - warp_sum(D * w));
    } else {
#pragma unroll
      for (int i = 0; i < kPer; ++i) total += l[i] > -kInf ? exp_below(l[i], top) : 0.0f;
      total = warp_sum(total);
      const float inv = total > 0.0f ? 1.0f / total : 0.0f;
      p *= inv;
      D *= p;
      spread = warp_sum(D) * inv;
    }
  }
  // An expert that a caller's choices name twice gets both.
  const uint32_t peers = __match_any_sync(0xffffffffu, e >= 0 ? e : -1 - lane);
  if (__any_sync(0xffffffffu, __popc(peers) > 1)) {
    for (int j = 0; j < a.top_k; ++j) {
      if (lane == j && e >= 0) row[e] += D;
      __syncwarp();
    }
  } else if (e >= 0) {
    row[e] = D;
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int x = i * 32 + lane;
    if (x >= a.experts) continue;
    float d = row[x];
    if (!a.sigmoid && !a.renormalize && l[i] > -kInf) d -= exp_below(l[i], top) * spread;
    const int64_t at = t * a.experts + x;
    if (a.bf16) {
      uint16_t b;
      asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(b) : "f"(d));
      static_cast<uint16_t*>(a.d_logits)[at] = b;
    } else {
      static_cast<float*>(a.d_logits)[at] = d;
    }
  }
}

template <int kPer>
cudaError_t launch_route(const RouteArgs& a, cudaStream_t s) {
  const dim3 grid(static_cast<uint32_t>((a.tokens + kRouteThreads / 32 - 1) / (kRouteThreads / 32)));
  return launch_pdl(a.d_logits ? moe_route_backward_kernel<kPer> : moe_route_kernel<kPer>, grid, dim3(kRouteThreads), 0,
                    s, a);
}

nvfp4_status route(const moe_route_options* o, const void* logits, int32_t type, int64_t ld, int64_t n_tokens,
                   int32_t experts, RouteArgs a, cudaStream_t s) {
  if (!o) return NVFP4_ERR_INVALID_ARG;
  if (type != NVFP4_F32 && type != NVFP4_BF16) return NVFP4_ERR_INVALID_ARG;
  if (o->score != MOE_SCORE_SOFTMAX && o->score != MOE_SCORE_SIGMOID) return NVFP4_ERR_INVALID_ARG;
  if (o->renormalize != 0 && o->renormalize != 1) return NVFP4_ERR_INVALID_ARG;
  if (o->bias && o->score != MOE_SCORE_SIGMOID) return NVFP4_ERR_INVALID_ARG;
  if (!(o->scale >= -FLT_MAX && o->scale <= FLT_MAX)) return NVFP4_ERR_INVALID_ARG;
  const nvfp4_status st = check_moe_sizes(n_tokens, a.top_k, experts);
  if (st != NVFP4_OK) return st;
  if (a.top_k > experts || ld < experts) return NVFP4_ERR_SHAPE;
  if (n_tokens == 0) return NVFP4_OK;
  if (!logits || !a.idx || (a.d_logits ? !a.d_weights : !a.weights)) return NVFP4_ERR_INVALID_ARG;
  const uintptr_t size = type == NVFP4_BF16 ? 2 : 4;
  if (!aligned(logits, size) || !aligned(a.d_logits, size) || !aligned(o->bias, 4) || !aligned(a.idx, 4) ||
      !aligned(a.weights, 4) || !aligned(a.d_weights, 4))
    return NVFP4_ERR_ALIGN;
  a.logits = logits;
  a.bias = o->bias;
  a.ld = ld;
  a.tokens = n_tokens;
  a.experts = experts;
  a.scale = o->scale;
  a.bf16 = type == NVFP4_BF16;
  a.sigmoid = o->score == MOE_SCORE_SIGMOID;
  a.renormalize = o->renormalize != 0;
  const cudaError_t e = experts <= 32    ? launch_route<1>(a, s)
                        : experts <= 64  ? launch_route<2>(a, s)
                        : experts <= 128 ? launch_route<4>(a, s)
                        : experts <= 256 ? launch_route<8>(a, s)
                        : experts <= 512 ? launch_route<16>(a, s)
                                         : launch_route<32>(a, s);
  if (e != cudaSuccess) return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}

}  // namespace
}  // namespace nvfp4

using namespace nvfp4;

NVFP4_API nvfp4_status moe_route(const void* logits, int32_t logits_type, int64_t ld, int64_t n_tokens,
                                 int32_t num_experts, int32_t top_k, const moe_route_options* options,
                                 int32_t* expert_idx, float* weights, void* stream) {
  NVFP4_TRACE("moe_route");
  RouteArgs a = {};
  a.top_k = top_k;
  a.idx = expert_idx;
  a.weights = weights;
  return route(options, logits, logits_type, ld, n_tokens, num_experts, a, static_cast<cudaStream_t>(stream));
}

NVFP4_API nvfp4_status moe_route_backward(const void* logits, int32_t logits_type, int64_t ld, int64_t n_tokens,
                                          int32_t num_experts, int32_t top_k, const moe_route_options* options,
                                          const int32_t* expert_idx, const float* d_weights, void* d_logits,
                                          void* stream) {
  NVFP4_TRACE("moe_route_backward");
  if (!d_logits && n_tokens > 0) return NVFP4_ERR_INVALID_ARG;
  RouteArgs a = {};
  a.top_k = top_k;
  a.idx = const_cast<int32_t*>(expert_idx);  // read alone where d_logits is given
  a.d_weights = d_weights;
  a.d_logits = d_logits;
  return route(options, logits, logits_type, ld, n_tokens, num_experts, a, static_cast<cudaStream_t>(stream));
}
