// The router of a mixture-of-experts layer: each token's top_k experts and their
// weights from the logits, and the logits' gradient.
//   score   p = softmax(l) over the experts, or p = 1 / (1 + e^-l)
//   choice  the top_k largest l, or with a bias the largest fp32(p) + bias; the lowest
//           index among equal ones
//   weight  w = scale * p [/ sum of the chosen p]
//   gradient, D_j = scale * dL/dw_j, with the weights normed w' = p / sum and without:
//           dL/dp_i = (D_i - sum_j D_j w'_j) / sum on the chosen, or D_i;
//           softmax dl = p (dp - sum dp p), sigmoid dl = dp p (1 - p)
// A warp has a token, a lane some of its logits in registers: they are read once.
// An expert whose logit is -inf or NaN is never chosen and has p = 0.
//
// Bound by issue slots for most of its time: 459 instructions a token of 256 experts and 8
// choices, 650 with sigmoid and a bias, of which a scheduler issues 0.71 a cycle: the choices'
// reductions wait for each other.  16384 tokens: 9.2 us, 11.8 with
// sigmoid and bias (a maximum over all registers for each choice: 23), of which the issue alone
// is 6.0 and 8.5 at 2.05 GHz and the rest 2.25 waves of CTAs, a start and an end; their bytes
// 2.5.  Gradient of 8191 x 128 in bf16 3.6 (through a row in shared memory 4.8).  32 tokens:
// 2.1 us, a launch's latency.
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

template <bool kBf16>
__device__ __forceinline__ float load_logit(const RouteArgs& a, int64_t at) {
  if (kBf16) return __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const uint16_t*>(a.logits) + at)) << 16);
  return __ldg(static_cast<const float*>(a.logits) + at);
}

// A lane's experts: 4 in a row of every 128, in wide loads, or (kWide false: rows that are not aligned for them) every 32nd.
template <bool kWide>
__device__ __forceinline__ int expert_at(int i, int lane) {
  return kWide ? (i >> 2) * 128 + 4 * lane + (i & 3) : 32 * i + lane;
}
// The lane's numbers of a row of `experts`; those behind the last one stay as they are.
template <int kPer, class T, bool kWide>
__device__ __forceinline__ void load_row(const T* row, int experts, int lane, float v[kPer]) {
  constexpr bool kBf16 = sizeof(T) == 2;
  if constexpr (kWide) {
#pragma unroll
    for (int i = 0; i < kPer; i += 4) {
      const int e = 32 * i + 4 * lane;  // the experts are a multiple of 4
      if (e >= experts) continue;
      if constexpr (kBf16) {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(row + e));
        v[i] = __uint_as_float(w.x << 16);
        v[i + 1] = __uint_as_float(w.x & 0xFFFF0000u);
        v[i + 2] = __uint_as_float(w.y << 16);
        v[i + 3] = __uint_as_float(w.y & 0xFFFF0000u);
      } else {
        const float4 w = __ldg(reinterpret_cast<const float4*>(row + e));
        v[i] = w.x;
        v[i + 1] = w.y;
        v[i + 2] = w.z;
        v[i + 3] = w.w;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int e = 32 * i + lane;
      if (e >= experts) continue;
      if constexpr (kBf16)
        v[i] = __uint_as_float(static_cast<uint32_t>(__ldg(row + e)) << 16);
      else
        v[i] = __ldg(row + e);
    }
  }
}
// The lane's logits of token t: -inf in place of NaN and behind the last expert.
template <int kPer, bool kBf16, bool kWide>
__device__ __forceinline__ void load_logits(const RouteArgs& a, int64_t t, int lane, float l[kPer]) {
#pragma unroll
  for (int i = 0; i < kPer; ++i) l[i] = -kInf;
  if constexpr (kBf16)
    load_row<kPer, uint16_t, kWide>(static_cast<const uint16_t*>(a.logits) + t * a.ld, a.experts, lane, l);
  else
    load_row<kPer, float, kWide>(static_cast<const float*>(a.logits) + t * a.ld, a.experts, lane, l);
#pragma unroll
  for (int i = 0; i < kPer; ++i) l[i] = fmaxf(l[i], -kInf);  // the number where the other is NaN
}

// Each operation rounded to nearest: the choice under a bias is by these 32 bits.
__device__ __forceinline__ float sigmoid_rn(float l) { return __frcp_rn(__fadd_rn(1.0f, expf(-l))); }

// e^(l - m), also where both are infinite.
__device__ __forceinline__ float exp_below(float l, float m) { return l == m ? 1.0f : __expf(l - m); }

__device__ __forceinline__ uint32_t pack_rn(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int s = 16; s; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
  return v;
}

// The largest of the warp's numbers (no NaN).
__device__ __forceinline__ float warp_max(float v) {
  float m;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
  return m;
}

// Keys are numbers, -inf those of experts that are not to be chosen; equal ones (both zeros are) go to the lowest expert.
// One choice after another: the largest key of the warp, of the lowest expert that has it.
template <int kPer, bool kWide>
__device__ __forceinline__ int choose_in_turn(float key[kPer], int top_k, int lane) {
  int chosen = -1;
  for (int j = 0; j < top_k; ++j) {
    float best = key[0];
#pragma unroll
    for (int i = 1; i < kPer; ++i) best = fmaxf(best, key[i]);
    const float all = warp_max(best);
    if (!(all > -kInf)) break;
    uint32_t at = 0xffffffffu;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) at = key[i] == all ? expert_at<kWide>(i, lane) : at;
    const uint32_t e = __reduce_min_sync(0xffffffffu, at);
#pragma unroll
    for (int i = 0; i < kPer; ++i) key[i] = e == static_cast<uint32_t>(expert_at<kWide>(i, lane)) ? -kInf : key[i];
    if (lane == j) chosen = static_cast<int>(e);
  }
  return chosen;
}

// The key under a bias, as it is defined, and within 2^-20 of it (and the sum's rounding) by the hardware's 2^x and 1 / x.
__device__ __forceinline__ float biased_key(float l, float bias) {
  return l > -kInf ? fmaxf(__fadd_rn(sigmoid_rn(l), bias), -kInf) : -kInf;  // not NaN
}
__device__ __forceinline__ float about_biased_key(float l, float bias) {
  float e, s;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(l * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.0f + e));
  return l > -kInf ? fmaxf(s + bias, -kInf) : -kInf;
}

// The same with fewer steps: the top_k-th largest of the lanes' own maxima is at most the top_k-th largest key, so few
// keys reach it; those are gathered, one a lane, and chosen in turn.  Under a bias the first part goes by approximate keys
// and a margin of more than twice their error, and a lane forms the key of its own candidate alone.  More than 32
// candidates (many equal keys), or fewer lanes with a key than top_k: all in turn.  list: [32] of the warp.
template <int kPer, bool kBf16, bool kWide>
__device__ __forceinline__ int choose(const RouteArgs& a, int64_t t, const float l[kPer], int lane, float2* list) {
  float key[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) key[i] = l[i];
  if (a.bias) {
    float b[kPer] = {};
    load_row<kPer, float, kWide>(a.bias, a.experts, lane, b);
#pragma unroll
    for (int i = 0; i < kPer; ++i) key[i] = kPer == 1 ? biased_key(l[i], b[i]) : about_biased_key(l[i], b[i]);
  }
  if constexpr (kPer == 1) return choose_in_turn<kPer, kWide>(key, a.top_k, lane);
  float best = key[0];
#pragma unroll
  for (int i = 1; i < kPer; ++i) best = fmaxf(best, key[i]);
  float least = -kInf;
  for (int j = 0; j < a.top_k; ++j) {
    least = warp_max(best);
    best = best == least ? -kInf : best;
  }
  const float from = a.bias ? least - 0x1p-18f * (1.0f + fabsf(least)) : least;
  int n = 0;
  const uint32_t lower = (1u << lane) - 1;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const bool in = key[i] >= from;
    const uint32_t vote = __ballot_sync(0xffffffffu, in);
    const int at = n + __popc(vote & lower);
    if (in && at < 32) list[at] = make_float2(key[i], __int_as_float(expert_at<kWide>(i, lane)));
    n += __popc(vote);
  }
  if (!(least > -kInf) || n > 32 || n < a.top_k) {
    if (a.bias) {
#pragma unroll
      for (int i = 0; i < kPer; ++i)
        if (l[i] > -kInf) key[i] = biased_key(l[i], __ldg(a.bias + expert_at<kWide>(i, lane)));
    }
    return choose_in_turn<kPer, kWide>(key, a.top_k, lane);
  }
  __syncwarp();
  const float2 mine = list[min(lane, n - 1)];
  const uint32_t expert = __float_as_uint(mine.y);
  float k = mine.x;
  if (a.bias) k = biased_key(fmaxf(load_logit<kBf16>(a, t * a.ld + expert), -kInf), __ldg(a.bias + expert));
  if (lane >= n) k = -kInf;
  int chosen = -1;
  for (int j = 0; j < a.top_k; ++j) {
    const float all = warp_max(k);
    const uint32_t e = __reduce_min_sync(0xffffffffu, k == all ? expert : 0xffffffffu);
    k = expert == e ? -kInf : k;
    if (lane == j) chosen = static_cast<int>(e);
  }
  return chosen;
}

template <int kPer, bool kBf16, bool kWide>
__global__ void __launch_bounds__(kRouteThreads) moe_route_kernel(const RouteArgs a) {
  __shared__ float2 lists[kRouteThreads / 32][32];
  griddep_wait_and_release();
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kRouteThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= a.tokens) return;
  float l[kPer];
  load_logits<kPer, kBf16, kWide>(a, t, lane, l);
  // Lane j: choice j and its logit.
  const int chosen = choose<kPer, kBf16, kWide>(a, t, l, lane, lists[threadIdx.x >> 5]);
  const float chosen_l = chosen >= 0 ? load_logit<kBf16>(a, t * a.ld + chosen) : -kInf;
  float p;
  if (a.sigmoid) {
    p = chosen >= 0 ? sigmoid_rn(chosen_l) : 0.0f;
    if (a.renormalize) {
      const float total = warp_sum(p);
      p = total > 0.0f ? p / total : 0.0f;
    }
  } else {
    const float top = __shfl_sync(0xffffffffu, chosen_l, 0);  // the first choice's
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

template <int kPer, bool kBf16, bool kWide>
__global__ void __launch_bounds__(kRouteThreads) moe_route_backward_kernel(const RouteArgs a) {
  griddep_wait_and_release();
  const int64_t t = static_cast<int64_t>(blockIdx.x) * (kRouteThreads / 32) + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (t >= a.tokens) return;
  // Lane j: choice j, its D and its logit.
  int e = lane < a.top_k ? __ldg(a.idx + t * a.top_k + lane) : -1;
  if (e >= a.experts) e = -1;
  float D = e >= 0 ? a.scale * __ldg(a.d_weights + t * a.top_k + lane) : 0.0f;
  float l[kPer];
  load_logits<kPer, kBf16, kWide>(a, t, lane, l);
  const float le = e >= 0 ? fmaxf(load_logit<kBf16>(a, t * a.ld + e), -kInf) : -kInf;
  if (!(le > -kInf)) {  // never chosen by the forward pass
    e = -1;
    D = 0.0f;
  }
  float top = -kInf;
#pragma unroll
  for (int i = 0; i < kPer; ++i) top = fmaxf(top, l[i]);
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
    top = warp_max(top);
    if (a.renormalize) {
      // Shares among the chosen: against the largest of them, which a caller's own choices may have far below the rest.
      const bool none = top == kInf && le < kInf;
      top = warp_max(le);
      p = e >= 0 && !none ? exp_below(le, top) : 0.0f;
      total = warp_sum(p);
      const float w = total > 0.0f ? p / total : 0.0f;
      D = w * (D - warp_sum(D * w));
    } else {
      p = e >= 0 ? exp_below(le, top) : 0.0f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) total += l[i] > -kInf ? exp_below(l[i], top) : 0.0f;
      total = warp_sum(total);
      const float inv = total > 0.0f ? 1.0f / total : 0.0f;
      p *= inv;
      D *= p;
      spread = warp_sum(D) * inv;
    }
  }
  // To the lanes that hold the chosen experts; one that a caller's choices name twice gets both, in order.
  float d[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i)
    d[i] = !a.sigmoid && !a.renormalize && l[i] > -kInf ? -exp_below(l[i], top) * spread : 0.0f;
  for (int j = 0; j < a.top_k; ++j) {
    const int x = __shfl_sync(0xffffffffu, e, j);
    const float v = __shfl_sync(0xffffffffu, D, j);
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (x == expert_at<kWide>(i, lane)) d[i] += v;
  }
  const int64_t out = t * a.experts;
#pragma unroll
  for (int i = 0; i < kPer; i += kWide ? 4 : 1) {
    const int x = expert_at<kWide>(i, lane);
    if (x >= a.experts) continue;
    if constexpr (kWide && kBf16) {
      *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.d_logits) + out + x) =
          make_uint2(pack_rn(d[i], d[i + 1]), pack_rn(d[i + 2], d[i + 3]));
    } else if constexpr (kWide) {
      *reinterpret_cast<float4*>(static_cast<float*>(a.d_logits) + out + x) =
          make_float4(d[i], d[i + 1], d[i + 2], d[i + 3]);
    } else if constexpr (kBf16) {
      static_cast<uint16_t*>(a.d_logits)[out + x] = static_cast<uint16_t>(pack_rn(d[i], 0.0f));
    } else {
      static_cast<float*>(a.d_logits)[out + x] = d[i];
    }
  }
}

template <int kPer, bool kBf16, bool kWide>
cudaError_t launch_route(const RouteArgs& a, cudaStream_t s) {
  const dim3 grid(static_cast<uint32_t>((a.tokens + kRouteThreads / 32 - 1) / (kRouteThreads / 32)));
  return launch_pdl(a.d_logits ? moe_route_backward_kernel<kPer, kBf16, kWide> : moe_route_kernel<kPer, kBf16, kWide>,
                    grid, dim3(kRouteThreads), 0, s, a);
}
template <int kPer>
cudaError_t launch_route(const RouteArgs& a, cudaStream_t s) {
  if constexpr (kPer >= 4) {
    const uintptr_t wide = a.bf16 ? 8 : 16;
    if (a.experts % 4 == 0 && a.ld % 4 == 0 && aligned(a.logits, wide) && aligned(a.d_logits, wide) &&
        aligned(a.bias, 16))
      return a.bf16 ? launch_route<kPer, true, true>(a, s) : launch_route<kPer, false, true>(a, s);
  }
  return a.bf16 ? launch_route<kPer, true, false>(a, s) : launch_route<kPer, false, false>(a, s);
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
