// Tokens to their experts' rows and back, with the gradients of both.
//   moe_sort              the rows: pairs (token, choice) counted and placed by expert
//   moe_dispatch          rows[row_of[t, j]] = [w[t, j]] x[t], bf16; or quantized to NVFP4 / MXFP4
//   moe_combine           out[t] = [base[t]] + sum_j [w[t, j]] y[row_of[t, j]]
//   moe_combine_backward  dy[row_of[t, j]] = w[t, j] g[t],  dw[t, j] = <g[t], y[row_of[t, j]]>
// All walk tokens, not rows: a token is read once however many experts it has,
// its sums are in the order of its choices, and no row needs an atomic.
//
// HBM-bound from some hundred tokens on.  Of the measured copy rate: 8192 tokens of
// 5120 to 4 bf16 rows each 63 us (0.98), to NVFP4 rows 33.5 (0.79: 4-byte scale words
// apart), back with weights and a base 74 (1.0); the gradients of 4099 x 2048 with 8
// rows each 41.8 (0.87) and 22.0 (0.90).  One token: 1.7 to 2.4 us, a launch's latency.
#include <atomic>
#include <cfloat>

#include "moe_plan.cuh"
#include "nvfp4_quant.cuh"

namespace nvfp4 {
namespace {

// ------------------------------------------------------------------ sort ---
// A CTA of 32 warps places a chunk of pairs.  Each warp ranks its segment's pairs
// among those of the same expert (lanes with the same expert find each other by
// votes; a histogram in shared memory has what came before), the warps' counts
// are summed, and a pair's row is its expert's first row + the pairs of earlier
// chunks + of earlier warps + its rank.  The order is that of the pairs: no atomics
// decide it.  Latency-bound, so the chunks' counts travel the shortest way: none for
// up to 2048 pairs (one CTA), through the shared memory of a cluster of 8 CTAs for up
// to 32768, beyond it through global memory from a kernel before (131072 pairs: in the
// cluster 16 us, a few SMs' issue slots).

constexpr int kSortWarps = 32;
constexpr int kSortThreads = 32 * kSortWarps;
constexpr int kSortSteps = 16;  // steps of a warp over its segment, at most
constexpr int64_t kSortAlone = 2048;
constexpr int kSortCluster = 8;
constexpr int64_t kSortClustered = 32768;
constexpr int64_t kSortSpread = 64;  // CTAs of kChunks, until a chunk is kSortChunk
constexpr int64_t kSortChunk = kSortSteps * kSortThreads;

enum SortForm { kAlone, kCluster, kChunks };
struct SortShape {
  SortForm form;
  int64_t chunk;  // pairs of a CTA, a multiple of kSortThreads
  int64_t chunks;
};
SortShape sort_shape(int64_t pairs) {
  auto up = [](int64_t n) { return (n + kSortThreads - 1) / kSortThreads * kSortThreads; };
  SortShape s;
  s.form = pairs <= kSortAlone ? kAlone : pairs <= kSortClustered ? kCluster : kChunks;
  const int64_t ctas = s.form == kAlone ? 1 : s.form == kCluster ? kSortCluster : kSortSpread;
  s.chunk = up((pairs + ctas - 1) / ctas);
  if (s.chunk == 0) s.chunk = kSortThreads;
  if (s.chunk > kSortChunk) s.chunk = kSortChunk;
  s.chunks = s.form == kChunks ? (pairs + s.chunk - 1) / s.chunk : ctas;
  return s;
}

struct SortArgs {
  const int32_t* idx;
  int32_t* row_start;
  int32_t* rows;
  int32_t* row_of;
  uint32_t* counts;  // [chunks, experts] of kChunks
  int64_t pairs, chunk;
  int experts;
  int* status;
};

// The expert of a pair, or -1: none, or not one of the experts (reported).
__device__ __forceinline__ int expert_of(const SortArgs& a, int64_t i, int64_t end) {
  int e = i < end ? __ldg(a.idx + i) : -1;
  if (e >= a.experts) {
    set_status(a.status, NVFP4_ERR_INVALID_ARG);
    e = -1;
  }
  return max(e, -1);
}

__global__ void __launch_bounds__(kSortThreads) moe_count_kernel(const SortArgs a) {
  __shared__ uint32_t hist[kMoeMaxExperts];
  griddep_wait_and_release();
  for (int e = threadIdx.x; e < a.experts; e += kSortThreads) hist[e] = 0;
  __syncthreads();
  const int64_t begin = blockIdx.x * a.chunk, end = min(begin + a.chunk, a.pairs);
  for (int64_t i = begin + threadIdx.x; i < end; i += kSortThreads) {
    const int e = expert_of(a, i, end);
    if (e >= 0) atomicAdd(&hist[e], 1u);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.experts; e += kSortThreads)
    a.counts[blockIdx.x * static_cast<uint64_t>(a.experts) + e] = hist[e];
}

__device__ __forceinline__ uint32_t ld_cluster_u32(const uint32_t* p, uint32_t rank) {
  uint32_t at, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

// The lanes with this lane's expert, -1 counting as one: a vote for each of its bits and the sign.  (match_any takes some
// 60 cycles of a unit that all warps of an SM share: 131072 pairs on 8 SMs 19.5 us.)
__device__ __forceinline__ uint32_t same_expert(int e, int bits) {
  const uint32_t some = __ballot_sync(0xffffffffu, e >= 0);
  uint32_t peers = e >= 0 ? some : ~some;
  for (int b = 0; b < bits; ++b) {
    const bool on = e >> b & 1;
    const uint32_t vote = __ballot_sync(0xffffffffu, on);
    peers &= on ? vote : ~vote;
  }
  return peers;
}

template <SortForm kForm>
__global__ void __launch_bounds__(kSortThreads) moe_place_kernel(const SortArgs a) {
  constexpr int kSteps = kForm == kAlone ? static_cast<int>(kSortAlone / kSortThreads) : kSortSteps;
  extern __shared__ uint32_t sort_smem[];  // [warps, experts] counts, then places; [experts] first rows; [experts] counts
  __shared__ uint32_t warp_sum[kSortWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, E = a.experts;
  uint32_t* hist = sort_smem + warp * E;
  uint32_t* base = sort_smem + kSortWarps * E;
  uint32_t* count = base + E;
  for (int i = threadIdx.x; i < kSortWarps * E; i += kSortThreads) sort_smem[i] = 0;
  griddep_wait_and_release();
  const int64_t chunk_end = min((blockIdx.x + 1) * a.chunk, a.pairs);
  const int64_t begin = blockIdx.x * a.chunk + warp * (a.chunk / kSortWarps) + lane;
  const int steps = static_cast<int>(a.chunk / kSortThreads), bits = 32 - __clz(E - 1);
  int at[kSteps];  // a pair's expert, and then its rank among the warp's << 10 | expert; -1: none
#pragma unroll
  for (int i = 0; i < kSteps; ++i) at[i] = i < steps ? expert_of(a, begin + 32 * i, chunk_end) : -1;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    if (i >= steps) break;
    const int e = at[i];
    const uint32_t peers = same_expert(e, bits), lower = peers & ((1u << lane) - 1);
    uint32_t before = 0;
    if (e >= 0) before = hist[e];
    __syncwarp();
    if (e >= 0) {
      if (lower == 0) hist[e] = before + __popc(peers);
      at[i] = static_cast<int>((before + __popc(lower)) << 10) | e;
    }
    __syncwarp();
  }
  __syncthreads();
  // Thread e: expert e's pairs in this chunk before each warp, in earlier chunks, and in all.
  const int e = threadIdx.x;
  uint32_t total = 0, before = 0;
  if (e < E) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      uint32_t n[kSortWarps / 2];
      uint32_t* h = sort_smem + half * (kSortWarps / 2) * E + e;
#pragma unroll
      for (int w = 0; w < kSortWarps / 2; ++w) n[w] = h[w * E];
#pragma unroll
      for (int w = 0; w < kSortWarps / 2; ++w) {
        h[w * E] = total;
        total += n[w];
      }
    }
  }
  if constexpr (kForm == kCluster) {
    if (e < E) count[e] = total;
    cluster_sync_all();
    if (e < E) {
      const uint32_t own = cluster_ctarank();
      uint32_t n[kSortCluster];
#pragma unroll
      for (uint32_t c = 0; c < kSortCluster; ++c) n[c] = ld_cluster_u32(count + e, c);
      total = 0;
#pragma unroll
      for (uint32_t c = 0; c < kSortCluster; ++c) {
        total += n[c];
        before += c < own ? n[c] : 0u;
      }
    }
  } else if constexpr (kForm == kChunks) {
    // The chunks in as many shares as there are threads for.
    __shared__ uint32_t sums[2][kSortThreads];
    const uint32_t shares = kSortThreads / E, share = threadIdx.x / E, x = threadIdx.x - share * E;
    if (share < shares) {
      uint32_t all = 0, lower = 0;
#pragma unroll 8
      for (uint32_t c = share; c < gridDim.x; c += shares) {
        const uint32_t n = __ldcg(a.counts + c * static_cast<uint64_t>(E) + x);
        all += n;
        lower += c < blockIdx.x ? n : 0u;
      }
      sums[0][threadIdx.x] = all;
      sums[1][threadIdx.x] = lower;
    }
    __syncthreads();
    if (e < E) {
      total = 0;
      for (uint32_t i = 0; i < shares; ++i) {
        total += sums[0][i * E + e];
        before += sums[1][i * E + e];
      }
    }
  }
  const uint32_t padded = (total + kMoeRowTile - 1) / kMoeRowTile * kMoeRowTile;
  uint32_t sum = padded;  // inclusive over the experts
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, sum, s);
    if (lane >= s) sum += v;
  }
  if (lane == 31) warp_sum[warp] = sum;
  __syncthreads();
  sum += __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[lane] : 0u);
  if (e < E) {
    base[e] = sum - padded + before;
    if (blockIdx.x == 0) {
      a.rows[e] = static_cast<int32_t>(total);
      a.row_start[e] = static_cast<int32_t>(sum - padded);
      if (e == E - 1) a.row_start[E] = static_cast<int32_t>(sum);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    if (i >= steps) break;
    int row = -1;
    if (at[i] >= 0) {
      const int x = at[i] & 1023;
      row = static_cast<int>(base[x] + hist[x]) + (at[i] >> 10);
    }
    if (begin + 32 * i < chunk_end) a.row_of[begin + 32 * i] = row;
  }
  if constexpr (kForm == kCluster) cluster_sync_all();  // no CTA leaves while another may read its counts
}

size_t place_smem(int experts) { return static_cast<size_t>(kSortWarps + 2) * experts * sizeof(uint32_t); }

// The shared-memory opt-in of a form's kernel, once for each device and for as many experts as there can be: the limit is
// the kernel's, whose other callers, in other threads, may need more than this one.
bool place_opted_in(void (*kernel)(SortArgs), SortForm form) {
  static std::atomic<uint64_t> done[3];  // a bit a device
  int d = 0;
  if (cudaGetDevice(&d) != cudaSuccess) return false;
  const uint64_t bit = d < 64 ? 1ull << d : 0;
  if (done[form].load(std::memory_order_acquire) & bit) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           static_cast<int>(place_smem(kMoeMaxExperts))) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  done[form].fetch_or(bit, std::memory_order_release);
  return true;
}

// ------------------------------------------------------- walks over tokens ---
// `vecs` units of a token's channels.  A CTA has a token, or several short ones; the
// GPU's many CTAs cover the latency, without a loop over tokens (one over resident
// CTAs: 8192 tokens of 5120 to 4 rows each in NVFP4 39 us).  Loops are uniform in a
// warp.

constexpr uint32_t kWalkThreads = 512;  // at most

struct Walk {
  int64_t tokens;
  uint32_t vecs, per_cta;  // per_cta: tokens of a CTA
};
struct WalkLaunch {
  Walk w;
  dim3 grid, block;
};
// Tokens of a CTA of 256 threads where a token has few units: not more than leave a CTA to each SM.
uint32_t short_tokens(int64_t tokens, uint32_t vecs) {
  const int64_t spread = tokens / sm_count();
  return vecs >= 128 || spread <= 1 ? 1u : static_cast<uint32_t>(spread < 256 / vecs ? spread : 256 / vecs);
}
WalkLaunch make_walk(int64_t tokens, uint32_t vecs) {
  WalkLaunch l;
  l.w = {tokens, vecs, short_tokens(tokens, vecs)};
  const uint32_t passes = (vecs + kWalkThreads - 1) / kWalkThreads;
  l.block = dim3(l.w.per_cta > 1 ? 256 : ((vecs + passes - 1) / passes + 31) / 32 * 32);
  l.grid = dim3(static_cast<uint32_t>((tokens + l.w.per_cta - 1) / l.w.per_cta));
  return l;
}
// f(token, unit, live) for all of this thread's units.
template <class F>
__device__ __forceinline__ void walk(const Walk& w, F&& f) {
  const uint32_t sub = w.per_cta > 1 ? threadIdx.x / w.vecs : 0u;
  const uint32_t v0 = threadIdx.x - sub * w.vecs;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * w.per_cta + sub;
  for (uint32_t v = 0; v < w.vecs; v += blockDim.x)
    f(t, v + v0, sub < w.per_cta && t < w.tokens && v + v0 < w.vecs);
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ uint4 pack8(const float v[8]) {
  return make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
}

struct RowArgs {
  const int32_t* row_of;
  int top_k, max_rows;
  int* status;
};
constexpr int kBatch = 4;  // choices whose loads are in flight together
// The rows of choices j0 .. j0 + B - 1 of token t, or -1.  A plan that names rows outside the buffers has none there.
template <int B>
__device__ __forceinline__ void rows_of(const RowArgs& a, int64_t t, int j0, int (&r)[B]) {
#pragma unroll
  for (int i = 0; i < B; ++i) {
    r[i] = j0 + i < a.top_k ? __ldg(a.row_of + t * a.top_k + j0 + i) : -1;
    if (r[i] >= a.max_rows) r[i] = -1;
  }
}

// A token's units among `threads` threads, U for each (and a pass), `threads` apart.  Bf16 rows with U = 2 / 1, us, there and
// back: 16384 tokens of 2048, one row each 21.0 / 30.4 and 30.0 / 36.1, two 30.9 / 37.6 and 35.6 / 40.9, eight 92 / 91 and
// 86 / 88; 600, one each 1.54 / 1.93 and 1.99 / 2.57; one token to and from eight, 2.05 / 1.89 and 2.90 / 2.57: 1 for up to a
// token an SM.  Four take long tokens in one pass; a loop over passes (5120 channels back 89 for 74) only the longest (2000 x
// 32768 from four rows in passes of two units 112, of four 99).
struct Split {
  int64_t tokens;
  uint32_t vecs, threads, per_cta;
  dim3 grid() const { return dim3(static_cast<uint32_t>((tokens + per_cta - 1) / per_cta)); }
  dim3 block() const { return dim3((per_cta * threads + 31) / 32 * 32); }
};
template <int U>
Split make_split(int64_t tokens, uint32_t vecs) {
  const uint32_t passes = (vecs + 512 * U - 1) / (512 * U);
  Split w = {tokens, vecs, (vecs + U * passes - 1) / (U * passes), 1u};
  w.per_cta = short_tokens(tokens, w.threads);
  return w;
}

template <int U, bool kLoop>
__global__ void __launch_bounds__(512)
    moe_dispatch_kernel(const RowArgs a, const Split w, const uint16_t* __restrict__ x, int64_t ld,
                        const float* __restrict__ weights, uint16_t* __restrict__ out) {
  griddep_wait_and_release();
  const uint32_t sub = w.per_cta > 1 ? threadIdx.x / w.threads : threadIdx.x >= w.threads, vecs = w.vecs;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * w.per_cta + sub;
  if (sub >= w.per_cta || t >= w.tokens) return;
  uint32_t v0 = threadIdx.x - sub * w.threads;
  do {
    uint4 in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t v = v0 + u * w.threads;
      if (v < vecs) in[u] = __ldg(reinterpret_cast<const uint4*>(x + t * ld) + v);
    }
    for (int j0 = 0; j0 < a.top_k; j0 += kBatch) {
      int r[kBatch];
      rows_of(a, t, j0, r);
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (r[j] < 0) continue;
        const float c = weights ? __ldg(weights + t * a.top_k + j0 + j) : 1.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t v = v0 + u * w.threads;
          if (v >= vecs) continue;
          uint4 d = in[u];
          if (weights) {
            float f[8];
            unpack_bf16x8(in[u], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] *= c;
            d = pack8(f);
          }
          reinterpret_cast<uint4*>(out)[static_cast<int64_t>(r[j]) * vecs + v] = d;
        }
      }
    }
    v0 += U * w.threads;
  } while (kLoop && v0 < vecs);
}

template <int U, bool kLoop = false>
cudaError_t launch_dispatch(const RowArgs& a, int64_t tokens, uint32_t vecs, const void* x, int64_t ld,
                            const float* weights, void* rows, cudaStream_t s) {
  const Split w = make_split<U>(tokens, vecs);
  return launch_pdl(moe_dispatch_kernel<U, kLoop>, w.grid(), w.block(), 0, s, a, w, static_cast<const uint16_t*>(x), ld,
                    weights, static_cast<uint16_t*>(rows));
}

// Codes and scale word of a thread's 32 channels to the token's rows.
__device__ __forceinline__ void store_operand(const RowArgs& a, const Walk& w, int64_t t, uint32_t v, uint4 codes,
                                              uint32_t word, uint4* out_codes, uint8_t* scales) {
  for (int j0 = 0; j0 < a.top_k; j0 += kBatch) {
    int r[kBatch];
    rows_of(a, t, j0, r);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (r[j] < 0) continue;
      out_codes[static_cast<int64_t>(r[j]) * w.vecs + v] = codes;
      if ((v & 1) == 0) {
        const uint64_t off = mma_scale_offset(static_cast<uint64_t>(r[j]), 2 * v, w.vecs >> 1);
        if (in_bounds(a.status, off + 4 <= static_cast<uint64_t>(a.max_rows) * 2 * w.vecs))
          *reinterpret_cast<uint32_t*>(scales + off) = word;
      }
    }
  }
}

// A thread has 32 channels, two NVFP4 blocks; two lanes have a scale word.
__global__ void __launch_bounds__(kWalkThreads)
    moe_dispatch_nvfp4_kernel(const RowArgs a, const Walk w, const uint16_t* __restrict__ x, int64_t ld,
                              const float* __restrict__ g_dev, uint4* __restrict__ codes, uint8_t* __restrict__ scales) {
  griddep_wait_and_release();
  const float g_in = __ldg(g_dev);
  const bool g_ok = g_in > 0.0f && g_in <= FLT_MAX;
  if (!g_ok && blockIdx.x == 0 && threadIdx.x == 0) set_status(a.status, NVFP4_ERR_INVALID_ARG);
  const float g = g_ok ? g_in : 1.0f, six_g = __fmul_rn(6.0f, g);
  walk(w, [&](int64_t t, uint32_t v, bool live) {
    const uint4* src = reinterpret_cast<const uint4*>(x + t * ld) + 4 * v;
    uint4 in[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) in[q] = live ? __ldg(src + q) : make_uint4(0, 0, 0, 0);
    uint32_t c[4], word = 0;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      float f[16];
      unpack_bf16x8(in[2 * b], f);
      unpack_bf16x8(in[2 * b + 1], f + 8);
      const uint32_t top = max(amax_bits_bf16x8(in[2 * b]), amax_bits_bf16x8(in[2 * b + 1]));
      const BlockScale s = block_scale(__uint_as_float(top << 16), g, six_g);
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = __fmul_rn(f[i], s.mult);
      c[2 * b] = e2m1x8(f);
      c[2 * b + 1] = e2m1x8(f + 8);
      word |= s.code << (8 * (2 * (v & 1) + b));
    }
    word |= __shfl_xor_sync(0xffffffffu, word, 1);
    if (live) store_operand(a, w, t, v, g_ok ? make_uint4(c[0], c[1], c[2], c[3]) : make_uint4(0, 0, 0, 0),
                            g_ok ? word : 0u, codes, scales);
  });
}

// A thread has 32 channels, one MXFP4 block, whose scale is stored for both of its halves.
template <bool kRotate>
__global__ void __launch_bounds__(kWalkThreads)
    moe_dispatch_mxfp4_kernel(const RowArgs a, const Walk w, const uint16_t* __restrict__ x, int64_t ld,
                              uint4* __restrict__ codes, uint8_t* __restrict__ scales) {
  griddep_wait_and_release();
  walk(w, [&](int64_t t, uint32_t v, bool live) {
    const uint4* src = reinterpret_cast<const uint4*>(x + t * ld) + 4 * v;
    float f[32];
#pragma unroll
    for (int q = 0; q < 4; ++q) unpack_bf16x8(live ? __ldg(src + q) : make_uint4(0, 0, 0, 0), f + 8 * q);
    if (kRotate) hadamard32(f);
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) amax = fmaxf(amax, fabsf(f[i]));
    const uint32_t code = mx_scale_code(amax);
    const float inv = mx_inv_scale(code);
#pragma unroll
    for (int i = 0; i < 32; ++i) f[i] = __fmul_rn(f[i], inv);
    const uint4 c = make_uint4(e2m1x8(f), e2m1x8(f + 8), e2m1x8(f + 16), e2m1x8(f + 24));
    uint32_t word = (code | (code << 8)) << (16 * (v & 1));
    word |= __shfl_xor_sync(0xffffffffu, word, 1);
    if (live) store_operand(a, w, t, v, c, word, codes, scales);
  });
}

// The sum is in 32 bits, in the order of the choices, rounded once.  The loads of a batch of choices are all in flight
// (without the batch 89 us for 8192 tokens of 5120 from 4 rows each; with it 74, the measured copy rate); a
// batch of two where there are no more choices, for its fewer registers (16384 tokens of 2048 from one row each 30.0 -> 26.7,
// from two 35.7 -> 32.9; of 5120 from two 90.9 -> 86.9).
template <int U, bool kLoop, int B>
__global__ void __launch_bounds__(512)
    moe_combine_kernel(const RowArgs a, const Split w, const uint16_t* __restrict__ y,
                       const float* __restrict__ weights, const uint16_t* base, int64_t ld_base, uint16_t* out,
                       int64_t ld_out) {
  griddep_wait_and_release();
  const uint32_t sub = w.per_cta > 1 ? threadIdx.x / w.threads : threadIdx.x >= w.threads, vecs = w.vecs;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * w.per_cta + sub;
  if (sub >= w.per_cta || t >= w.tokens) return;
  uint32_t v0 = threadIdx.x - sub * w.threads;
  do {
    float acc[U][8] = {};
    if (base) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t v = v0 + u * w.threads;
        if (v < vecs) unpack_bf16x8(reinterpret_cast<const uint4*>(base + t * ld_base)[v], acc[u]);  // out may be base
      }
    }
    for (int j0 = 0; j0 < a.top_k; j0 += B) {
      int r[B];
      float c[B];
      uint4 in[B][U];
      rows_of(a, t, j0, r);
#pragma unroll
      for (int j = 0; j < B; ++j) {
        c[j] = r[j] < 0 ? 0.0f : weights ? __ldg(weights + t * a.top_k + j0 + j) : 1.0f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t v = v0 + u * w.threads;
          if (r[j] >= 0 && v < vecs)
            in[j][u] = __ldg(reinterpret_cast<const uint4*>(y) + static_cast<int64_t>(r[j]) * vecs + v);
        }
      }
#pragma unroll
      for (int j = 0; j < B; ++j) {
        if (r[j] < 0) continue;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          float f[8];
          unpack_bf16x8(in[j][u], f);
#pragma unroll
          for (int i = 0; i < 8; ++i) acc[u][i] = fmaf(c[j], f[i], acc[u][i]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t v = v0 + u * w.threads;
      if (v < vecs) reinterpret_cast<uint4*>(out + t * ld_out)[v] = pack8(acc[u]);
    }
    v0 += U * w.threads;
  } while (kLoop && v0 < vecs);
}

template <int U, bool kLoop = false, int B = kBatch>
cudaError_t launch_combine(const RowArgs& a, int64_t tokens, uint32_t vecs, const void* y, const float* weights,
                           const void* base, int64_t ld_base, void* out, int64_t ld_out, cudaStream_t s) {
  const Split w = make_split<U>(tokens, vecs);
  return launch_pdl(moe_combine_kernel<U, kLoop, B>, w.grid(), w.block(), 0, s, a, w, static_cast<const uint16_t*>(y),
                    weights, static_cast<const uint16_t*>(base), ld_base, static_cast<uint16_t*>(out), ld_out);
}

// kWarps warps have a token, a batch of choices at a time: one load of d_out serves the batch.  Their parts of a sum are
// added in order.
constexpr int kBackThreads = 256;
template <int kWarps>
__global__ void __launch_bounds__(kBackThreads)
    moe_combine_backward_kernel(const RowArgs a, int64_t tokens, uint32_t vecs, const uint16_t* __restrict__ d_out,
                                int64_t ld, const uint16_t* __restrict__ y, const float* __restrict__ weights,
                                uint16_t* __restrict__ d_y, float* __restrict__ d_weights) {
  constexpr int kPer = kBackThreads / 32 / kWarps;  // tokens of a CTA
  __shared__ float parts[kMoeMaxTopK][kPer][kWarps];
  griddep_wait_and_release();
  const int warp = threadIdx.x >> 5, sub = warp / kWarps, part = warp % kWarps;
  const int64_t t = static_cast<int64_t>(blockIdx.x) * kPer + sub;
  const uint32_t lane = threadIdx.x & 31;
  const bool live = t < tokens;
  const uint4* g4 = reinterpret_cast<const uint4*>(d_out + t * ld);
  for (int j0 = 0; live && j0 < a.top_k; j0 += kBatch) {
    int r[kBatch];
    float c[kBatch], dot[kBatch] = {};
    rows_of(a, t, j0, r);
#pragma unroll
    for (int j = 0; j < kBatch; ++j) c[j] = r[j] >= 0 ? __ldg(weights + t * a.top_k + j0 + j) : 0.0f;
#pragma unroll 2
    for (uint32_t v = part * 32 + lane; v < vecs; v += 32 * kWarps) {
      const uint4 gv = __ldg(g4 + v);
      uint4 in[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j)
        if (r[j] >= 0) in[j] = __ldg(reinterpret_cast<const uint4*>(y) + static_cast<int64_t>(r[j]) * vecs + v);
      float g[8];
      unpack_bf16x8(gv, g);
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (r[j] < 0) continue;
        float f[8];
        unpack_bf16x8(in[j], f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          dot[j] = fmaf(g[i], f[i], dot[j]);
          f[i] = g[i] * c[j];
        }
        if (d_y) reinterpret_cast<uint4*>(d_y)[static_cast<int64_t>(r[j]) * vecs + v] = pack8(f);
      }
    }
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
#pragma unroll
      for (int s = 16; s; s >>= 1) dot[j] += __shfl_xor_sync(0xffffffffu, dot[j], s);
      if (lane == 0 && j0 + j < a.top_k) parts[j0 + j][sub][part] = dot[j];
    }
  }
  __syncthreads();
  if (d_weights && live && part == 0 && static_cast<int>(lane) < a.top_k) {
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) sum += parts[lane][sub][w];
    d_weights[t * a.top_k + lane] = sum;
  }
}

RowArgs row_args(const moe_plan* p) {
  RowArgs a;
  a.row_of = p->row_of;
  a.top_k = p->top_k;
  a.max_rows = static_cast<int>(moe_rows_bound(p->n_tokens, p->top_k, p->num_experts));
  a.status = status_word_dev();
  return a;
}

// What every call over tokens checks: the plan, [tokens, cols] with rows ld apart, cols a multiple of `step`.
nvfp4_status check_tokens(const moe_plan* p, int64_t cols, int64_t step, int64_t ld) {
  const nvfp4_status st = check_moe_plan(p);
  if (st != NVFP4_OK) return st;
  if (cols < step || cols > 65536 || cols % step || ld < cols) return NVFP4_ERR_SHAPE;
  return ld % 8 ? NVFP4_ERR_ALIGN : NVFP4_OK;
}

}  // namespace
}  // namespace nvfp4

using namespace nvfp4;

NVFP4_API int64_t moe_max_rows(int64_t n_tokens, int32_t top_k, int32_t num_experts) {
  return check_moe_sizes(n_tokens, top_k, num_experts) == NVFP4_OK ? moe_rows_bound(n_tokens, top_k, num_experts) : 0;
}

NVFP4_API size_t moe_sort_workspace_size(int64_t n_tokens, int32_t top_k, int32_t num_experts) {
  if (check_moe_sizes(n_tokens, top_k, num_experts) != NVFP4_OK) return 0;
  const SortShape s = sort_shape(n_tokens * top_k);
  return s.form == kChunks ? static_cast<size_t>(s.chunks) * num_experts * sizeof(uint32_t) : 0;
}

NVFP4_API nvfp4_status moe_sort(const moe_plan* plan, const int32_t* expert_idx, void* workspace,
                                size_t workspace_bytes, void* stream) {
  NVFP4_TRACE("moe_sort");
  const nvfp4_status st = check_moe_plan(plan);
  if (st != NVFP4_OK) return st;
  const size_t need = moe_sort_workspace_size(plan->n_tokens, plan->top_k, plan->num_experts);
  if ((!expert_idx && plan->n_tokens) || (need && !workspace)) return NVFP4_ERR_INVALID_ARG;
  if (workspace_bytes < need) return NVFP4_ERR_SHAPE;
  if (!aligned(expert_idx, 4) || (need && !aligned(workspace, 16))) return NVFP4_ERR_ALIGN;
  SortArgs a;
  a.idx = expert_idx;
  a.row_start = plan->row_start;
  a.rows = plan->rows;
  a.row_of = plan->row_of;
  a.counts = static_cast<uint32_t*>(workspace);
  a.pairs = plan->n_tokens * plan->top_k;
  a.experts = plan->num_experts;
  a.status = status_word_dev();
  const SortShape s = sort_shape(a.pairs);
  a.chunk = s.chunk;
  const cudaStream_t cs = static_cast<cudaStream_t>(stream);
  const size_t smem = place_smem(a.experts);
  const auto kernel = s.form == kAlone ? moe_place_kernel<kAlone>
                      : s.form == kCluster ? moe_place_kernel<kCluster> : moe_place_kernel<kChunks>;
  // With the static part beside it, 48 KB are passed earlier.
  if (smem > 32 * 1024 && !place_opted_in(kernel, s.form)) return NVFP4_ERR_CUDA;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kSortCluster;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<uint32_t>(s.chunks));
  cfg.blockDim = dim3(kSortThreads);
  cfg.stream = cs;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (s.form == kChunks) {
    if (cudaLaunchKernelEx(&cfg, moe_count_kernel, a) != cudaSuccess) return NVFP4_ERR_CUDA;
    count_launches(1);
  }
  cfg.dynamicSmemBytes = smem;
  cfg.numAttrs = s.form == kCluster ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, a) != cudaSuccess) return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}

NVFP4_API nvfp4_status moe_dispatch(const moe_plan* plan, const void* x_bf16, int64_t ld_x, int64_t cols,
                                    const float* weights, void* rows_bf16, void* stream) {
  NVFP4_TRACE("moe_dispatch");
  const nvfp4_status st = check_tokens(plan, cols, 8, ld_x);
  if (st != NVFP4_OK) return st;
  if (plan->n_tokens == 0) return NVFP4_OK;
  if (!x_bf16 || !rows_bf16) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(x_bf16, 16) || !aligned(rows_bf16, 16) || !aligned(weights, 4)) return NVFP4_ERR_ALIGN;
  const uint32_t vecs = static_cast<uint32_t>(cols / 8);
  const auto launch = vecs <= 512 && plan->n_tokens <= sm_count() ? launch_dispatch<1>
                      : vecs <= 1024 ? launch_dispatch<2> : vecs <= 2048 ? launch_dispatch<4> : launch_dispatch<2, true>;
  if (launch(row_args(plan), plan->n_tokens, vecs, x_bf16, ld_x, weights, rows_bf16,
             static_cast<cudaStream_t>(stream)) != cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}

NVFP4_API nvfp4_status moe_dispatch_nvfp4(const moe_plan* plan, const void* x_bf16, int64_t ld_x, int64_t cols,
                                          const float* g_dev, uint8_t* codes, uint8_t* scales, void* stream) {
  NVFP4_TRACE("moe_dispatch_nvfp4");
  const nvfp4_status st = check_tokens(plan, cols, 64, ld_x);
  if (st != NVFP4_OK) return st;
  if (plan->n_tokens == 0) return NVFP4_OK;
  if (!x_bf16 || !g_dev || !codes || !scales) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(x_bf16, 16) || !aligned(codes, 16) || !aligned(scales, 4) || !aligned(g_dev, 4)) return NVFP4_ERR_ALIGN;
  const WalkLaunch l = make_walk(plan->n_tokens, static_cast<uint32_t>(cols / 32));
  if (launch_pdl(moe_dispatch_nvfp4_kernel, l.grid, l.block, 0,
                 static_cast<cudaStream_t>(stream), row_args(plan), l.w, static_cast<const uint16_t*>(x_bf16), ld_x,
                 g_dev, reinterpret_cast<uint4*>(codes), scales) != cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}

NVFP4_API nvfp4_status moe_dispatch_mxfp4(const moe_plan* plan, const void* x_bf16, int64_t ld_x, int64_t cols,
                                          int rotate, uint8_t* codes, uint8_t* scales, void* stream) {
  NVFP4_TRACE("moe_dispatch_mxfp4");
  const nvfp4_status st = check_tokens(plan, cols, 64, ld_x);
  if (st != NVFP4_OK) return st;
  if (rotate != 0 && rotate != 1) return NVFP4_ERR_INVALID_ARG;
  if (plan->n_tokens == 0) return NVFP4_OK;
  if (!x_bf16 || !codes || !scales) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(x_bf16, 16) || !aligned(codes, 16) || !aligned(scales, 4)) return NVFP4_ERR_ALIGN;
  const WalkLaunch l = make_walk(plan->n_tokens, static_cast<uint32_t>(cols / 32));
  if (launch_pdl(rotate ? moe_dispatch_mxfp4_kernel<true> : moe_dispatch_mxfp4_kernel<false>, l.grid, l.block, 0,
                 static_cast<cudaStream_t>(stream), row_args(plan), l.w, static_cast<const uint16_t*>(x_bf16), ld_x,
                 reinterpret_cast<uint4*>(codes), scales) != cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}

NVFP4_API nvfp4_status moe_combine(const moe_plan* plan, const void* y_bf16, int64_t cols, const float* weights,
                                   const void* base_bf16, int64_t ld_base, void* out_bf16, int64_t ld_out,
                                   void* stream) {
  NVFP4_TRACE("moe_combine");
  nvfp4_status st = check_tokens(plan, cols, 8, ld_out);
  if (st != NVFP4_OK) return st;
  if (base_bf16 && ld_base < cols) return NVFP4_ERR_SHAPE;
  if (plan->n_tokens == 0) return NVFP4_OK;
  if (!y_bf16 || !out_bf16) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(y_bf16, 16) || !aligned(out_bf16, 16) || !aligned(base_bf16, 16) || !aligned(weights, 4) ||
      (base_bf16 && ld_base % 8))
    return NVFP4_ERR_ALIGN;
  const uint32_t vecs = static_cast<uint32_t>(cols / 8);
  const auto launch = vecs <= 512 && plan->n_tokens <= sm_count() ? launch_combine<1>
                      : vecs <= 1024 ? (plan->top_k <= 2 ? launch_combine<2, false, 2> : launch_combine<2>)
                      : vecs <= 2048 ? launch_combine<4> : launch_combine<4, true>;
  if (launch(row_args(plan), plan->n_tokens, vecs, y_bf16, weights, base_bf16, ld_base, out_bf16, ld_out,
             static_cast<cudaStream_t>(stream)) != cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}

NVFP4_API nvfp4_status moe_combine_backward(const moe_plan* plan, const void* d_out_bf16, int64_t ld_d_out,
                                            const void* y_bf16, int64_t cols, const float* weights, void* d_y_bf16,
                                            float* d_weights, void* stream) {
  NVFP4_TRACE("moe_combine_backward");
  const nvfp4_status st = check_tokens(plan, cols, 8, ld_d_out);
  if (st != NVFP4_OK) return st;
  if (plan->n_tokens == 0) return NVFP4_OK;
  if (!d_out_bf16 || !y_bf16 || !weights || (!d_y_bf16 && !d_weights)) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(d_out_bf16, 16) || !aligned(y_bf16, 16) || !aligned(d_y_bf16, 16) || !aligned(weights, 4) ||
      !aligned(d_weights, 4))
    return NVFP4_ERR_ALIGN;
  // A token's warps: eight where it has many units, or where the tokens are few; us with eight / two:
  //   8192 tokens  2048 x 8 rows 87.8 / 90.3, 5120 x 4 112 / 114, 2048 x 2 38.5 / 33.5, 512 x 8 50.8 / 26.1
  //   600 tokens   2048 x 8 7.9 / 11.8, 2048 x 2 3.6 / 5.5, 512 x 8 4.0 / 3.6;  64 tokens  2048 x 8 2.8 / 5.5, 512 x 8 2.3 / 2.6
  // (one: 97, 119, 33.5, 26.8 at 8192 tokens; four: 89.8, 113, 36.3, 36.2).
  const bool eight = cols / 8 * plan->top_k >= 1024 || 8 * plan->n_tokens <= 32 * static_cast<int64_t>(sm_count());
  const int warps = eight ? 8 : 2;
  const auto kernel = eight ? moe_combine_backward_kernel<8> : moe_combine_backward_kernel<2>;
  const int64_t per = kBackThreads / 32 / warps, grid = (plan->n_tokens + per - 1) / per;
  if (launch_pdl(kernel, dim3(static_cast<uint32_t>(grid)), dim3(kBackThreads), 0,
                 static_cast<cudaStream_t>(stream), row_args(plan), plan->n_tokens, static_cast<uint32_t>(cols / 8),
                 static_cast<const uint16_t*>(d_out_bf16), ld_d_out, static_cast<const uint16_t*>(y_bf16), weights,
                 static_cast<uint16_t*>(d_y_bf16), d_weights) != cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}
