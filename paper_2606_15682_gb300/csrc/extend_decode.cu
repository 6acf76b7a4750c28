// Attention of new tokens, up to 8 rows of a sequence and KV head.
//
// A CTA takes 8 rows and a range of keys.  Warp 0 streams the keys' codes and scales
// into a two-stage ring of 128 keys; four warps take two 16-key tiles of a stage
// each, dequantize in registers (exact in f16) and multiply with mma.sync m16n8k16:
// S^T[16 keys, 8 rows] = K Q^T, O^T[128, 8 rows] += V^T P^T.  Four CTAs an SM.  What
// bounds it is latency: DRAM is at 50 %, the issue slots at 56 %, the tensor pipe at 19 %
// (38 x 8192 keys); warps wait for their stage and for one another's results in
// dequantization.  64 ragged sequences of up to 16384 keys, 40 on 8 heads: 143 us,
// 3.5 TB/s, 0.52 of the measured copy rate; 38 x 8192 keys 95 us, 0.56, 100 with a bias, 103
// with a cap.  (extend_rows_kernel, whose shared-memory traffic does not shrink with the
// rows, took 187 us where this one took 149, and this one loses at 16 rows: it has twice
// the MMAs then.)
//
// Lane roles (g = lane / 4, t = lane % 4), as the fragments have them:
//   K rows g and g + 8 of the tile, channels 32t..32t+31; V rows 2t, 2t+1, 2t+8,
//   2t+9, channels 16g..16g+15; Q row g, channels 32t..32t+31.
// Row m of a 16-key tile is key (m & 1) * 4 + (m >> 1 & 3) + (m & 8), so that a V
// load covers four consecutive keys.
#include "extend_attention.cuh"

namespace nvfp4 {
namespace {

constexpr int kRows = 8, kWarps = 4;
constexpr int kThreads = 32 * (1 + kWarps);
constexpr int kRing = 2;
constexpr uint32_t kStageCodes = kBlock * 64, kStageBytes = 2 * kBlock * (64 + 8);  // K, V codes, K, V scales
constexpr int kMergeRow = 148;  // floats of a row's 128 channels in the merge buffer: 2 of padding per 16

__device__ __forceinline__ int tile_key(int m) { return (m & 1) * 4 + ((m >> 1) & 3) + (m & 8); }
__device__ __forceinline__ void mma16816(float c[4], const uint32_t a[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
struct DecodeShared {
  uint64_t full[kRing], empty[kRing];
  alignas(16) uint32_t present[kRing][4];
  Item item;
  int lo, hi;  // of this part
  float m[kWarps][kRows], l[kWarps][kRows];
  volatile int abort;
};
constexpr uint32_t kSmem = kRing * kStageBytes + kWarps * kRows * kMergeRow * 4;

// kMods: a cap or a bias.
template <bool kE1M2, bool kMods>
__global__ void __launch_bounds__(kThreads, 4) extend_decode_kernel(const ExtendArgs a) {
  extern __shared__ __align__(128) uint8_t smem_raw[];
  __shared__ DecodeShared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&sh.full[i], 1 + 32 + lost_arrivals(a, i));  // the armed bytes, and each lane's own copies
      mbar_init(&sh.empty[i], kWarps);
    }
    sh.abort = 0;
    fence_mbar_init();
  }
  griddep_wait_and_release();
  const uint32_t group = a.group.d;
  if (warp == 0) {
    const Item it = find_item<kRows>(a, blockIdx.x);
    // The keys that the tile's rows see, in this part.
    int lo = 0x7fffffff, hi = 0;
    const uint32_t rows = it.tile.b < a.map.batch ? min(it.seq.n * group - it.tile.row0, static_cast<uint32_t>(kRows)) : 0;
    if (lane < static_cast<int>(rows)) {
      const uint32_t tok = a.group.div(it.tile.row0 + lane);
      const int p = it.seq.len - static_cast<int>(it.seq.n) + static_cast<int>(tok);
      const int2 vis = visible(a, p, it.seq.len, a.prefix_lens ? __ldg(a.prefix_lens + it.tile.b) : 0,
                               a.doc_start ? __ldg(a.doc_start + it.seq.first + tok) : 0);
      if (p >= 0 && vis.x < vis.y) {
        lo = vis.x;
        hi = vis.y;
      }
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) {
      sh.item = it;
      const int64_t part = static_cast<int64_t>(a.part_blocks) * kBlock, from = it.span.lo + it.part * part;
      sh.lo = static_cast<int>(max(static_cast<int64_t>(lo), from));
      sh.hi = static_cast<int>(min(static_cast<int64_t>(hi), from + part));
    }
  }
  __syncthreads();
  const Tile tile = sh.item.tile;
  if (tile.b >= a.map.batch) return;  // more CTAs than items
  const Seq seq = sh.item.seq;
  const uint32_t kvh = sh.item.kvh, parts = sh.item.span.parts;
  const uint32_t rows = min(seq.n * group - tile.row0, static_cast<uint32_t>(kRows));
  const int t_base = sh.lo, t_end = sh.hi, n = t_end > t_base ? (t_end - t_base + kBlock - 1) / kBlock : 0;

  if (warp == 0) {
    // ------------------------------------------------------------ producer ---
    // Lane i has keys i, i + 32, i + 64, i + 96 of a stage.  Codes come by bulk
    // copies, one for each run of keys within a page; scales, 8 bytes a key, by
    // the lane's own copies.  A key that is not there (past the end, or its page
    // absent) gets scales of zero, whatever its codes' bytes.
    const int64_t head = static_cast<int64_t>(kvh) * a.map.size.d;
    int issued = 0;
    for (int i = 0; i < n; ++i) {
      const int st = i & 1, t0 = t_base + (n - 1 - i) * kBlock;  // the newest keys first: maxima settle early
      int64_t row[4];
      uint32_t here[4], total = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int t = t0 + 32 * k + lane;
        row[k] = t < t_end ? a.map.row(tile.b, t) : -1;
        here[k] = __ballot_sync(0xffffffffu, row[k] >= 0);
        total += __popc(here[k]);
      }
      if (!__all_sync(0xffffffffu, wait_bar(&sh.empty[st], ((i >> 1) & 1) ^ 1, &sh.abort))) {
        if (lane == 0 && !sh.abort) {
          set_status(a.status, NVFP4_ERR_TIMEOUT);
          sh.abort = 1;
        }
        break;
      }
      uint8_t* stage = smem_raw + st * kStageBytes;
      uint8_t* scales = stage + 2 * kStageCodes;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (row[k] < 0) {
          reinterpret_cast<uint2*>(scales)[32 * k + lane] = make_uint2(0, 0);
          reinterpret_cast<uint2*>(scales + kBlock * 8)[32 * k + lane] = make_uint2(0, 0);
        }
      if (lane < 4) sh.present[st][lane] = lane == 0 ? here[0] : lane == 1 ? here[1] : lane == 2 ? here[2] : here[3];
      __syncwarp();
      if (lane == 0) mbar_arrive_expect_tx(&sh.full[st], total * 128);
      __syncwarp();
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int c = 32 * k + lane;
        if (row[k] < 0) continue;
        const int64_t at = row[k] + head;
        const uint32_t off = static_cast<uint32_t>(a.map.table ? (t0 + c) - static_cast<int>(a.map.size.div(t0 + c)) * static_cast<int>(a.map.size.d) : t0 + c);
        if (c == 0 || off == 0) {  // a run of keys begins
          const int len = min(min(static_cast<int>(a.map.size.d - off), kBlock - c), t_end - (t0 + c));
          bulk_load(stage + c * 64, a.map.k_codes + at * 64, len * 64, &sh.full[st]);
          bulk_load(stage + kStageCodes + c * 64, a.map.v_codes + at * 64, len * 64, &sh.full[st]);
        }
        const uint32_t to = smem_u32(scales + c * 8);
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(a.map.k_scales + at * 8) : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to + kBlock * 8), "l"(a.map.v_scales + at * 8) : "memory");
      }
      asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&sh.full[st])) : "memory");
      issued = i + 1;
    }
    // Copies in flight land before the CTA's memory goes to another (its
    // consumers have waited for them unless a wait ran out): the last two stages issued.
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (sh.abort)
      for (int i = max(issued - 2, 0); i < issued; ++i)
        mbar_wait_bounded(&sh.full[i & 1], (i >> 1) & 1, nullptr, kDrainLimitNs);
    return;
  }

  // ------------------------------------------------------------- consumers ---
  const int cw = warp - 1, g = lane >> 2, t = lane & 3;
  // Rows of the lane's columns in a tile of scores: 2t and 2t + 1.
  int2 vis[2];
  float mult[2], slope[2];
  int pos[2];
  int all_lo = 0, all_hi = 0x7fffffff;  // keys that every row sees
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const uint32_t lr = 2 * t + c;
    const bool live = lr < rows;
    const uint32_t r = tile.row0 + (live ? lr : 0), tok = a.group.div(r), h = kvh * group + (r - tok * group);
    const int p = seq.len - static_cast<int>(seq.n) + static_cast<int>(tok);
    vis[c] = visible(a, p, seq.len, a.prefix_lens ? __ldg(a.prefix_lens + tile.b) : 0,
                     a.doc_start ? __ldg(a.doc_start + seq.first + tok) : 0);
    if (!live || p < 0) vis[c] = make_int2(0x7fffffff, 0);
    if (live) {
      all_lo = max(all_lo, vis[c].x);
      all_hi = min(all_hi, vis[c].y);
    }
    pos[c] = p;
    slope[c] = a.slopes && live ? __ldg(a.slopes + h) * kLog2e : 0.0f;
  }
  all_lo = __reduce_max_sync(0xffffffffu, all_lo);
  all_hi = __reduce_min_sync(0xffffffffu, all_hi);
  // Queries: f16 after an exact scaling by a power of two to below 1.
  uint32_t qf[16];
  {
    const bool live = g < static_cast<int>(rows);
    const uint32_t r = tile.row0 + (live ? g : 0), tok = a.group.div(r);
    const uint4* src = reinterpret_cast<const uint4*>(a.q + static_cast<int64_t>(seq.first + tok) * a.ld_q +
                                                      (kvh * group + (r - tok * group)) * kD + 32 * t);
    uint4 w[4];
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[i] = live ? __ldg(src + i) : make_uint4(0, 0, 0, 0);
      top = max(top, amax_bits_bf16x8(w[i]));
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const RowScale by = row_scale(top);
    const float up = score_factor(a.scale, by.up);
    mult[0] = __shfl_sync(0xffffffffu, up, (2 * t) * 4);
    mult[1] = __shfl_sync(0xffffffffu, up, (2 * t + 1) * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[8];
      unpack_bf16x8(w[i], x);
      const uint4 f = q_chunk<kE1M2>(x, by.down);  // k-steps 2i and 2i + 1
      qf[4 * i] = f.x;
      qf[4 * i + 1] = f.y;
      qf[4 * i + 2] = f.z;
      qf[4 * i + 3] = f.w;
    }
  }

  // No maximum yet: any score exceeds it.
  float o[8][4], minus[2] = {FLT_MAX, FLT_MAX}, l_run[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
  const int rk0 = tile_key(g), rk1 = tile_key(g + 8);
  const int rv[4] = {tile_key(2 * t), tile_key(2 * t + 1), tile_key(2 * t + 8), tile_key(2 * t + 9)};
  bool ok = true;
  for (int i = 0; i < n; ++i) {
    const int st = i & 1;
    ok = __all_sync(0xffffffffu, wait_bar(&sh.full[st], (i >> 1) & 1, &sh.abort));
    if (!ok) {
      if (lane == 0 && !sh.abort) {
        set_status(a.status, NVFP4_ERR_TIMEOUT);
        sh.abort = 1;
      }
      break;
    }
    const uint8_t* stage = smem_raw + st * kStageBytes;
    const uint8_t* k_scales = stage + 2 * kStageCodes;
    const uint8_t* v_scales = k_scales + kBlock * 8;
    // Every row sees every key of the stage.
    const uint4 present = *reinterpret_cast<const uint4*>(sh.present[st]);
    const int t_stage = t_base + (n - 1 - i) * kBlock;
    const bool open = t_stage >= all_lo && t_stage + kBlock <= all_hi && (present.x & present.y & present.z & present.w) == 0xffffffffu;
#pragma unroll
    for (int sub = 0; sub < kBlock / (16 * kWarps); ++sub) {
      const int r0 = 16 * (cw + kWarps * sub), t0 = t_stage + r0;
      const uint32_t there = open ? 0xFFFFu : (sh.present[st][r0 >> 5] >> (r0 & 31)) & 0xFFFFu;
      if (!there) continue;
      // ---- S^T = K Q^T: 8 k-steps of 16 channels --------------------------
      const uint4 ka = *reinterpret_cast<const uint4*>(stage + (r0 + rk0) * 64 + 16 * t);
      const uint4 kb = *reinterpret_cast<const uint4*>(stage + (r0 + rk1) * 64 + 16 * t);
      const uint32_t ksa = kv_scales16<kE1M2>(*reinterpret_cast<const uint16_t*>(k_scales + (r0 + rk0) * 8 + 2 * t));
      const uint32_t ksb = kv_scales16<kE1M2>(*reinterpret_cast<const uint16_t*>(k_scales + (r0 + rk1) * 8 + 2 * t));
      const uint32_t sa_lo = __byte_perm(ksa, ksa, 0x1010), sa_hi = __byte_perm(ksa, ksa, 0x3232);
      const uint32_t sb_lo = __byte_perm(ksb, ksb, 0x1010), sb_hi = __byte_perm(ksb, ksb, 0x3232);
      float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      const uint32_t kaw[4] = {ka.x, ka.y, ka.z, ka.w}, kbw[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t ha[4], hb[4];
        scaled8<kE1M2>(kaw[w], w < 2 ? sa_lo : sa_hi, ha);
        scaled8<kE1M2>(kbw[w], w < 2 ? sb_lo : sb_hi, hb);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t f[4] = {ha[2 * h], hb[2 * h], ha[2 * h + 1], hb[2 * h + 1]};
          mma16816(s, f, qf[4 * w + 2 * h], qf[4 * w + 2 * h + 1]);
        }
      }
      // ---- scores, masks, the running maximum ------------------------------
      bool up = false;
#pragma unroll
      for (int c = 0; c < 4; ++c) s[c] *= mult[c & 1];
      if (kMods) {
        if (a.cap > 0.0f) cap_scores<4>(s, a.cap * kLog2e);
#pragma unroll
        for (int c = 0; c < 4; ++c)
          s[c] = fmaf(-slope[c & 1], fabsf(static_cast<float>(pos[c & 1] - (t0 + (c < 2 ? rk0 : rk1)))), s[c]);
      }
      if (!open) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int key = t0 + (c < 2 ? rk0 : rk1);
          if (key < vis[c & 1].x || key >= vis[c & 1].y || !((there >> (key - t0)) & 1u)) s[c] = -INFINITY;
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) up = up || s[c] + minus[c & 1] > kWeightLog2 + kRescaleLog2;
      if (__any_sync(0xffffffffu, up)) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float top = fmaxf(s[c], s[c + 2]);
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
          if (top + minus[c] > kWeightLog2 + kRescaleLog2) {
            const float shrink = ex2(kWeightLog2 - top - minus[c]);
            minus[c] = kWeightLog2 - top;
            l_run[c] *= shrink;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              o[k][c] *= shrink;
              o[k][c + 2] *= shrink;
            }
          }
        }
      }
      const float p0 = ex2(s[0] + minus[0]), p1 = ex2(s[1] + minus[1]), p2 = ex2(s[2] + minus[0]), p3 = ex2(s[3] + minus[1]);
      l_run[0] += p0 + p2;
      l_run[1] += p1 + p3;
      const uint32_t pb0 = transposed(f16x2_rn(p0, p1)), pb1 = transposed(f16x2_rn(p2, p3));
      // ---- O^T += V^T P^T: 8 m-tiles, m-tile k = channels 16g+2k, 16g+2k+1 --
      const uint32_t vs01 = kv_scales16<kE1M2>(v_scales[(r0 + rv[0]) * 8 + g] | v_scales[(r0 + rv[1]) * 8 + g] << 8);
      const uint32_t vs89 = kv_scales16<kE1M2>(v_scales[(r0 + rv[2]) * 8 + g] | v_scales[(r0 + rv[3]) * 8 + g] << 8);
      const uint32_t vs01_hi = kE1M2 ? mul_f16x2(vs01, 0x2C002C00u) : vs01;
      const uint32_t vs89_hi = kE1M2 ? mul_f16x2(vs89, 0x2C002C00u) : vs89;
      uint2 vw[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) vw[k] = *reinterpret_cast<const uint2*>(stage + kStageCodes + (r0 + rv[k]) * 64 + 8 * g);
#pragma unroll
      for (int half = 0; half < 2; ++half) {  // channels 16g..16g+7, then the other eight
        const uint32_t wa = half ? vw[0].y : vw[0].x, wb = half ? vw[1].y : vw[1].x;
        const uint32_t wc = half ? vw[2].y : vw[2].x, wd = half ? vw[3].y : vw[3].x;
        uint32_t lo_ab[4], hi_ab[4], lo_cd[4], hi_cd[4];
        if (kE1M2) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {  // byte k of two keys: its low-nibble channel, and 16 times its high one
            const uint32_t ab = __byte_perm(wa, wb, 0x4400u + 0x1111u * k), cd = __byte_perm(wc, wd, 0x4400u + 0x1111u * k);
            lo_ab[k] = sub_f16x2((ab & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
            hi_ab[k] = sub_f16x2((ab & 0x00F000F0u) ^ 0x64806480u, 0x64806480u);
            lo_cd[k] = sub_f16x2((cd & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
            hi_cd[k] = sub_f16x2((cd & 0x00F000F0u) ^ 0x64806480u, 0x64806480u);
          }
        } else {  // the same channel of two keys in one byte, the first key in its low nibble
          elements8<false>((wa & 0x0F0F0F0Fu) | ((wb << 4) & 0xF0F0F0F0u), lo_ab);
          elements8<false>(((wa >> 4) & 0x0F0F0F0Fu) | (wb & 0xF0F0F0F0u), hi_ab);
          elements8<false>((wc & 0x0F0F0F0Fu) | ((wd << 4) & 0xF0F0F0F0u), lo_cd);
          elements8<false>(((wc >> 4) & 0x0F0F0F0Fu) | (wd & 0xF0F0F0F0u), hi_cd);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t f[4] = {mul_f16x2(lo_ab[k], vs01), mul_f16x2(hi_ab[k], vs01_hi), mul_f16x2(lo_cd[k], vs89),
                                 mul_f16x2(hi_cd[k], vs89_hi)};
          mma16816(o[4 * half + k], f, pb0, pb1);
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.empty[st]);
  }

  // ---- join the warps -------------------------------------------------------
  float* merge = reinterpret_cast<float*>(smem_raw + kRing * kStageBytes);
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) l_run[c] += __shfl_xor_sync(0xffffffffu, l_run[c], x);
    if (g == 0) {
      sh.m[cw][2 * t + c] = l_run[c] == 0.0f ? -INFINITY : -minus[c];  // weights are 2^(score - m)
      sh.l[cw][2 * t + c] = l_run[c];
    }
  }
  float* mine = merge + cw * kRows * kMergeRow;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int c = 18 * g + 2 * k;  // channels 16g + 2k and the next, 2 floats of padding per 16
    *reinterpret_cast<float2*>(mine + (2 * t) * kMergeRow + c) = make_float2(o[k][0], o[k][2]);
    *reinterpret_cast<float2*>(mine + (2 * t + 1) * kMergeRow + c) = make_float2(o[k][1], o[k][3]);
  }
  asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
  for (int idx = threadIdx.x - 32; idx < static_cast<int>(rows) * (kD / 4); idx += 32 * kWarps) {
    const int lr = idx / (kD / 4), c = idx % (kD / 4) * 4;
    float big = -INFINITY, sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kWarps; ++w) big = fmaxf(big, sh.m[w][lr]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float mw = sh.m[w][lr], f = mw == -INFINITY ? 0.0f : ex2(mw - big);
      const float2* from = reinterpret_cast<const float2*>(merge + (w * kRows + lr) * kMergeRow + c + 2 * (c >> 4));
      const float2 u = from[0], v = from[1];
      sum = fmaf(f, sh.l[w][lr], sum);
      acc[0] = fmaf(f, u.x, acc[0]);
      acc[1] = fmaf(f, u.y, acc[1]);
      acc[2] = fmaf(f, v.x, acc[2]);
      acc[3] = fmaf(f, v.y, acc[3]);
    }
    if (parts > 1) {
      const uint64_t rec = ((static_cast<uint64_t>(sh.item.tile_id) * a.map.hkv + kvh) * a.splits + sh.item.part) * kRows + lr;
      if (!record_in_bounds<kRows>(a, rec)) continue;
      if (c == 0) a.ml_ws[rec] = make_float2(big, sum);
      if (big != -INFINITY) *reinterpret_cast<float4*>(a.o_ws + rec * kD + c) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    } else {
      const float f = per_sum(sum, a.gv);
      const uint32_t r = tile.row0 + lr, tok = a.group.div(r);
      const uint64_t row = static_cast<uint64_t>(seq.first + tok) * a.hq + kvh * group + r - tok * group;
      if (!out_in_bounds(a, row)) continue;
      *reinterpret_cast<uint2*>(a.out + row * kD + c) =
          make_uint2(bf16x2_rn(acc[0] * f, acc[1] * f), bf16x2_rn(acc[2] * f, acc[3] * f));
    }
  }
}

}  // namespace

ExtendLaunch extend_decode(bool e1m2, bool mods) {
  const ExtendKernel k = e1m2 ? (mods ? extend_decode_kernel<true, true> : extend_decode_kernel<true, false>)
                              : (mods ? extend_decode_kernel<false, true> : extend_decode_kernel<false, false>);
  return {k, kThreads, kSmem};
}

}  // namespace nvfp4
