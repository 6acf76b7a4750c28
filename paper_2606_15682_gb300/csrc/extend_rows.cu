// Attention of new tokens, few rows of a sequence and KV head.
//
// HBM-bound work: every byte of K and V is needed once for up to 32 rows.  A CTA
// takes kC rows and a range of keys, and multiplies the other way round, so that
// the rows are the short side of every product (kN = 16 or 32 of the tensor core):
//   S^T[128 keys, kN] = K Q^T: K dequantized into TMEM (lane = key), Q in shared memory
//   O^T[128 channels, kN] += V^T P^T: V dequantized into shared memory, P too
//   warps 0-3   softmax (thread = key; in the end, channel of O^T)
//   warps 4-7   K (thread = key)
//   warps 8-11  V
//   warp 12     issues the MMAs; 13-15 complete its warpgroup
// Two CTAs share an SM.  32 x 4 drafted tokens on 4001 keys, 40 on 8 heads (24 rows),
// take 65 us in E2M1 and 74 in E1M2, 0.34 and 0.30 of the measured copy rate; HBM alone
// would take 22.  16 rows take 56, 32 rows 68.  What bounds it is the softmax warps' turn
// per block, at one key a thread: it goes by its instructions, which the four roles' code,
// too long for the instruction caches near the schedulers, makes expensive (issue slots 57 %
// used, "no instruction" 1.1 stalls an issue).  (By mma.sync in registers it took 148 us.)
#include "extend_attention.cuh"

namespace nvfp4 {
namespace {

constexpr int kRowsThreads = 16 * 32;
constexpr uint32_t kRowsTmem = 256;  // columns: K 2 x 64, S^T 2 x 32, O^T 32
constexpr uint32_t kColS = 128, kColO = 192;
constexpr int kAhead = 3;  // blocks whose K and V are on their way to L2, past the one in registers

template <int kC>
struct RowsConfig {
  static constexpr int kN = kC <= 16 ? 16 : 32;
  // Shared memory: V, two blocks; Q; P, two blocks of one term (two with kFull).
  static constexpr uint32_t kB = kN * 256;  // bytes of a kN x 128 f16 operand
  static constexpr uint32_t kOffQ = 2 * kOperand, kOffP = kOffQ + kB;
  static constexpr uint32_t kBytes = kOffP + 4 * kB + 1024;
};

template <int kC>
struct RowsShared {
  uint64_t s_full[2], k_full[2], k_free[2], v_full[2], v_free[2], p_full[2], q_full, drain;
  uint32_t tmem;
  Item item;
  int lo, hi, all_lo, all_hi, rows;
  alignas(16) float mult[kC];  // score -> log2 domain
  alignas(16) float minus[kC], none[kC];  // 4 - the row's maximum: x = score + minus is a weight's exponent
  int pos0;  // the position of the tile's first query, from which the others and the keys are counted
  alignas(16) float slope[kC], pos[kC];  // slopes[h] log2(e); the query's position from pos0
  alignas(16) int first[kC], last[kC];  // keys that it sees: first <= t < last
  uint32_t out[kC];                     // its row of the output; past the tile's rows: none
  float top[4][kC], sum[4][kC];
  uint32_t present[4][4];
  volatile int abort;
};

// kC consecutive columns of the warp's lanes.
template <int kC>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  if (kC == 32) {
    tmem_ld32(taddr, r);
    return;
  }
  if (kC >= 16)
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
                   "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
                 : "r"(taddr));
  if (kC == 8 || kC == 24) {
    constexpr int o = kC - 8;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(u[o]), "=r"(u[o + 1]), "=r"(u[o + 2]), "=r"(u[o + 3]), "=r"(u[o + 4]), "=r"(u[o + 5]),
                   "=r"(u[o + 6]), "=r"(u[o + 7])
                 : "r"(taddr + o));
  }
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const float* r) {
  const uint32_t* u = reinterpret_cast<const uint32_t*>(r);
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "r"(u[0]), "r"(u[1]),
               "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
               : "memory");
}
// P as the operand B: key k's rows 8g..8g+7 are the 16 bytes at 2048 g + 16 k (no
// swizzle, N contiguous: 8 x 8 core matrices of 128 bytes, 128 bytes from eight
// keys to the next, 2048 from eight rows to the next).
constexpr uint32_t kDescPlainHigh = (2048u >> 4) | (1u << 14);
__device__ __forceinline__ uint32_t plain_desc(uint32_t saddr) { return ((saddr & 0x3FFFFu) >> 4) | ((128u >> 4) << 16); }
__device__ __forceinline__ void mma_v_p(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n .reg .pred p;\n .reg .b64 da, db;\n setp.ne.b32 p, %4, 0;\n mov.b64 da, {%1, %5};\n"
               " mov.b64 db, {%2, %6};\n tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n}" ::"r"(d),
               "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"(kDescHigh), "n"(kDescPlainHigh)
               : "memory");
}

// kCap: the scores may be capped.  (A kernel of its own: the cap's code in the kernel of calls
// without one cost their softmax warps registers and instruction fetches: 32 x 6 drafted tokens
// on 4001 keys 81.5 instead of 72.5 us when it was measured.)
template <int kC, bool kE1M2, bool kCap, bool kFull>
__global__ void __launch_bounds__(kRowsThreads, 2) extend_rows_kernel(const ExtendArgs a) {
  using C = RowsConfig<kC>;
  constexpr int kN = C::kN;
  extern __shared__ uint8_t smem_raw[];
  __shared__ RowsShared<kC> sh;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.k_full[i], 4 + lost_arrivals(a, i));
      mbar_init(&sh.k_free[i], 1);
      mbar_init(&sh.v_full[i], 4);
      mbar_init(&sh.v_free[i], 1);
      mbar_init(&sh.p_full[i], 4);
    }
    mbar_init(&sh.drain, 1);
    mbar_init(&sh.q_full, 4);
    sh.abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&sh.tmem, kRowsTmem);
    tmem_relinquish();  // the SM's other CTA allocates too
  }
  // The next kernel's CTAs, which may allocate as well, start once this one has its columns.
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_wait_and_release();
  const uint32_t group = a.group.d;
  if (warp == 0) {
    const Item it = find_item<kC>(a, blockIdx.x);
    const Tile tl = it.tile;
    const Seq sq = it.seq;
    const uint32_t kvh = it.kvh;
    const bool any = tl.b < a.map.batch;  // else more CTAs than items
    // A row a lane: what it sees, and where its output goes.
    const uint32_t rows = any ? min(sq.n * group - tl.row0, static_cast<uint32_t>(kC)) : 0;
    const bool live = lane < static_cast<int>(rows);
    const uint32_t r = tl.row0 + (live ? lane : 0), tok = a.group.div(r), h = kvh * group + (r - tok * group);
    const int pos = sq.len - static_cast<int>(sq.n) + static_cast<int>(tok);
    int2 vis = make_int2(0, 0);
    if (live && pos >= 0)
      vis = visible(a, pos, sq.len, a.prefix_lens ? __ldg(a.prefix_lens + tl.b) : 0,
                    a.doc_start ? __ldg(a.doc_start + sq.first + tok) : 0);
    if (vis.x >= vis.y) vis = make_int2(0x7fffffff, 0);
    const int pos0 = __shfl_sync(0xffffffffu, pos, 0);
    if (lane < kC) {
      sh.first[lane] = vis.x;
      sh.last[lane] = vis.y;
      sh.pos[lane] = static_cast<float>(pos - pos0);
      sh.slope[lane] = a.slopes && live ? __ldg(a.slopes + h) * kLog2e : 0.0f;
      sh.out[lane] = live ? (sq.first + tok) * a.hq + h : 0xffffffffu;
    }
    const int lo = __reduce_min_sync(0xffffffffu, vis.x), hi = __reduce_max_sync(0xffffffffu, vis.y);
    const int all_lo = __reduce_max_sync(0xffffffffu, live ? vis.x : 0);
    const int all_hi = __reduce_min_sync(0xffffffffu, live ? vis.y : 0x7fffffff);
    if (lane == 0) {
      sh.item = it;
      // Of the keys that the rows see, those of this part.
      const int64_t part = static_cast<int64_t>(a.part_blocks) * kBlock, from = any ? it.span.lo + it.part * part : 0;
      const int l = static_cast<int>(max(static_cast<int64_t>(lo), from));
      const int h = static_cast<int>(min(static_cast<int64_t>(hi), from + part));
      sh.lo = h > l ? l : 0;
      sh.hi = h > l ? h : 0;
      sh.rows = static_cast<int>(rows);
      sh.pos0 = pos0;
      sh.all_lo = all_lo;
      sh.all_hi = all_hi;
    }
  }
  __syncthreads();
  const uint32_t tmem = sh.tmem;
  const Tile tile = sh.item.tile;
  const uint32_t kvh = sh.item.kvh;
  const bool none = tile.b >= a.map.batch;
  const int t_base = sh.lo, end = sh.hi, nblk = (end - t_base + kBlock - 1) / kBlock;

  // A key's page and row in it, from the page table or, contiguous, at once.
  const int64_t base_row = (static_cast<int64_t>(a.map.table ? 0 : tile.b) * a.map.hkv + kvh) * a.map.size.d;
  const int64_t page_rows = static_cast<int64_t>(a.map.hkv) * a.map.size.d;
  const int32_t* table = a.map.table + (none ? 0 : static_cast<uint64_t>(tile.b) * a.map.per_seq);
  const auto find = [&](int j, int key, uint32_t* page, uint32_t* off) {
    const int t = t_base + max(nblk - 1 - j, 0) * kBlock + key;  // the newest keys first, as in the tile kernel
    *off = t;
    *page = j < nblk && t < end ? 0u : 0xffffffffu;
    if (a.map.table && *page == 0u) {
      const uint32_t i = a.map.size.div(t);
      *off -= i * a.map.size.d;
      *page = static_cast<uint32_t>(__ldg(table + i));
    }
  };
  const uint32_t pages = a.map.table ? a.map.pages : 1u;
  const auto wait = [&](uint64_t* bar, int phase) {
    const bool ok = __all_sync(0xffffffffu, wait_bar(bar, phase & 1, &sh.abort));
    if (!ok && lane == 0 && !sh.abort) {
      set_status(a.status, NVFP4_ERR_TIMEOUT);
      sh.abort = 1;
    }
    tc_fence_after();
    return ok;
  };

  // 104, 64, 64 and 24 registers a thread by warpgroup: the 512 x 64 that the CTA starts with.
  // (96, 64, 64 and 32, on 32 x 4001 keys: 16 rows 54 to 72 us instead of 56 to 72, 24 rows 62 and
  // with a cap 85 instead of 65 and 73, 32 rows 75 and 102 instead of 68 and 90.)
  if (warp < 4) {
    // ------------------------------------------------------------- softmax ---
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    // Q rows as f16, scaled by a power of two (exact) to below 1: 16 lanes a row.
    uint4 w[kN / 8];
#pragma unroll
    for (int i = 0; i < kN / 8; ++i) {
      const uint32_t lr = i * 8 + warp * 2 + (lane >> 4), out = lr < kC ? sh.out[lr] : 0xffffffffu;
      w[i] = make_uint4(0, 0, 0, 0);
      if (out != 0xffffffffu) {
        const uint32_t tk = out / a.hq;
        w[i] = __ldg(reinterpret_cast<const uint4*>(a.q + static_cast<int64_t>(tk) * a.ld_q + (out - tk * a.hq) * kD) + (lane & 15));
      }
    }
    bool coarse = false;  // a product of Q and K is below 2^19
#pragma unroll
    for (int i = 0; i < kN / 8; ++i) {
      const uint32_t lr = i * 8 + warp * 2 + (lane >> 4), c = lane & 15;
      uint32_t top = amax_bits_bf16x8(w[i]);
#pragma unroll
      for (int s = 1; s < 16; s <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
      const RowScale by = row_scale(top);
      if (c == 0 && lr < kC) {
        // No maximum yet: any score exceeds it.  (A row past the tile's has scores of 0.)
        const bool live = sh.out[lr] != 0xffffffffu;
        sh.mult[lr] = live ? score_factor(a.scale, by.up) : 0.0f;
        coarse = coarse || !(sh.mult[lr] <= 8.0f) || !(fabsf(sh.slope[lr]) * static_cast<float>(a.map.context) <= 0x1p21f);
        sh.minus[lr] = live ? FLT_MAX : 0.0f;
        sh.none[lr] = 0.0f;
      }
      float x[8];
      unpack_bf16x8(w[i], x);
      const uint4 f = q_chunk<kE1M2>(x, by.down);
      sts128(smem + C::kOffQ + (c >> 3) * (kN * 128) + lr * 128 + (((c ^ lr) & 7) << 4), f.x, f.y, f.z, f.w);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.q_full);
    // (Also the barrier after which all rows' multipliers are there.)  Scores that may
    // pass 2^22 are rounded before `minus` is added, as the maxima are: else an exponent
    // could be above the largest by the rounding of one product.
    const bool exact = any_of_128(coarse) || (kCap && a.cap > 0.0f);
    const auto bias = [&](float* x, int tk) {
      if (!a.slopes) return;
      const float tf = static_cast<float>(tk - sh.pos0);
#pragma unroll
      for (int n = 0; n < kC; n += 4) {
        const float4 f = *reinterpret_cast<const float4*>(&sh.slope[n]), at = *reinterpret_cast<const float4*>(&sh.pos[n]);
        x[n] = fmaf(-f.x, fabsf(at.x - tf), x[n]);
        x[n + 1] = fmaf(-f.y, fabsf(at.y - tf), x[n + 1]);
        x[n + 2] = fmaf(-f.z, fabsf(at.z - tf), x[n + 2]);
        x[n + 3] = fmaf(-f.w, fabsf(at.w - tf), x[n + 3]);
      }
    };
    const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
    const int key = warp * 32 + lane;
    float l[kC];
#pragma unroll
    for (int n = 0; n < kC; ++n) l[n] = 0.0f;
    bool ok = true;
    for (int j = 0; j < nblk; ++j) {
      const int b = j & 1, t0 = t_base + (nblk - 1 - j) * kBlock, tk = t0 + key;
      const uint32_t p_at = smem + C::kOffP + b * 2 * C::kB + key * 16;
      ok = wait(&sh.s_full[b], j >> 1);  // and so P of block j - 2 is used up
      const bool there = (sh.present[j & 3][warp] >> lane) & 1u;
      const bool open = t0 >= sh.all_lo && t0 + kBlock <= sh.all_hi && __all_sync(0xffffffffu, there);
      // The weights' exponents, score + minus.  Maxima move only where a weight would be
      // 2^11 times its row's maximum: then the scores alone, and the exponents once more.
      float x[kC];
      bool moved = false;
      for (const float* minus = sh.minus;;) {
        tmem_ld_cols<kC>(tmem + lanes + kColS + b * 32, x);
        tmem_wait_ld();
        if (exact) {
#pragma unroll
          for (int n = 0; n < kC; ++n) x[n] *= sh.mult[n];
          if (kCap && a.cap > 0.0f) cap_scores<kC>(x, a.cap * kLog2e);
          bias(x, tk);
#pragma unroll
          for (int n = 0; n < kC; ++n) x[n] += minus[n];
        } else {
#pragma unroll
          for (int n = 0; n < kC; n += 4) {
            const ulonglong2 m = *reinterpret_cast<const ulonglong2*>(&sh.mult[n]), c = *reinterpret_cast<const ulonglong2*>(&minus[n]);
            unpair(fma2(pair(x[n], x[n + 1]), m.x, c.x), x[n], x[n + 1]);
            unpair(fma2(pair(x[n + 2], x[n + 3]), m.y, c.y), x[n + 2], x[n + 3]);
          }
          bias(x, tk);
        }
        if (!open) {
          const int t = there ? tk : -1;  // below every first key
#pragma unroll
          for (int n = 0; n < kC; n += 4) {
            const int4 lo = *reinterpret_cast<const int4*>(&sh.first[n]), hi = *reinterpret_cast<const int4*>(&sh.last[n]);
            if (t < lo.x || t >= hi.x) x[n] = -INFINITY;
            if (t < lo.y || t >= hi.y) x[n + 1] = -INFINITY;
            if (t < lo.z || t >= hi.z) x[n + 2] = -INFINITY;
            if (t < lo.w || t >= hi.w) x[n + 3] = -INFINITY;
          }
        }
        if (minus == sh.minus) {
          if (moved) break;
          float most = -INFINITY;
#pragma unroll
          for (int n = 0; n < kC; n += 2) most = max3(x[n], x[n + 1], most);
          if (!any_of_128(most > kWeightLog2 + kRescaleLog2 || !ok)) break;
          minus = sh.none;
          continue;
        }
        // Each row's largest score in the block, by warp, then of all four.
#pragma unroll
        for (int n = 0; n < kC; ++n) {
          const float v = warp_max(x[n]);
          if (lane == 0) sh.top[warp][n] = v;
        }
        if (any_of_128(!ok)) {
          ok = false;
          break;  // a wait ran out: the four warps leave together
        }
        const auto top_of = [&](int n) { return max3(max3(sh.top[0][n], sh.top[1][n], sh.top[2][n]), sh.top[3][n], -INFINITY); };
        const auto shrink = [&](int n) {
          const float top = top_of(n), minus = sh.minus[n];
          return top + minus > kWeightLog2 + kRescaleLog2 ? ex2(kWeightLog2 - top - minus) : 1.0f;
        };
#pragma unroll
        for (int n = 0; n < kC; ++n) l[n] *= shrink(n);
        if (j > 0) {
          ok = wait(&sh.v_free[(j - 1) & 1], (j - 1) >> 1);
#pragma unroll 1
          for (int n0 = 0; n0 < kC; n0 += 8) {
            float o[8];
            tmem_ld_cols<8>(tmem + lanes + kColO + n0, o);
            tmem_wait_ld();
#pragma unroll
            for (int n = 0; n < 8; ++n) o[n] *= shrink(n0 + n);
            tmem_st8(tmem + lanes + kColO + n0, o);
          }
          tmem_wait_st();
        }
        const bool bad = any_of_128(!ok);  // also: every warp has read the old maxima
        if (warp == 0 && lane < kC && shrink(lane) != 1.0f) sh.minus[lane] = kWeightLog2 - top_of(lane);
        any_of_128(false);
        if (bad) {
          ok = false;
          break;
        }
        minus = sh.minus;
        moved = true;
      }
      if (!ok) break;
#pragma unroll
      for (int n = 0; n < kC; ++n) x[n] = ex2(x[n]);
#pragma unroll
      for (int n = 0; n < kC; n += 8) {
        if (kFull) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t xb = __float_as_uint(x[n + 2 * k]), yb = __float_as_uint(x[n + 2 * k + 1]);
            hi[k] = __byte_perm(xb, yb, 0x7632);
            lo[k] = bf16x2_rn(x[n + 2 * k] - __uint_as_float(xb & 0xFFFF0000u), x[n + 2 * k + 1] - __uint_as_float(yb & 0xFFFF0000u));
          }
          sts128(p_at + n * 256, hi[0], hi[1], hi[2], hi[3]);
          sts128(p_at + n * 256 + C::kB, lo[0], lo[1], lo[2], lo[3]);
        } else {
          sts128(p_at + n * 256, f16x2_rn(x[n], x[n + 1]), f16x2_rn(x[n + 2], x[n + 3]), f16x2_rn(x[n + 4], x[n + 5]),
                 f16x2_rn(x[n + 6], x[n + 7]));
        }
      }
      fence_proxy_async_smem();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.p_full[b]);
#pragma unroll
      for (int n = 0; n < kC; n += 2) add2(l[n], l[n + 1], x[n], x[n + 1]);
    }
    const bool done = wait(&sh.drain, 0);
    // ---- epilogue: thread = channel -----------------------------------------
#pragma unroll
    for (int n = 0; n < kC; ++n) {
#pragma unroll
      for (int x = 16; x; x >>= 1) l[n] += __shfl_xor_sync(0xffffffffu, l[n], x);
      if (lane == 0) sh.sum[warp][n] = l[n];
    }
    any_of_128(false);
    float o[kC];
    if (nblk > 0) {
      tmem_ld_cols<kC>(tmem + lanes + kColO, o);
      tmem_wait_ld();
    }
    const uint64_t rec0 = ((static_cast<uint64_t>(sh.item.tile_id) * a.map.hkv + kvh) * a.splits + sh.item.part) * kC;
    const bool joined = sh.item.span.parts > 1;
    const int channel = channel_of<kE1M2>(key);
    if (done && !none)
#pragma unroll
      for (int n = 0; n < kC; ++n) {
        if (n >= sh.rows) break;
        const float sum = nblk > 0 ? (sh.sum[0][n] + sh.sum[1][n]) + (sh.sum[2][n] + sh.sum[3][n]) : 0.0f;
        const float v = sum == 0.0f ? 0.0f : o[n];
        if (!(joined ? record_in_bounds<kC>(a, rec0 + n) : out_in_bounds(a, sh.out[n]))) continue;
        if (joined) {
          if (key == 0) a.ml_ws[rec0 + n] = make_float2(sum == 0.0f ? -INFINITY : -sh.minus[n], sum);
          a.o_ws[(rec0 + n) * kD + channel] = v;
        } else {
          const uint32_t bits = bf16x2_rn(v * per_sum(sum, a.gv), 0.0f);
          a.out[static_cast<uint64_t>(sh.out[n]) * kD + channel] = static_cast<uint16_t>(bits);
        }
      }
    tc_fence_before();
  } else if (warp < 8) {
    // ------------------------------------------------------------------- K ---
    const int w = warp - 4, key = w * 32 + lane;
    const uint32_t k_col = tmem + (static_cast<uint32_t>(w * 32) << 16);
    const uint8_t* codes = a.map.k_codes + base_row * 64;
    const uint8_t* scales = a.map.k_scales + base_row * 8;
    // The next block's row is in flight in registers, and those of the kAhead after
    // it on their way to L2, with V's; their pages are known.
    uint32_t page[kAhead + 1], off[kAhead + 1];
    uint4 c[4];
    uint2 sc;
    bool there;
    const auto load = [&] {
      there = page[0] < pages;
      const int64_t row = page[0] * page_rows + off[0];
      sc = there ? __ldg(reinterpret_cast<const uint2*>(scales + row * 8)) : make_uint2(0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = there ? __ldg(reinterpret_cast<const uint4*>(codes + row * 64) + i) : make_uint4(0, 0, 0, 0);
    };
    const auto prefetch = [&](int i) {
      if (page[i] >= pages) return;
      const int64_t at = base_row + page[i] * page_rows + off[i];
      if (!(at & 1) || off[i] == 0) {  // a line has two keys' codes
        prefetch_l2(a.map.k_codes + at * 64);
        prefetch_l2(a.map.v_codes + at * 64);
      }
      if (!(at & 15) || off[i] == 0) {  // and 16 keys' scales
        prefetch_l2(a.map.k_scales + at * 8);
        prefetch_l2(a.map.v_scales + at * 8);
      }
    };
#pragma unroll
    for (int i = 0; i <= kAhead; ++i) find(i, key, &page[i], &off[i]);
    load();
#pragma unroll
    for (int i = 1; i <= kAhead; ++i) prefetch(i);
    for (int j = 0; j < nblk; ++j) {
      const int b = j & 1;
      const uint32_t here = __ballot_sync(0xffffffffu, there);
      if (!wait(&sh.k_free[b], (j >> 1) ^ 1)) break;
      if (lane == 0) sh.present[j & 3][w] = here;
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // 32 channels
        const uint32_t word[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
        const uint32_t f = kv_scales16<kE1M2>(__byte_perm(sc.x, sc.y, 0x10 + 0x22 * i));
        const uint32_t f0 = __byte_perm(f, f, 0x1010), f1 = __byte_perm(f, f, 0x3232);
        uint32_t e[16];
#pragma unroll
        for (int k = 0; k < 4; ++k) scaled8<kE1M2>(word[k], k < 2 ? f0 : f1, e + 4 * k);
        tmem_st16(k_col + b * 64 + 16 * i, e);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        page[i] = page[i + 1];
        off[i] = off[i + 1];
      }
      load();
      find(j + 1 + kAhead, key, &page[kAhead], &off[kAhead]);
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.k_full[b]);
      prefetch(kAhead);
    }
  } else if (warp < 12) {
    // ------------------------------------------------------------------- V ---
    // Four lanes a key, 32 channels each; eight keys a warp and turn, four turns.
    const int w = warp - 8, sub = lane >> 2, qd = lane & 3;
    const uint8_t* codes = a.map.v_codes + base_row * 64 + 16 * qd;
    const uint8_t* scales = a.map.v_scales + base_row * 8 + 2 * qd;
    const bool sw = qd & 2;  // as in the tile kernel: eight lanes, eight bank groups
    uint32_t at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) at[k] = smem + operand_chunk(w * 8 + sub, 4 * qd + (sw ? k ^ 2 : k));
    uint32_t page[4], off[4], sc[4];
    uint4 c[4];
    const auto rows_of = [&](int j) {
#pragma unroll
      for (int it = 0; it < 4; ++it) find(j, it * 32 + w * 8 + sub, &page[it], &off[it]);
    };
    const auto load = [&] {
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const bool there = page[it] < pages;
        const int64_t row = page[it] * page_rows + off[it];
        c[it] = there ? __ldg(reinterpret_cast<const uint4*>(codes + row * 64)) : make_uint4(0, 0, 0, 0);
        sc[it] = there ? __ldg(reinterpret_cast<const uint16_t*>(scales + row * 8)) : 0u;
      }
    };
    rows_of(0);
    load();
    rows_of(1);
    for (int j = 0; j < nblk; ++j) {
      const int b = j & 1;
      if (!wait(&sh.v_free[b], (j >> 1) ^ 1)) break;
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const uint32_t g = kv_scales16<kE1M2>(sc[it]);
        const uint32_t g0 = __byte_perm(g, g, sw ? 0x3232 : 0x1010), g1 = __byte_perm(g, g, sw ? 0x1010 : 0x3232);
        const uint4 v = c[it];
        const uint32_t words[4] = {sw ? v.z : v.x, sw ? v.w : v.y, sw ? v.x : v.z, sw ? v.y : v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t e[4];
          scaled8<kE1M2>(words[k], k < 2 ? g0 : g1, e);
          if (kFull)
#pragma unroll
            for (int x = 0; x < 4; ++x) e[x] = bf16x2_of_f16x2(e[x]);
          sts128(at[k] + b * kOperand + it * 4096, e[0], e[1], e[2], e[3]);
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.v_full[b]);
      load();
      rows_of(j + 2);
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 24;");
    // ----------------------------------------------------------------- MMA ---
    if (warp == 12) {
      const bool leader = elect_one();
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      const auto qk = [&](int j) {
        const int b = j & 1;
        if (leader) {
          constexpr uint32_t kIdesc = (1u << 4) | (static_cast<uint32_t>(kN / 8) << 17) | (8u << 24);
#pragma unroll
          for (int s = 0; s < 8; ++s) {
            const uint32_t at = C::kOffQ + (s >> 2) * (kN * 128) + (s & 3) * 32;
            mma_ts(tm + kColS + b * 32, tm + b * 64 + s * 8, ((smem + at) & 0x3FFFFu) >> 4, kIdesc, s != 0);
          }
          tc_commit(&sh.s_full[b]);
          tc_commit(&sh.k_free[b]);
        }
        __syncwarp();
      };
      bool ok = nblk > 0 && wait(&sh.q_full, 0);
      for (int j = 0; j < 2 && j < nblk && ok; ++j)
        if ((ok = wait(&sh.k_full[j], 0))) qk(j);
      for (int j = 0; j < nblk && ok; ++j) {
        const int b = j & 1;
        if (!wait(&sh.v_full[b], j >> 1) || !wait(&sh.p_full[b], j >> 1)) break;
        if (leader) {
          // A = V^T (bit 15: stored with M contiguous), B = P (bit 16: N), 16 keys a step.
          constexpr uint32_t kIdesc = (1u << 4) | (3u << 15) | (static_cast<uint32_t>(kN / 8) << 17) | (8u << 24) |
                                      (kFull ? (1u << 7) | (1u << 10) : 0u);
          const uint32_t v = operand_desc(smem + b * kOperand), p = plain_desc(smem + C::kOffP + b * 2 * C::kB);
#pragma unroll
          for (int s = 0; s < (kFull ? 16 : 8); ++s)
            mma_v_p(tm + kColO, v + (((s & 7) * 2048) >> 4), p + (((s >> 3) * C::kB + (s & 7) * 256) >> 4), kIdesc,
                    j != 0 || s != 0);
          tc_commit(&sh.v_free[b]);
        }
        __syncwarp();
        // P is there, and so the scores that it came from are read.
        if (j + 2 < nblk) {
          if (!wait(&sh.k_full[b], (j + 2) >> 1)) break;
          qk(j + 2);
        }
      }
      // Nothing that was issued, MMA or arrival, outlives the CTA.
      if (leader) tc_commit(&sh.drain);
      mbar_wait_bounded(&sh.drain, 0, nullptr, kDrainLimitNs);
      __syncwarp();
    }
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kRowsTmem);
  }
}

template <int kC, bool kE1M2>
ExtendLaunch launch(bool cap, bool full) {
  const ExtendKernel k = full  ? extend_rows_kernel<kC, kE1M2, true, true>
                         : cap ? extend_rows_kernel<kC, kE1M2, true, false>
                               : extend_rows_kernel<kC, kE1M2, false, false>;
  return {k, kRowsThreads, RowsConfig<kC>::kBytes};
}
template <bool kE1M2>
ExtendLaunch pick(int rows, bool cap, bool full) {
  if (rows == 8) return {extend_rows_kernel<8, kE1M2, true, true>, kRowsThreads, RowsConfig<8>::kBytes};  // else extend_decode.cu
  if (rows == 16) return launch<16, kE1M2>(cap, full);
  return rows == 24 ? launch<24, kE1M2>(cap, full) : launch<32, kE1M2>(cap, full);
}

}  // namespace

ExtendLaunch extend_rows(int rows, bool e1m2, bool cap, bool full) {
  return e1m2 ? pick<true>(rows, cap, full) : pick<false>(rows, cap, full);
}

}  // namespace nvfp4
