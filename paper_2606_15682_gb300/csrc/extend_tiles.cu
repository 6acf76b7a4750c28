// Attention of new tokens, many rows of a sequence and KV head.
//
// A CTA holds 256 rows as two 128-row tiles, streams blocks of 128 keys, and
// computes S = Q K^T and O += P V with tcgen05.mma kind::f16, 64 keys at a time.
//   warps 0-3, 4-7  softmax of tile 0 and 1 (thread = row): read S from TMEM,
//                   write P over it, rescale O where a maximum moved
//   warps 8-15      dequantize the blocks' K and V into shared memory (f16,
//                   exact: an E2M1 x E4M3 product has at most 6 significant
//                   bits), one warpgroup each
//   warps 16, 17    issue the MMAs of tile 0 and 1 (by one warp, the waits before
//                   one tile's MMAs left the tensor core idle: 4300 cycles a
//                   block); warps 18, 19 complete their warpgroup and idle
// TMEM holds O of both tiles (256 columns) and two 64-column S of each tile: while
// a softmax works on one, the other is already multiplied, so that neither the
// softmax nor the tensor core waits for the other's latency.  (One 128-column S
// a tile, whose QK^T has to wait for PV: 4230 cycles per block and two tiles;
// N = 64 costs the QK^T a half more shared-memory reads of Q.)
// With at most 128 rows the second tile takes the same rows with every second
// block, and the two are joined at the end.
//
// A prompt of 4096 (40 on 8 heads, causal) takes 182 us, 0.49 of the measured bf16
// rate; a chunk of 2048 on 16384 keys (64 on 8 heads) 926 us, 0.58, 1103 with a bias,
// 1422 with a cap, 1722 with both.  A step of 64 keys and both tiles takes some 1790 cycles where the
// MMAs need 1250 (48 for 128 x 64 x 16 with Q from shared memory, 64 for 128 x 128 x 16):
// the rest is the ring softmax, PV, QK^T, softmax, each link short of issue slots
// beside the dequantizing warps.  (Issuers per half, one thread as issuer, or the two
// tiles in fixed turns: 1 to 30 % slower.)
#include "extend_attention.cuh"

namespace nvfp4 {
namespace {

constexpr int kTileThreads = 20 * 32;
constexpr int kDequantWarp = 8, kMmaWarp = 16;
constexpr uint32_t kOffK = 2 * kOperand, kOffV = 4 * kOperand;
constexpr uint32_t kTileSmem = 6 * kOperand + 1024;  // and alignment

// f16 operands, fp32 accumulator, 128 x 64 (QK^T) and 128 x 128; bit 16: B is
// stored with N contiguous.
constexpr uint32_t kIdescQK = (1u << 4) | (8u << 17) | (8u << 24);
constexpr uint32_t kIdescPV = (1u << 4) | (1u << 16) | (16u << 17) | (8u << 24);
constexpr uint32_t kIdescPVFull = kIdescPV | (1u << 7) | (1u << 10);  // bf16 operands
// What a row's scores are made of: x = s * mult in the log2 domain; capped,
// x = c log2(e) tanh(s * mult / (c log2(e))) (cap_scores).
struct RowScore {
  float mult;   // softmax_scale * g_K * log2(e) / the query's scale
  float slope;  // slopes[h] * log2(e)
};

struct TileShared {
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2][2], p_full[2][2], o_done[2], q_full, drain[2];
  uint32_t tmem;
  Tile tile;
  Seq seq;
  int lo, hi;       // keys that some row of the tile sees
  float mult[kTileRows];
  float2 ml[kBlock];             // tile 1's (max, sum), for the join
  alignas(16) uint32_t present[4][4];  // bit per key of a block: loaded, in the last four blocks' slots
  volatile int abort;
};

// 32 scores of a row, capped and biased, in the log2 domain.  `behind`: no key is
// newer than the query, in the whole warp.  kMods: kCap, kBias, or both (either may be
// absent); each has a kernel of its own, since in a longer loop every role waits more
// for its instructions (both in one: a chunk of 2048 on 16384 keys with a bias
// 1263 us instead of 1113, with a cap 1528 instead of 1424).
constexpr int kCap = 1, kBias = 2;
template <int kMods>
__device__ __forceinline__ void score32(float* s, const RowScore& rs, const ExtendArgs& a, int p_minus_t0, bool behind) {
  const bool capped = kMods == kCap || (kMods == (kCap | kBias) && a.cap > 0.0f);
  const bool biased = kMods == kBias || (kMods == (kCap | kBias) && a.slopes);
  if (capped) {
    // (Finite, so that a score of 0 stays 0 whatever the query's scale.)
    const float out = a.cap * kLog2e, in = fminf(rs.mult / out, FLT_MAX);
    cap_scores<32>(s, in, out);
  } else if (!(biased && behind)) {
#pragma unroll
    for (int i = 0; i < 32; ++i) s[i] *= rs.mult;
  }
  if (!biased) return;
  const float d = static_cast<float>(p_minus_t0);
  if (behind) {
    // s - slope (d - i), two at a time; the terms slope (i - d) by four additions from exact starts.
    const float base = -rs.slope * d;
    const uint64_t mult = both(capped ? 1.0f : rs.mult), step = both(8.0f * rs.slope);
    uint64_t b[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) b[k] = pair(fmaf(rs.slope, 2.0f * k, base), fmaf(rs.slope, 2.0f * k + 1.0f, base));
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
      uint64_t& t = b[(i >> 1) & 3];
      unpair(fma2(pair(s[i], s[i + 1]), mult, t), s[i], s[i + 1]);
      t = add2(t, step);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) s[i] = fmaf(-rs.slope, fabsf(d - static_cast<float>(i)), s[i]);
  }
}

// kFull: weights as two bf16 terms (16 significant bits at fp32's range) and V in
// bf16, a second PV product per block.  In f16 a weight below 2^-28 of the row's
// largest is lost, which shows only where all heavier keys hold a zero in a
// channel: among few keys.
template <bool kE1M2, int kMods, bool kFull>
__global__ void __launch_bounds__(kTileThreads, 1) extend_tile_kernel(const ExtendArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ TileShared sh;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.k_full[i], 4 + lost_arrivals(a, i));
      mbar_init(&sh.k_empty[i], 2);
      mbar_init(&sh.v_full[i], 4);
      mbar_init(&sh.v_empty[i], 2);
      for (int v = 0; v < 2; ++v) {
        mbar_init(&sh.s_full[i][v], 1);
        mbar_init(&sh.p_full[i][v], 4);
      }
      mbar_init(&sh.o_done[i], 1);
      mbar_init(&sh.drain[i], 1);
    }
    mbar_init(&sh.q_full, 8);
    sh.abort = 0;
    sh.lo = 0x7fffffff;
    sh.hi = 0;
    fence_mbar_init();
  }
  if (warp == kMmaWarp) tmem_alloc(&sh.tmem, 512);
  // The next kernel's CTAs, which may allocate as well, start once this one has its columns.
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_wait_and_release();
  // Item: split fastest, then KV head, then tile.
  const uint32_t split = blockIdx.x % a.splits, rest = blockIdx.x / a.splits;
  const uint32_t tile_id = rest / a.map.hkv, kvh = rest - tile_id * a.map.hkv;
  if (warp == 0) {
    const Tile t = find_tile<kTileRows>(a, tile_id);
    if (lane == 0) {
      sh.tile = t;
      if (t.b < a.map.batch) sh.seq = sequence(a, t.b);
    }
  }
  __syncthreads();
  const uint32_t tmem = sh.tmem;
  const bool none = sh.tile.b >= a.map.batch;  // more CTAs than tiles
  const Seq seq = sh.seq;
  const uint32_t group = a.group.d;
  const uint32_t rows = none ? 0 : min(seq.n * group - sh.tile.row0, static_cast<uint32_t>(kTileRows));
  const bool two = rows > 128;

  // Row of a softmax thread: tile 1 has rows 128.. of a large tile, or rows 0.. again.
  const int t = warp >> 2;
  const uint32_t in_tile = threadIdx.x & 127, local = (two ? t * 128u : 0u) + in_tile;
  const bool live = warp < kDequantWarp && local < rows;
  const uint32_t r = sh.tile.row0 + (live ? local : 0), tok = a.group.div(r), head = kvh * group + (r - tok * group);
  int2 vis = make_int2(0, 0);
  const int p = seq.len - static_cast<int>(seq.n) + static_cast<int>(tok);
  if (live && !none && p >= 0)
    vis = visible(a, p, seq.len, a.prefix_lens ? __ldg(a.prefix_lens + sh.tile.b) : 0,
                  a.doc_start ? __ldg(a.doc_start + seq.first + tok) : 0);
  if (vis.x >= vis.y) vis = make_int2(0x7fffffff, 0);
  if (warp < kDequantWarp) {
    const int lo = __reduce_min_sync(0xffffffffu, vis.x), hi = __reduce_max_sync(0xffffffffu, vis.y);
    if (lane == 0) {
      atomicMin(&sh.lo, lo);
      atomicMax(&sh.hi, hi);
    }
  }
  __syncthreads();
  // The tile's blocks of keys, and this CTA's part of them.
  const int lo = sh.hi > sh.lo ? sh.lo : 0, total = sh.hi > sh.lo ? (sh.hi - lo + kBlock - 1) / kBlock : 0;
  const int per = (total + static_cast<int>(a.splits) - 1) / static_cast<int>(a.splits);
  const int j0 = min(static_cast<int>(split) * per, total), nblk = min(per, total - j0);
  const int t_base = lo + j0 * kBlock;
  const int subs_of[2] = {two ? 2 * nblk : (nblk + 1) / 2 * 2, two ? 2 * nblk : nblk / 2 * 2};  // 64-key steps of a tile

  if (warp < kDequantWarp) {
    // ------------------------------------------------------------- softmax ---
    asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
    // Q rows as f16: 16 lanes a row, two rows a turn, 32 rows a warp.  Each row is
    // scaled by a power of two (exact) to below 1; `mult` undoes it.
    if (two || warp < 4) {
      const int c = lane & 15;
      uint4 w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t lr = warp * 32 + 2 * i + (lane >> 4);
        const uint32_t rr = sh.tile.row0 + (lr < rows ? lr : 0), tk = a.group.div(rr);
        w[i] = lr < rows ? __ldg(reinterpret_cast<const uint4*>(a.q + static_cast<int64_t>(seq.first + tk) * a.ld_q +
                                                                (kvh * group + rr - tk * group) * kD) + c)
                         : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t lr = warp * 32 + 2 * i + (lane >> 4);
        uint32_t top = amax_bits_bf16x8(w[i]);
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
        const RowScale by = row_scale(top);
        if (c == 0) sh.mult[lr] = score_factor(a.scale, by.up);
        float x[8];
        unpack_bf16x8(w[i], x);
        const uint4 f = q_chunk<kE1M2>(x, by.down);
        sts128(smem + (lr >> 7) * kOperand + operand_chunk(lr & 127, c), f.x, f.y, f.z, f.w);
      }
      fence_proxy_async_smem();
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.q_full);
    if (!two) asm volatile("bar.sync 1, 256;" ::: "memory");  // tile 1 reads the multipliers of tile 0's rows
    const int subs = subs_of[t];
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_tile = tmem + lanes + t * 128, o_col = tmem + lanes + 256 + t * 128;
    RowScore rs;
    rs.mult = sh.mult[local];  // rows past the tile's have one too, of their own warp or behind the barrier
    rs.slope = (kMods & kBias) && a.slopes && live ? __ldg(a.slopes + head) * kLog2e : 0.0f;
    // Keys that every row of the warp sees need no mask.
    const int all_lo = __reduce_max_sync(0xffffffffu, live ? vis.x : 0);
    const int all_hi = __reduce_min_sync(0xffffffffu, live ? vis.y : 0x7fffffff);
    const int p_min = __reduce_min_sync(0xffffffffu, live ? p : 0x7fffffff - 64);
    // The product and the sum round once, the maximum was rounded by itself: an exponent
    // may exceed the largest by half a unit of the maximum's last place.  A product of Q
    // and K is below 2^19; where scores may pass 2^22 they are rounded first too.
    const bool coarse = kMods == 0 && __any_sync(0xffffffffu, !(rs.mult <= 8.0f));
    const float to_log2 = kMods || coarse ? 1.0f : rs.mult;
    const uint64_t to_log2x2 = both(to_log2);
    float minus = FLT_MAX, l0 = 0.0f, l1 = 0.0f;  // no maximum yet: any score exceeds it
    bool ok = true;
    for (int v = 0; v < subs; ++v) {
      const int j = two ? v >> 1 : (v & ~1) + t, hf = v & 1, t0 = t_base + (nblk - 1 - j) * kBlock + 64 * hf;
      const uint32_t s_col = s_tile + 64 * hf;
      ok = __all_sync(0xffffffffu, wait_bar(&sh.s_full[t][hf], (v >> 1) & 1, &sh.abort));
      if (!ok) break;
      tc_fence_after();
      const uint2 pres = *reinterpret_cast<const uint2*>(&sh.present[j & 3][2 * hf]);
      // The row's scores, all in registers, and their maximum.
      float s[64];
      tmem_ld32(s_col, s);
      tmem_ld32(s_col + 32, s + 32);
      tmem_wait_ld();
      if (__builtin_expect(coarse, false)) {
#pragma unroll
        for (int k = 0; k < 64; ++k) s[k] *= rs.mult;
      }
      if (kMods) {
#pragma unroll
        for (int k = 0; k < 64; k += 32) score32<kMods>(s + k, rs, a, p - t0 - k, t0 + 64 <= p_min + 1);
      }
      if (t0 < all_lo || t0 + 64 > all_hi || (pres.x & pres.y) != 0xffffffffu) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int a0 = max(vis.x - (t0 + 32 * c), 0), a1 = min(vis.y - (t0 + 32 * c), 32);
          const uint32_t mask = a1 > a0 ? (c ? pres.y : pres.x) & (0xffffffffu << a0) & (0xffffffffu >> (32 - a1)) : 0u;
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (!((mask >> k) & 1u)) s[32 * c + k] = -INFINITY;
        }
      }
      float tops[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        tops[c] = fmaxf(s[c], s[c + 4]);
#pragma unroll
        for (int k = 8; k < 64; k += 8) tops[c] = max3(s[k + c], s[k + c + 4], tops[c]);
      }
      const float top = fmaxf(max3(tops[0], tops[1], tops[2]), tops[3]) * to_log2;
      const bool up = top + minus > kWeightLog2 + kRescaleLog2;
      if (__any_sync(0xffffffffu, up)) {
        const float shrink = up ? ex2(kWeightLog2 - top - minus) : 1.0f;  // 0 where there was none
        if (up) minus = kWeightLog2 - top;
        l0 *= shrink;
        l1 *= shrink;
        if (v > 0) {
          ok = __all_sync(0xffffffffu, wait_bar(&sh.o_done[t], (v - 1) & 1, &sh.abort));
          if (!ok) break;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < 4; ++c) {
            float o[32];
            tmem_ld32(o_col + 32 * c, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] *= shrink;
            tmem_st16(o_col + 32 * c, reinterpret_cast<uint32_t*>(o));
            tmem_st16(o_col + 32 * c + 16, reinterpret_cast<uint32_t*>(o) + 16);
          }
        }
      }
      const uint64_t minus2 = both(minus);
      // The weights, over the scores they came from.
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t w[16], rest[kFull ? 16 : 1];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          float x = s[32 * c + 2 * k], y = s[32 * c + 2 * k + 1];
          fma2(x, y, to_log2x2, minus2);
          x = ex2(x);
          y = ex2(y);
          add2(l0, l1, x, y);
          if (kFull) {
            const uint32_t xb = __float_as_uint(x), yb = __float_as_uint(y);
            w[k] = __byte_perm(xb, yb, 0x7632);
            rest[k] = bf16x2_rn(x - __uint_as_float(xb & 0xFFFF0000u), y - __uint_as_float(yb & 0xFFFF0000u));
          } else {
            w[k] = f16x2_rn(x, y);
          }
        }
        tmem_st16(s_col + 16 * c, w);
        if (kFull) tmem_st16(s_col + 32 + 16 * c, rest);
      }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.p_full[t][hf]);
    }
    // The tile's last MMA.  (Not by o_done, whose last two phases may both have
    // passed by now, which a parity does not tell from none.)
    if (ok && subs > 0) {
      ok = __all_sync(0xffffffffu, wait_bar(&sh.drain[t], 0, &sh.abort));
      tc_fence_after();
    }
    if (!ok && lane == 0 && !sh.abort) {
      set_status(a.status, NVFP4_ERR_TIMEOUT);
      sh.abort = 1;
    }
    const float l = l0 + l1, m = l == 0.0f ? -INFINITY : -minus;  // weights are 2^(score - m)
    // A tile that took the other blocks of the same rows hands over its part.
    float* hand = reinterpret_cast<float*>(smem_raw + (smem - smem_u32(smem_raw)) + kOffK);  // [channel][row]
    float other_m = -INFINITY, other_l = 0.0f;
    if (!two) {
      asm volatile("bar.sync 1, 256;" ::: "memory");  // neither tile's MMAs read K any more
      if (t == 1) {
        sh.ml[in_tile] = make_float2(m, l);
        if (ok && subs > 0) {
          for (int c = 0; c < 4; ++c) {
            float o[32];
            tmem_ld32(o_col + 32 * c, o);
            tmem_wait_ld();
#pragma unroll
            for (int k = 0; k < 32; ++k) hand[(32 * c + k) * 128 + in_tile] = o[k];
          }
        }
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      const float2 other = sh.ml[in_tile];
      if (t == 0 && subs_of[1] > 0) {
        other_m = other.x;
        other_l = other.y;
      }
    }
    if (ok && !none && (two || t == 0)) {
      // Every QK^T is done: the warp's 32 rows of Q hold its output until the
      // stores, which take whole rows.
      const float big = fmaxf(m, other_m);
      const float w0 = m == -INFINITY ? 0.0f : ex2(m - big), w1 = other_m == -INFINITY ? 0.0f : ex2(other_m - big);
      const float sum = w0 * l + w1 * other_l;
      const float f = a.splits > 1 ? 1.0f : per_sum(sum, a.gv);
      const uint64_t rec0 = ((static_cast<uint64_t>(tile_id) * a.map.hkv + kvh) * a.splits + split) * kTileRows;
      if (a.splits > 1 && live && record_in_bounds<kTileRows>(a, rec0 + local)) a.ml_ws[rec0 + local] = make_float2(big, sum);
      const uint32_t stage = smem + warp * 8192, row0 = local - lane;
      const auto at = [&](uint32_t row, uint32_t c) { return stage + row * 256 + ((c ^ (row & 7)) << 4); };
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        float o[32];
        if (subs > 0) {
          tmem_ld32(o_col + 32 * c, o);
          tmem_wait_ld();
        }
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          o[k] = subs > 0 && w0 != 0.0f ? o[k] * w0 : 0.0f;
          if (w1 != 0.0f) o[k] = fmaf(hand[(32 * c + k) * 128 + in_tile], w1, o[k]);
          o[k] *= f;
        }
        if (a.splits == 1) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t w[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) w[x] = bf16x2_rn(o[place_of<kE1M2>(8 * k + 2 * x)], o[place_of<kE1M2>(8 * k + 2 * x + 1)]);
            sts128(at(lane, 4 * c + k), w[0], w[1], w[2], w[3]);
          }
          continue;
        }
        // A record in fp32: 128 bytes of each row at a time.
#pragma unroll
        for (int k = 0; k < 8; ++k)
          sts128(at(lane, k), __float_as_uint(o[place_of<kE1M2>(4 * k)]), __float_as_uint(o[place_of<kE1M2>(4 * k + 1)]),
                 __float_as_uint(o[place_of<kE1M2>(4 * k + 2)]), __float_as_uint(o[place_of<kE1M2>(4 * k + 3)]));
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t row = 4 * i + (lane >> 3);
          if (row0 + row < rows && record_in_bounds<kTileRows>(a, rec0 + row0 + row))
            reinterpret_cast<uint4*>(a.o_ws + (rec0 + row0 + row) * kD)[8 * c + (lane & 7)] = lds128(at(row, lane & 7));
        }
        __syncwarp();
      }
      if (a.splits == 1) {
        __syncwarp();
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
          const uint32_t row = 2 * i + (lane >> 4);
          if (row0 + row >= rows) continue;
          const uint32_t rr = sh.tile.row0 + row0 + row, tk = a.group.div(rr);
          const uint64_t to = static_cast<uint64_t>(seq.first + tk) * a.hq + kvh * group + rr - tk * group;
          if (out_in_bounds(a, to)) reinterpret_cast<uint4*>(a.out + to * kD)[lane & 15] = lds128(at(row, lane & 15));
        }
      }
    }
    tc_fence_before();
  } else if (warp < kMmaWarp) {
    // ---------------------------------------------------------- dequantize ---
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    // Four lanes a key: 16 bytes (32 channels) of its codes and two scale bytes
    // each, so a warp's load covers 8 keys' rows; four turns an operand.  One
    // warpgroup takes all K, the other all V; where the tiles take a block each,
    // the even and the odd blocks.  The next operand is in flight, the rows of the
    // one after it are known.
    const int wg = (warp >> 2) & 1, w = warp & 3, sub = lane >> 2, qd = lane & 3;
    const int end = sh.hi, operands = two ? nblk : (nblk + 1 - wg) / 2 * 2;
    const auto is_v = [&](int q) { return two ? wg : q & 1; };
    const auto block = [&](int q) { return two ? q : (q & ~1) + wg; };
    const int64_t base_row =
        (static_cast<int64_t>(a.map.table ? 0 : sh.tile.b) * a.map.hkv + kvh) * a.map.size.d;  // contiguous: of token 0
    const int64_t page_rows = static_cast<int64_t>(a.map.hkv) * a.map.size.d;
    // Of the operand that is loaded next: the page (contiguous: 0) and the row in it.
    uint32_t page[4], off[4];
    uint4 codes[4];
    uint32_t scales[4], here = 0;
    constexpr uint32_t kNone = 0xffffffffu;
    const uint32_t pages = a.map.table ? a.map.pages : 1u;
    const auto find = [&](int q) {
      // The blocks from the last to the first: the newest keys tend to have the
      // largest scores (with a distance bias, all of them), so maxima settle early.
      const int t0 = t_base + max(nblk - 1 - block(q), 0) * kBlock + w * 8 + sub;
      const int stop = q < operands && block(q) < nblk ? end : 0;
      const int32_t* table = a.map.table + static_cast<uint64_t>(sh.tile.b) * a.map.per_seq;
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        off[it] = t0 + it * 32;
        page[it] = t0 + it * 32 < stop ? 0u : kNone;
        if (a.map.table && page[it] == 0u) {
          const uint32_t i = a.map.size.div(off[it]);
          off[it] -= i * a.map.size.d;
          page[it] = static_cast<uint32_t>(__ldg(table + i));
        }
      }
    };
    const auto load = [&](int q) {
      const uint8_t* c = (is_v(q) ? a.map.v_codes : a.map.k_codes) + base_row * 64 + 16 * qd;
      const uint8_t* s = (is_v(q) ? a.map.v_scales : a.map.k_scales) + base_row * 8 + 2 * qd;
      here = 0;
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const bool ok = page[it] < pages;
        const int64_t row = page[it] * page_rows + off[it];
        codes[it] = ok ? __ldg(reinterpret_cast<const uint4*>(c + row * 64)) : make_uint4(0, 0, 0, 0);
        scales[it] = ok ? __ldg(reinterpret_cast<const uint16_t*>(s + row * 8)) : 0u;
        here |= ok ? 1u << it : 0u;
      }
    };
    // Lanes of the second 64 channels start with their other pair of words, so that
    // eight lanes' chunks meet eight different bank groups.
    const bool sw = qd & 2;
    uint32_t at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) at[k] = smem + operand_chunk(w * 8 + sub, 4 * qd + (sw ? k ^ 2 : k));
    const auto store = [&](uint32_t offset, bool bf16) {
#pragma unroll
      for (int it = 0; it < 4; ++it) {
        const uint32_t g = kv_scales16<kE1M2>(scales[it]);
        const uint32_t g0 = __byte_perm(g, g, sw ? 0x3232 : 0x1010), g1 = __byte_perm(g, g, sw ? 0x1010 : 0x3232);
        const uint4 v = codes[it];
        const uint32_t words[4] = {sw ? v.z : v.x, sw ? v.w : v.y, sw ? v.x : v.z, sw ? v.y : v.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t e[4];
          scaled8<kE1M2>(words[k], k < 2 ? g0 : g1, e);
          if (bf16)
#pragma unroll
            for (int x = 0; x < 4; ++x) e[x] = bf16x2_of_f16x2(e[x]);
          sts128(at[k] + offset + it * 4096, e[0], e[1], e[2], e[3]);  // 32 rows of 128 bytes further
        }
      }
    };
    // False: a wait ran out.
    const auto operand = [&](int q) {
      const int j = block(q), st = j & 1;
      if (!__all_sync(0xffffffffu, wait_bar(is_v(q) ? &sh.v_empty[st] : &sh.k_empty[st], ((j >> 1) & 1) ^ 1, &sh.abort)))
        return false;
      if (is_v(q)) {
        store(kOffV + st * kOperand, kFull);
      } else {
        // Which keys are there: byte it * 4 + w has this warp's 8 keys of turn it.
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          uint32_t v = __ballot_sync(0xffffffffu, qd == 0 && ((here >> it) & 1u));  // bits 0, 4, 8, ...
          v = (v | v >> 3) & 0x03030303u;
          v = (v | v >> 6) & 0x000F000Fu;
          v = (v | v >> 12) & 0xFFu;
          if (lane == 0) reinterpret_cast<uint8_t*>(sh.present[j & 3])[it * 4 + w] = static_cast<uint8_t>(v);
        }
        store(kOffK + st * kOperand, false);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(is_v(q) ? &sh.v_full[st] : &sh.k_full[st]);
      load(q + 1);
      find(q + 2);
      return true;
    };
    find(0);
    load(0);
    find(1);
    for (int q = 0; q < operands; ++q)
      if (!operand(q)) {
        if (lane == 0 && !sh.abort) {
          set_status(a.status, NVFP4_ERR_TIMEOUT);
          sh.abort = 1;
        }
        break;
      }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    if (warp < kMmaWarp + 2) {
      // --------------------------------------------------------------- MMA ---
      // The warp stays converged, so that descriptors live in uniform registers;
      // one lane issues.
      const bool leader = elect_one();
      bool ok = true;
      auto wait = [&](uint64_t* bar, int phase) {
        ok = ok && __all_sync(0xffffffffu, wait_bar(bar, phase & 1, &sh.abort));
        tc_fence_after();
        return ok;
      };
      auto commit = [&](uint64_t* bar) {
        if (leader) tc_commit(bar);
      };
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      // Step v of tile t: half v & 1 of its block v >> 1.
      const int t = warp - kMmaWarp, subs = subs_of[t];
      const uint32_t s_tile = tm + t * 128, o_tile = tm + 256 + t * 128;
      const auto block_of = [&](int v) { return two ? v >> 1 : (v & ~1) + t; };
      // A buffer is free when both tiles are done with it, or the one that has it.
      const auto release = [&](uint64_t* bar) {
        commit(bar);
        if (!two) commit(bar);
      };
      const auto qk = [&](int v) {
        const int j = block_of(v), st = j & 1, hf = v & 1;
        if (!hf && !wait(&sh.k_full[st], j >> 1)) return;
        const uint32_t q = operand_desc(smem + (two ? t : 0) * kOperand), k = operand_desc(smem + kOffK + st * kOperand + hf * 8192);
        if (leader) {
#pragma unroll
          for (int s = 0; s < 8; ++s) {
            const uint32_t at = ((s >> 2) * (kOperand / 2) + (s & 3) * 32) >> 4;
            mma_ss(s_tile + hf * 64, q + at, k + at, kIdescQK, s != 0);
          }
          tc_commit(&sh.s_full[t][hf]);
        }
        if (hf) release(&sh.k_empty[st]);
      };
      const auto pv = [&](int v) {
        const int j = block_of(v), st = j & 1, hf = v & 1;
        if (!hf && !wait(&sh.v_full[st], j >> 1)) return;
        if (!wait(&sh.p_full[t][hf], v >> 1)) return;
        const uint32_t vd = operand_desc(smem + kOffV + st * kOperand + hf * 8192), p = s_tile + hf * 64;
        if (leader) {
#pragma unroll
          for (int s = 0; s < (kFull ? 8 : 4); ++s)
            mma_ts(o_tile, p + s * 8, vd + (((s & 3) * 2048) >> 4), kFull ? kIdescPVFull : kIdescPV, v != 0 || s != 0);
          tc_commit(&sh.o_done[t]);
        }
        if (hf) release(&sh.v_empty[st]);
      };
      wait(&sh.q_full, 0);
      for (int v = 0; v < 2 && v < subs && ok; ++v) qk(v);
      for (int v = 0; v < subs && ok; ++v) {
        pv(v);
        if (ok && v + 2 < subs) qk(v + 2);
      }
      if (!ok && leader && !sh.abort) {
        set_status(a.status, NVFP4_ERR_TIMEOUT);
        sh.abort = 1;
      }
      // Nothing that was issued, MMA or arrival, outlives the CTA.
      commit(&sh.drain[t]);
      mbar_wait_bounded(&sh.drain[t], 0, nullptr, kDrainLimitNs);
      __syncwarp();
    }
  }
  __syncthreads();
  if (warp == kMmaWarp) {
    tc_fence_after();
    tmem_relinquish();
    tmem_dealloc(tmem, 512);
  }
}

template <bool kE1M2>
ExtendKernel pick(int mods, bool full) {
  if (full) return mods ? extend_tile_kernel<kE1M2, kCap | kBias, true> : extend_tile_kernel<kE1M2, 0, true>;
  switch (mods) {
    case 0: return extend_tile_kernel<kE1M2, 0, false>;
    case kCap: return extend_tile_kernel<kE1M2, kCap, false>;
    case kBias: return extend_tile_kernel<kE1M2, kBias, false>;
  }
  return extend_tile_kernel<kE1M2, kCap | kBias, false>;
}

}  // namespace

ExtendLaunch extend_tiles(bool e1m2, bool cap, bool bias, bool full) {
  const int mods = (cap ? kCap : 0) | (bias ? kBias : 0);
  return {e1m2 ? pick<true>(mods, full) : pick<false>(mods, full), kTileThreads, kTileSmem};
}

}  // namespace nvfp4
