// Attention of new tokens (one, a few, a chunk, a whole prompt) over the 4-bit
// cache that already holds them, contiguous or paged: scores optionally capped
// and biased by distance, keys limited by causality, window, prefix, document.
#include "kv_pages.cuh"

namespace nvfp4 {
namespace {

constexpr int kD = 128;
constexpr float kLog2e = 1.4426950408889634f;

// The running maximum moves only when a score exceeds it by 2^11: weights are kept
// as 2^4 w, at most 2^15 in f16, whose steps end at 2^-28 of the maximum.
constexpr float kRescaleLog2 = 11.0f;
constexpr float kWeightLog2 = 4.0f;

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
  uint32_t tiles, tiles_per_seq;  // row tiles; of each sequence where q_start is null
  uint32_t splits;                // parts of a tile's keys
  float* o_ws;                    // [tile][kv head][split][row][128] and, behind them,
  float2* ml_ws;                  // (max, sum) of each such row; unused with one split
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


// ---- row tiles -----------------------------------------------------------
// The rows of a (sequence, KV head) are its (token, head of the group) pairs,
// token-major: row r is token r / group, head r % group.  A tile is kRows of them.

struct Tile {
  uint32_t b, row0;  // sequence, first row
};
// Tile number `tile` of all sequences' tiles, the last tile of a sequence first
// (causal: it has the most keys).  By a converged warp; b = batch: none.
template <int kRows>
__device__ __forceinline__ Tile find_tile(const ExtendArgs& a, uint32_t tile) {
  const uint32_t lane = threadIdx.x & 31;
  if (!a.q_start) {
    const uint32_t b = tile / a.tiles_per_seq;
    return {b, (a.tiles_per_seq - 1 - (tile - b * a.tiles_per_seq)) * kRows};
  }
  uint32_t before = 0;
  for (uint32_t base = 0; base < a.map.batch; base += 32) {
    const uint32_t b = base + lane;
    const uint32_t mine = b < a.map.batch ? (sequence(a, b).n * a.group.d + kRows - 1) / kRows : 0;
    uint32_t incl = mine;
#pragma unroll
    for (int sh = 1; sh < 32; sh <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, incl, sh);
      if (lane >= static_cast<uint32_t>(sh)) incl += v;
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, tile < before + incl);
    if (hit) {
      const int l = __ffs(hit) - 1;
      const uint32_t end = before + __shfl_sync(0xffffffffu, incl, l);
      return {base + l, (end - 1 - tile) * kRows};
    }
    before += __shfl_sync(0xffffffffu, incl, 31);
  }
  return {a.map.batch, 0};
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t f16x2_rn(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// What a row's scores are made of: x = s * mult in the log2 domain; capped,
// x = c log2(e) tanh(s * in), tanh(y) = 1 - 2 / (1 + 2^(2 log2(e) y)) (absolute
// error some 2^-22, which `cap` scales; the hardware tanh's 2^-11 would show).
struct RowScore {
  float mult;   // softmax_scale * g_K * log2(e) / the query's scale
  float slope;  // slopes[h] * log2(e)
};

// ---- many rows: tensor cores of the fifth generation ----------------------
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
constexpr int kTileRows = 256;
constexpr int kBlock = 128;  // keys per block
constexpr int kTileThreads = 20 * 32;
constexpr int kDequantWarp = 8, kMmaWarp = 16;
constexpr uint32_t kOperand = 32768;  // bytes of a 128 x 128 f16 operand
constexpr uint32_t kOffK = 2 * kOperand, kOffV = 4 * kOperand;
constexpr uint32_t kTileSmem = 6 * kOperand + 1024;  // and alignment

// f16 operands, fp32 accumulator, 128 x 64 (QK^T) and 128 x 128; bit 16: B is
// stored with N contiguous.
constexpr uint32_t kIdescQK = (1u << 4) | (8u << 17) | (8u << 24);
constexpr uint32_t kIdescPV = (1u << 4) | (1u << 16) | (16u << 17) | (8u << 24);
constexpr uint32_t kIdescPVFull = kIdescPV | (1u << 7) | (1u << 10);  // bf16 operands
// 128-byte-swizzled operand: rows of 128 bytes, 8-row groups 1024 bytes apart
// (sbo), the second 64 columns kOperand / 2 further (lbo, used with N contiguous).
// The low word; the high word is the same for all of them.
__device__ __forceinline__ uint32_t operand_desc(uint32_t saddr) {
  return ((saddr & 0x3FFFFu) >> 4) | ((kOperand / 2 >> 4) << 16);
}
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
// Byte of 16-byte chunk c (of 16) of row r in such an operand.
__device__ __forceinline__ uint32_t operand_chunk(uint32_t r, uint32_t c) {
  return (c >> 3) * (kOperand / 2) + r * 128 + (((c ^ r) & 7) << 4);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n .reg .pred p;\n .reg .b64 da, db;\n setp.ne.b32 p, %4, 0;\n mov.b64 da, {%1, %5};\n"
               " mov.b64 db, {%2, %5};\n tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n}" ::"r"(d),
               "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"(kDescHigh)
               : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile("{\n .reg .pred p;\n .reg .b64 db;\n setp.ne.b32 p, %4, 0;\n mov.b64 db, {%2, %5};\n"
               " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n}" ::"r"(d),
               "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"(kDescHigh)
               : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
      "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
        "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]),
        "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]),
        "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* u) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
      "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15])
      : "memory");
}
// Two fp32 lanes at once: (x, y) = (x, y) * m + b, and (x, y) += (u, v).
__device__ __forceinline__ uint64_t both(float v) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %1};" : "=l"(d) : "f"(v));
  return d;
}
__device__ __forceinline__ void fma2(float& x, float& y, uint64_t m, uint64_t b) {
  asm("{\n .reg .b64 v;\n mov.b64 v, {%0, %1};\n fma.rn.f32x2 v, v, %2, %3;\n mov.b64 {%0, %1}, v;\n}"
      : "+f"(x), "+f"(y)
      : "l"(m), "l"(b));
}
__device__ __forceinline__ void add2(float& x, float& y, float u, float v) {
  asm("{\n .reg .b64 a, b;\n mov.b64 a, {%0, %1};\n mov.b64 b, {%2, %3};\n add.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a;\n}"
      : "+f"(x), "+f"(y)
      : "f"(u), "f"(v));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ float warp_max(float v) {
  float d;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(d) : "f"(v));
  return d;
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
// Whether any of the barrier's 128 threads says so; also their barrier.
__device__ __forceinline__ bool any_of_128(bool mine) {
  uint32_t any;
  tc_fence_before();
  asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, %2, 128, p;\n selp.u32 %0, 1, 0, q;\n}"
               : "=r"(any)
               : "r"(static_cast<uint32_t>(mine)), "n"(1)
               : "memory");
  tc_fence_after();
  return any != 0;
}

// mbar_wait_bounded, the flag that another role gave up looked at in every turn.
__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity, volatile int* abort) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = globaltimer_ns();
  while (!mbar_try_wait(bar, parity))
    if (*abort || globaltimer_ns() - t0 > kWaitLimitNs) return false;
  return true;
}

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

// 32 scores of a row, capped and biased, in the log2 domain.
__device__ __forceinline__ void score32(float* s, const RowScore& rs, const ExtendArgs& a, int p_minus_t0) {
  if (a.cap > 0.0f) {
    const float in = rs.mult * (2.0f / a.cap), out = a.cap * kLog2e;  // 2 log2(e) s / c
#pragma unroll
    for (int i = 0; i < 32; ++i) s[i] = fmaf(-2.0f * out, rcp(1.0f + ex2(s[i] * in)), out);
  } else {
#pragma unroll
    for (int i = 0; i < 32; ++i) s[i] *= rs.mult;
  }
  if (a.slopes) {
#pragma unroll
    for (int i = 0; i < 32; ++i) s[i] = fmaf(-rs.slope, fabsf(static_cast<float>(p_minus_t0 - i)), s[i]);
  }
}

// The eight elements of a code word times their block scale (kv_scales16) as four
// f16x2.  E2M1: channels (0,1) (2,3) (4,5) (6,7).  E1M2: (0,4) (1,5) (2,6) (3,7): a
// nibble is decoded where it stands, those in bits 4-7 as 16 times their value,
// for which the scale is divided (exact).  Q is laid out in the same order, and
// O comes in V's.
template <bool kE1M2>
__device__ __forceinline__ void scaled8(uint32_t w, uint32_t scale, uint32_t e[4]) {
  if (kE1M2) {
    const uint32_t t = w >> 8, scale16 = mul_f16x2(scale, 0x2C002C00u);
    e[0] = mul_f16x2(sub_f16x2((w & 0x000F000Fu) ^ 0x64086408u, 0x64086408u), scale);
    e[1] = mul_f16x2(sub_f16x2((w & 0x00F000F0u) ^ 0x64806480u, 0x64806480u), scale16);
    e[2] = mul_f16x2(sub_f16x2((t & 0x000F000Fu) ^ 0x64086408u, 0x64086408u), scale);
    e[3] = mul_f16x2(sub_f16x2((t & 0x00F000F0u) ^ 0x64806480u, 0x64806480u), scale16);
  } else {
    elements8<false>(w, e);
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = mul_f16x2(e[i], scale);
  }
}
// Place of channel c, and channel at place c, in that order.
template <bool kE1M2>
__device__ __forceinline__ constexpr int place_of(int c) { return kE1M2 ? (c & ~7) | (c & 3) << 1 | (c >> 2 & 1) : c; }
template <bool kE1M2>
__device__ __forceinline__ constexpr int channel_of(int c) { return kE1M2 ? (c & ~7) | (c & 1) << 2 | (c >> 1 & 3) : c; }
// Eight channels of Q, scaled, as f16 in that order.
template <bool kE1M2>
__device__ __forceinline__ uint4 q_chunk(const float x[8], float down) {
  uint32_t f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = f16x2_rn(x[channel_of<kE1M2>(2 * i)] * down, x[channel_of<kE1M2>(2 * i + 1)] * down);
  return make_uint4(f[0], f[1], f[2], f[3]);
}

// Two f16 values of at most 7 significant bits, at least 2^-14 or zero -> bf16,
// exact: the 5-bit exponent moves into the 8-bit field, 2^112 makes up for the bias.
__device__ __forceinline__ uint32_t bf16x2_of_f16x2(uint32_t h) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(((h >> 3) & 0x0FFF0FFFu) | (h & 0x80008000u)), "r"(0x77807780u));
  return d;
}

// kFull: weights as two bf16 terms (16 significant bits at fp32's range) and V in
// bf16, a second PV product per block.  In f16 a weight below 2^-28 of the row's
// largest is lost, which shows only where all heavier keys hold a zero in a
// channel: among few keys.
template <bool kE1M2, bool kMods, bool kFull>
__global__ void __launch_bounds__(kTileThreads, 1) extend_tile_kernel(const ExtendArgs a) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ TileShared sh;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.k_full[i], 4);
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
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
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
        // 2^-e with 2^e > amax, both within the normal fp32 range.
        const int e = max(-125, min(static_cast<int>(top >> 7) - 126, 126));
        const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
        if (c == 0) sh.mult[lr] = a.scale * kLog2e * __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
        float x[8];
        unpack_bf16x8(w[i], x);
        const uint4 f = q_chunk<kE1M2>(x, down);
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
    rs.mult = sh.mult[live ? local : 0];
    rs.slope = kMods && a.slopes && live ? __ldg(a.slopes + head) * kLog2e : 0.0f;
    // Keys that every row of the warp sees need no mask.
    const int all_lo = __reduce_max_sync(0xffffffffu, live ? vis.x : 0);
    const int all_hi = __reduce_min_sync(0xffffffffu, live ? vis.y : 0x7fffffff);
    const float to_log2 = kMods ? 1.0f : rs.mult;
    const uint64_t to_log2x2 = both(to_log2);
    float m = -INFINITY, l0 = 0.0f, l1 = 0.0f;
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
      if (kMods) {
#pragma unroll
        for (int k = 0; k < 64; k += 32) score32(s + k, rs, a, p - t0 - k);
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
      const bool up = top > m + kRescaleLog2 || (m == -INFINITY && top > -INFINITY);
      if (__any_sync(0xffffffffu, up)) {
        const float shrink = up ? ex2(m - top) : 1.0f;  // 0 where there was none
        if (up) m = top;
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
      const uint64_t minus = both((m == -INFINITY ? 0.0f : -m) + kWeightLog2);
      // The weights, over the scores they came from.
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t w[16], rest[kFull ? 16 : 1];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          float x = s[32 * c + 2 * k], y = s[32 * c + 2 * k + 1];
          fma2(x, y, to_log2x2, minus);
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
    const float l = l0 + l1;
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
      const float f = a.splits > 1 ? 1.0f : sum > 0.0f ? a.gv / sum : 0.0f;
      const uint64_t rec0 = ((static_cast<uint64_t>(tile_id) * a.map.hkv + kvh) * a.splits + split) * kTileRows;
      if (a.splits > 1 && live) a.ml_ws[rec0 + local] = make_float2(big, sum);
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
          if (row0 + row < rows)
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
          reinterpret_cast<uint4*>(a.out + (static_cast<uint64_t>(seq.first + tk) * a.hq + kvh * group + rr - tk * group) * kD)
              [lane & 15] = lds128(at(row, lane & 15));
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

// ---- few rows: keys on the M side -----------------------------------------
// HBM-bound work: every byte of K and V is needed once for up to 32 rows.  A CTA
// takes kC rows and a range of keys, and multiplies the other way round, so that
// the rows are the short side of every product (kN = 16 or 32 of the tensor core):
//   S^T[128 keys, kN] = K Q^T: K dequantized into TMEM (lane = key), Q in shared memory
//   O^T[128 channels, kN] += V^T P^T: V dequantized into shared memory, P too
//   warps 0-3   softmax (thread = key; in the end, channel of O^T)
//   warps 4-7   K (thread = key)
//   warps 8-11  V
//   warp 12, 13 issue the PV and the QK^T; 14, 15 complete the warpgroup
// Two CTAs share an SM.  What a softmax thread does per block is kept short: the
// four roles' code does not fit the instruction caches that are near the
// schedulers, and a role's turn goes by its instructions more than by its work.
// (By mma.sync in registers the tensor pipe's rate for that form is the bound: 64
// ragged sequences of up to 16384 tokens 174 us, 32 x 4 new tokens on 4001 148.)
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

struct RowInfo {
  float slope;
  int pos, lo, hi;
  uint32_t out;  // (token, head) row of the output; rows past the tile's: none
};
template <int kC>
struct RowsShared {
  uint64_t s_full[2], s_free[2], k_full[2], k_free[2], v_full[2], v_free[2], p_full[2], q_full, drain, drain_qk;
  uint32_t tmem;
  Tile tile;
  Seq seq;
  int lo, hi, all_lo, all_hi, rows;
  alignas(16) float mult[kC];   // score -> log2 domain
  alignas(16) float minus[kC];  // 4 - the row's maximum: x = score + minus is a weight's exponent
  RowInfo row[kC];
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

template <int kC, bool kE1M2, bool kFull>
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
      mbar_init(&sh.s_free[i], 4);
      mbar_init(&sh.k_full[i], 4);
      mbar_init(&sh.k_free[i], 1);
      mbar_init(&sh.v_full[i], 4);
      mbar_init(&sh.v_free[i], 1);
      mbar_init(&sh.p_full[i], 4);
    }
    mbar_init(&sh.drain, 1);
    mbar_init(&sh.drain_qk, 1);
    mbar_init(&sh.q_full, 4);
    sh.abort = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    tmem_alloc(&sh.tmem, kRowsTmem);
    tmem_relinquish();  // the SM's other CTA allocates too
  }
  griddep_wait_and_release();
  const uint32_t split = blockIdx.x % a.splits, rest = blockIdx.x / a.splits;
  const uint32_t tile_id = rest / a.map.hkv, kvh = rest - tile_id * a.map.hkv, group = a.group.d;
  if (warp == 0) {
    const Tile tl = find_tile<kC>(a, tile_id);
    const bool any = tl.b < a.map.batch;  // else more CTAs than tiles
    Seq sq = {0, 0, 0};
    if (any) sq = sequence(a, tl.b);
    // A row a lane: what it sees, and where its output goes.
    const uint32_t rows = any ? min(sq.n * group - tl.row0, static_cast<uint32_t>(kC)) : 0;
    const bool live = lane < static_cast<int>(rows);
    const uint32_t r = tl.row0 + (live ? lane : 0), tok = a.group.div(r), h = kvh * group + (r - tok * group);
    RowInfo row;
    row.pos = sq.len - static_cast<int>(sq.n) + static_cast<int>(tok);
    int2 vis = make_int2(0, 0);
    if (live && row.pos >= 0)
      vis = visible(a, row.pos, sq.len, a.prefix_lens ? __ldg(a.prefix_lens + tl.b) : 0,
                    a.doc_start ? __ldg(a.doc_start + sq.first + tok) : 0);
    if (vis.x >= vis.y) vis = make_int2(0x7fffffff, 0);
    row.lo = vis.x;
    row.hi = vis.y;
    row.slope = a.slopes && live ? __ldg(a.slopes + h) * kLog2e : 0.0f;
    row.out = live ? (sq.first + tok) * a.hq + h : 0xffffffffu;
    if (lane < kC) sh.row[lane] = row;
    const int lo = __reduce_min_sync(0xffffffffu, vis.x), hi = __reduce_max_sync(0xffffffffu, vis.y);
    const int all_lo = __reduce_max_sync(0xffffffffu, live ? vis.x : 0);
    const int all_hi = __reduce_min_sync(0xffffffffu, live ? vis.y : 0x7fffffff);
    if (lane == 0) {
      sh.tile = tl;
      sh.seq = sq;
      sh.lo = hi > lo ? lo : 0;
      sh.hi = hi > lo ? hi : 0;
      sh.rows = static_cast<int>(rows);
      sh.all_lo = all_lo;
      sh.all_hi = all_hi;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = sh.tmem;
  const Tile tile = sh.tile;
  const bool none = tile.b >= a.map.batch;
  // This CTA's blocks of keys, counted from the tile's first key.
  const int end = sh.hi, total = (end - sh.lo + kBlock - 1) / kBlock;
  const int per = (total + static_cast<int>(a.splits) - 1) / static_cast<int>(a.splits);
  const int j0 = min(static_cast<int>(split) * per, total), nblk = min(per, total - j0);
  const int t_base = sh.lo + j0 * kBlock;

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

  // 104, 64, 64 and 24 registers a thread: the 512 x 64 that the CTA starts with.
  if (warp < 4) {
    // ------------------------------------------------------------- softmax ---
    asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
    // Q rows as f16, scaled by a power of two (exact) to below 1: 16 lanes a row.
    uint4 w[kN / 8];
#pragma unroll
    for (int i = 0; i < kN / 8; ++i) {
      const uint32_t lr = i * 8 + warp * 2 + (lane >> 4), out = lr < kC ? sh.row[lr].out : 0xffffffffu;
      w[i] = make_uint4(0, 0, 0, 0);
      if (out != 0xffffffffu) {
        const uint32_t tk = out / a.hq;
        w[i] = __ldg(reinterpret_cast<const uint4*>(a.q + static_cast<int64_t>(tk) * a.ld_q + (out - tk * a.hq) * kD) + (lane & 15));
      }
    }
#pragma unroll
    for (int i = 0; i < kN / 8; ++i) {
      const uint32_t lr = i * 8 + warp * 2 + (lane >> 4), c = lane & 15;
      uint32_t top = amax_bits_bf16x8(w[i]);
#pragma unroll
      for (int s = 1; s < 16; s <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
      const int e = max(-125, min(static_cast<int>(top >> 7) - 126, 126));
      const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
      if (c == 0 && lr < kC) {
        // No maximum yet: any score exceeds it.  (A row past the tile's has scores of 0.)
        const bool live = sh.row[lr].out != 0xffffffffu;
        sh.mult[lr] = live ? a.scale * kLog2e * __uint_as_float(static_cast<uint32_t>(127 + e) << 23) : 0.0f;
        sh.minus[lr] = live ? 1e30f : 0.0f;
      }
      float x[8];
      unpack_bf16x8(w[i], x);
      const uint4 f = q_chunk<kE1M2>(x, down);
      sts128(smem + C::kOffQ + (c >> 3) * (kN * 128) + lr * 128 + (((c ^ lr) & 7) << 4), f.x, f.y, f.z, f.w);
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.q_full);
    any_of_128(false);  // the multipliers of all rows
    const uint32_t lanes = static_cast<uint32_t>(warp * 32) << 16;
    const int key = warp * 32 + lane;
    const bool mods = a.cap > 0.0f || a.slopes;
    float l[kC];
#pragma unroll
    for (int n = 0; n < kC; ++n) l[n] = 0.0f;
    bool ok = true;
    for (int j = 0; j < nblk; ++j) {
      const int b = j & 1, t0 = t_base + (nblk - 1 - j) * kBlock, tk = t0 + key;
      const uint32_t p_at = smem + C::kOffP + b * 2 * C::kB + key * 16;
      ok = wait(&sh.s_full[b], j >> 1);
      ok = wait(&sh.v_full[b], j >> 1) && ok;  // and so P of block j - 2 is used up
      const bool there = (sh.present[j & 3][warp] >> lane) & 1u;
      const bool open = t0 >= sh.all_lo && t0 + kBlock <= sh.all_hi && __all_sync(0xffffffffu, there);
      float s[kC];
      tmem_ld_cols<kC>(tmem + lanes + kColS + b * 32, s);
      tmem_wait_ld();
#pragma unroll
      for (int n = 0; n < kC; n += 4) {
        const float4 f = *reinterpret_cast<const float4*>(&sh.mult[n]);
        s[n] *= f.x;
        s[n + 1] *= f.y;
        s[n + 2] *= f.z;
        s[n + 3] *= f.w;
      }
      if (mods) {
        const float cap = a.cap * kLog2e, in = 2.0f / a.cap;  // 2 log2(e) s / c
#pragma unroll
        for (int n = 0; n < kC; ++n) {
          if (a.cap > 0.0f) s[n] = fmaf(-2.0f * cap, rcp(1.0f + ex2(s[n] * in)), cap);
          s[n] = fmaf(-sh.row[n].slope, fabsf(static_cast<float>(sh.row[n].pos - tk)), s[n]);
        }
      }
      if (!open) {
#pragma unroll
        for (int n = 0; n < kC; ++n)
          if (!there || tk < sh.row[n].lo || tk >= sh.row[n].hi) s[n] = -INFINITY;
      }
      // Maxima move only where a weight would be 2^11 times its row's maximum.
      for (;;) {
        float most = -INFINITY;
#pragma unroll
        for (int n = 0; n < kC; n += 4) {
          const float4 f = *reinterpret_cast<const float4*>(&sh.minus[n]);
          most = max3(max3(s[n] + f.x, s[n + 1] + f.y, most), s[n + 2] + f.z, s[n + 3] + f.w);
        }
        if (!any_of_128(most > kWeightLog2 + kRescaleLog2 || !ok)) break;
        // Each row's largest score in the block, by warp, then of all four.
#pragma unroll
        for (int n = 0; n < kC; ++n) {
          const float v = warp_max(s[n]);
          if (lane == 0) sh.top[warp][n] = v;
        }
        if (any_of_128(!ok)) {
          ok = false;
          break;  // a wait ran out: the four warps leave together
        }
        const auto top_of = [&](int n) { return max3(max3(sh.top[0][n], sh.top[1][n], sh.top[2][n]), sh.top[3][n], -INFINITY); };
        const auto shrink = [&](int n) {
          const float x = top_of(n) + sh.minus[n];
          return x > kWeightLog2 + kRescaleLog2 ? ex2(kWeightLog2 - x) : 1.0f;
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
        any_of_128(false);  // every warp has read the old maxima
        if (warp == 0 && lane < kC && shrink(lane) != 1.0f) sh.minus[lane] = kWeightLog2 - top_of(lane);
        any_of_128(false);
      }
      if (!ok) break;
#pragma unroll
      for (int n = 0; n < kC; n += 4) {
        const float4 f = *reinterpret_cast<const float4*>(&sh.minus[n]);
        s[n] = ex2(s[n] + f.x);
        s[n + 1] = ex2(s[n + 1] + f.y);
        s[n + 2] = ex2(s[n + 2] + f.z);
        s[n + 3] = ex2(s[n + 3] + f.w);
      }
#pragma unroll
      for (int n = 0; n < kC; n += 8) {
        if (kFull) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t xb = __float_as_uint(s[n + 2 * k]), yb = __float_as_uint(s[n + 2 * k + 1]);
            hi[k] = __byte_perm(xb, yb, 0x7632);
            lo[k] = bf16x2_rn(s[n + 2 * k] - __uint_as_float(xb & 0xFFFF0000u), s[n + 2 * k + 1] - __uint_as_float(yb & 0xFFFF0000u));
          }
          sts128(p_at + n * 256, hi[0], hi[1], hi[2], hi[3]);
          sts128(p_at + n * 256 + C::kB, lo[0], lo[1], lo[2], lo[3]);
        } else {
          sts128(p_at + n * 256, f16x2_rn(s[n], s[n + 1]), f16x2_rn(s[n + 2], s[n + 3]), f16x2_rn(s[n + 4], s[n + 5]),
                 f16x2_rn(s[n + 6], s[n + 7]));
        }
      }
      fence_proxy_async_smem();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sh.p_full[b]);
        mbar_arrive(&sh.s_free[b]);
      }
#pragma unroll
      for (int n = 0; n < kC; ++n) l[n] += s[n];
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
    const uint64_t rec0 = ((static_cast<uint64_t>(tile_id) * a.map.hkv + kvh) * a.splits + split) * kC;
    const int channel = channel_of<kE1M2>(key);
    if (done && !none)
#pragma unroll
      for (int n = 0; n < kC; ++n) {
        if (n >= sh.rows) break;
        const float sum = nblk > 0 ? (sh.sum[0][n] + sh.sum[1][n]) + (sh.sum[2][n] + sh.sum[3][n]) : 0.0f;
        const float v = sum > 0.0f ? o[n] : 0.0f;
        if (a.splits > 1) {
          if (key == 0) a.ml_ws[rec0 + n] = make_float2(sum > 0.0f ? kWeightLog2 - sh.minus[n] : -INFINITY, sum);
          a.o_ws[(rec0 + n) * kD + channel] = v;
        } else {
          const uint32_t bits = bf16x2_rn(sum > 0.0f ? v * (a.gv / sum) : 0.0f, 0.0f);
          a.out[static_cast<uint64_t>(sh.row[n].out) * kD + channel] = static_cast<uint16_t>(bits);
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
    if (warp < 14) {
      const bool leader = elect_one();
      const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
      for (int j = 0; j < nblk; ++j) {
        const int b = j & 1;
        if (warp == 12) {
          if (!wait(&sh.p_full[b], j >> 1)) break;  // V is there too: the softmax has waited for it
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
        } else {
          if ((j == 0 && !wait(&sh.q_full, 0)) || !wait(&sh.k_full[b], j >> 1) || (j >= 2 && !wait(&sh.s_free[b], (j >> 1) ^ 1))) break;
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
        }
        __syncwarp();
      }
      // Nothing that was issued, MMA or arrival, outlives the CTA.
      uint64_t* drain = warp == 12 ? &sh.drain : &sh.drain_qk;
      if (leader) tc_commit(drain);
      mbar_wait_bounded(drain, 0, nullptr, kDrainLimitNs);
      __syncwarp();
    }
  }
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kRowsTmem);
  }
}

// Joins the parts of a tile's rows in split order: one warp a row, four channels
// a lane, eight parts in flight.  Rows of a tile are shared out over gridDim.z
// CTAs.
template <int kRows>
__global__ void __launch_bounds__(256) extend_combine_kernel(const ExtendArgs a) {
  griddep_wait_and_release();
  const uint32_t lane = threadIdx.x & 31;
  const Tile t = find_tile<kRows>(a, blockIdx.x);
  if (t.b >= a.map.batch) return;
  const Seq seq = sequence(a, t.b);
  const uint32_t rows = min(seq.n * a.group.d - t.row0, static_cast<uint32_t>(kRows)), kvh = blockIdx.y;
  for (uint32_t local = blockIdx.z * 8 + (threadIdx.x >> 5); local < rows; local += gridDim.z * 8) {
    const uint64_t rec = (static_cast<uint64_t>(blockIdx.x) * a.map.hkv + kvh) * a.splits * kRows + local;
    const float2* ml = a.ml_ws + rec;
    const float4* part = reinterpret_cast<const float4*>(a.o_ws + rec * kD) + lane;
    float2 mine = lane < a.splits ? ml[static_cast<uint64_t>(lane) * kRows] : make_float2(-INFINITY, 0.0f);
    float big = mine.x;
    for (uint32_t s = lane + 32; s < a.splits; s += 32) big = fmaxf(big, ml[static_cast<uint64_t>(s) * kRows].x);
#pragma unroll
    for (int sh = 16; sh; sh >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, sh));
    float sum = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (uint32_t s0 = 0; s0 < a.splits; s0 += 32) {
      if (s0) mine = s0 + lane < a.splits ? ml[static_cast<uint64_t>(s0 + lane) * kRows] : make_float2(-INFINITY, 0.0f);
      const float w = mine.x == -INFINITY ? 0.0f : ex2(mine.x - big);  // an empty part has no O
      for (uint32_t s = s0; s < min(s0 + 32, a.splits); s += 8) {
        float4 v[8];
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          f[k] = __shfl_sync(0xffffffffu, w, (s + k) & 31);
          if (s + k >= a.splits) f[k] = 0.0f;
          v[k] = f[k] != 0.0f ? part[static_cast<uint64_t>(s + k) * kRows * (kD / 4)] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          sum = fmaf(f[k], __shfl_sync(0xffffffffu, mine.y, (s + k) & 31), sum);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          o.x = fmaf(f[k], v[k].x, o.x);
          o.y = fmaf(f[k], v[k].y, o.y);
          o.z = fmaf(f[k], v[k].z, o.z);
          o.w = fmaf(f[k], v[k].w, o.w);
        }
      }
    }
    const float f = sum > 0.0f ? a.gv / sum : 0.0f;
    const uint32_t r = t.row0 + local, tok = a.group.div(r), head = kvh * a.group.d + (r - tok * a.group.d);
    reinterpret_cast<uint2*>(a.out + (static_cast<uint64_t>(seq.first + tok) * a.hq + head) * kD)[lane] =
        make_uint2(bf16x2_rn(o.x * f, o.y * f), bf16x2_rn(o.z * f, o.w * f));
  }
}

// ---- host ----------------------------------------------------------------

struct Plan {
  int rows;  // of a tile: kTileRows, or 8, 16, 24, 32 by the rows kernel
  int64_t tiles, tiles_per_seq, splits;
  bool full;  // weights in two terms (kFull)
};

// Contexts of up to this many keys take kFull.
constexpr int64_t kFullContext = 512;

// Which kernel, the tiles (at most), and the parts that each tile's keys are cut into.
Plan plan_for(int64_t batch, int64_t n_tokens, int64_t group, int64_t hkv, int64_t context, bool uniform) {
  Plan p;
  const int64_t sms = sm_count(), blocks = (context + kBlock - 1) / kBlock;
  const int64_t rows = (n_tokens * group + batch - 1) / batch;  // of a sequence and KV head, on average
  p.full = context <= kFullContext;
  p.rows = rows <= 32 ? static_cast<int>((rows + 7) / 8 * 8) : kTileRows;
  p.tiles_per_seq = (n_tokens / batch * group + p.rows - 1) / p.rows;
  const int64_t ragged = n_tokens * group / p.rows + (batch < n_tokens ? batch : n_tokens);
  p.tiles = uniform ? batch * p.tiles_per_seq : ragged;
  const int64_t items = p.tiles * hkv;
  p.splits = 1;
  if (p.rows != kTileRows) {
    // Enough CTAs for six rounds on what is resident, so that sequences of
    // different lengths even out, in parts of 512 keys or more; failing that,
    // one round in parts of a stage or more.
    const int64_t resident = sms * 2;
    const int64_t even = (6 * resident + items - 1) / items, long_parts = (blocks + 3) / 4;
    const int64_t fill = (resident + items - 1) / items;
    p.splits = even < long_parts ? even : long_parts;
    if (fill > p.splits) p.splits = fill;
    if (p.splits > blocks) p.splits = blocks;
    return p;
  }
  // As many as make the last wave of CTAs full, against what a part costs by
  // itself (its prologue; with several, its record written and read), in blocks
  // of 128 keys.
  double best = 0.0;
  for (int64_t s = 1; s == 1 || (s <= blocks && s <= 64 && items * s <= 4 * sms); ++s) {
    const double cost = static_cast<double>((items * s + sms - 1) / sms) * (static_cast<double>((blocks + s - 1) / s) + (s > 1 ? 6.0 : 2.0));
    if (s == 1 || cost < best) {
      best = cost;
      p.splits = s;
    }
  }
  return p;
}

size_t workspace_for(const Plan& p, int64_t hkv) {
  return p.splits > 1 ? static_cast<size_t>(p.tiles) * hkv * p.splits * p.rows * (kD + 2) * sizeof(float) : 0;
}

using Kernel = void (*)(const ExtendArgs);
uint32_t smem_for(const Plan& p) {
  return p.rows == kTileRows ? kTileSmem : p.rows <= 16 ? RowsConfig<16>::kBytes : RowsConfig<32>::kBytes;
}
template <bool kE1M2, bool kFull>
Kernel kernel_for(const Plan& p, bool mods) {
  switch (p.rows) {
    case 8: return extend_rows_kernel<8, kE1M2, kFull>;
    case 16: return extend_rows_kernel<16, kE1M2, kFull>;
    case 24: return extend_rows_kernel<24, kE1M2, kFull>;
    case 32: return extend_rows_kernel<32, kE1M2, kFull>;
  }
  return mods ? extend_tile_kernel<kE1M2, true, kFull> : extend_tile_kernel<kE1M2, false, kFull>;
}
Kernel combine_for(const Plan& p) {
  switch (p.rows) {
    case 8: return extend_combine_kernel<8>;
    case 16: return extend_combine_kernel<16>;
    case 24: return extend_combine_kernel<24>;
    case 32: return extend_combine_kernel<32>;
  }
  return extend_combine_kernel<kTileRows>;
}

}  // namespace
}  // namespace nvfp4

using namespace nvfp4;

NVFP4_API size_t extend_attention_nvfp4_workspace_size(int32_t batch, int64_t n_tokens, int32_t num_q_heads,
                                                       int32_t num_kv_heads, int64_t context) {
  if (batch <= 0 || n_tokens <= 0 || num_q_heads <= 0 || num_kv_heads <= 0 || num_q_heads % num_kv_heads ||
      context <= 0 || n_tokens >= (1ll << 31) || context >= (1ll << 31))
    return 0;
  // Both forms of q_start, so that one buffer serves either.
  const int64_t group = num_q_heads / num_kv_heads;
  const size_t ragged = workspace_for(plan_for(batch, n_tokens, group, num_kv_heads, context, false), num_kv_heads);
  const size_t uniform =
      n_tokens % batch ? 0 : workspace_for(plan_for(batch, n_tokens, group, num_kv_heads, context, true), num_kv_heads);
  return ragged > uniform ? ragged : uniform;
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
  if (n_tokens < 0 || num_q_heads <= 0 || num_q_heads > 65535 || n_tokens >= (1ll << 31) / num_q_heads ||
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
  const Plan p = plan_for(a.map.batch, n_tokens, a.group.d, a.map.hkv, a.map.context, !q_start);
  const int64_t grid = p.tiles * a.map.hkv * p.splits;
  if (grid >= (1ll << 31)) return NVFP4_ERR_SHAPE;
  a.tiles = static_cast<uint32_t>(p.tiles);
  a.tiles_per_seq = static_cast<uint32_t>(p.tiles_per_seq);
  a.splits = static_cast<uint32_t>(p.splits);
  a.o_ws = static_cast<float*>(workspace);
  a.ml_ws = reinterpret_cast<float2*>(a.o_ws + static_cast<size_t>(grid) * p.rows * kD);
  const bool mods = options->logit_cap > 0.0f || options->slopes, e1m2 = cache->kv_format == NVFP4_KV_E1M2;
  const Kernel kernel = e1m2 ? (p.full ? kernel_for<true, true>(p, mods) : kernel_for<true, false>(p, mods))
                             : (p.full ? kernel_for<false, true>(p, mods) : kernel_for<false, false>(p, mods));
  const bool by_tiles = p.rows == kTileRows;
  const uint32_t smem = smem_for(p);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // Raising the limit is idempotent.
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess ||
      launch_pdl(kernel, dim3(static_cast<uint32_t>(grid)), dim3(by_tiles ? kTileThreads : kRowsThreads), smem, s, a) != cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  if (p.splits > 1) {
    if (launch_pdl(combine_for(p), dim3(a.tiles, a.map.hkv, by_tiles ? 8 : (p.rows + 7) / 8), dim3(256), 0, s, a) != cudaSuccess)
      return NVFP4_ERR_CUDA;
    count_launches(1);
  }
  return launch_status();
}
