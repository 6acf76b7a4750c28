// Attention of new tokens (one, a few, a chunk, a whole prompt) over the 4-bit
// cache that already holds them, contiguous or paged: scores optionally capped
// and biased by distance, keys limited by causality, window, prefix, document.
#include "kv_pages.cuh"

namespace nvfp4 {
namespace {

constexpr int kD = 128;
constexpr float kLog2e = 1.4426950408889634f;

constexpr float kRescaleLog2 = 8.0f;  // the running maximum moves only when a score exceeds it by 2^8
constexpr float kWeightLog2 = 7.0f;   // weights are kept as 2^7 w: at most 2^15 in f16, and fine steps below 1

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
//                   write P over it, rescale O where a maximum moved by over 2^8
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

// mbar_wait_bounded with a hint of how long the hardware may suspend the thread,
// so that waiting warps leave the issue slots to the others.
__device__ __forceinline__ bool wait_bar(uint64_t* bar, uint32_t parity, volatile int* abort) {
  const uint32_t addr = smem_u32(bar);
  const auto once = [&] {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred p;\n"
        " mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n"
        " selp.u32 %0, 1, 0, p;\n}"
        : "=r"(ok)
        : "r"(addr), "r"(parity), "r"(100000u)
        : "memory");
    return ok != 0;
  };
  if (once()) return true;
  const uint64_t t0 = globaltimer_ns();
  while (!once()) {
    if (*abort || globaltimer_ns() - t0 > kWaitLimitNs) return false;
  }
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

// Two f16 values of at most 7 significant bits, at least 2^-14 or zero -> bf16,
// exact: the 5-bit exponent moves into the 8-bit field, 2^112 makes up for the bias.
__device__ __forceinline__ uint32_t bf16x2_of_f16x2(uint32_t h) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(((h >> 3) & 0x0FFF0FFFu) | (h & 0x80008000u)), "r"(0x77807780u));
  return d;
}

// kFull: weights as two bf16 terms (16 significant bits at fp32's range) and V in
// bf16, a second PV product per block.  In f16 a weight below 2^-31 of the row's
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
        sts128(smem + (lr >> 7) * kOperand + operand_chunk(lr & 127, c), f16x2_rn(x[0] * down, x[1] * down),
               f16x2_rn(x[2] * down, x[3] * down), f16x2_rn(x[4] * down, x[5] * down), f16x2_rn(x[6] * down, x[7] * down));
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
      const int j = two ? v >> 1 : (v & ~1) + t, hf = v & 1, t0 = t_base + j * kBlock + 64 * hf;
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
          for (int k = 0; k < 4; ++k)
            sts128(at(lane, 4 * c + k), bf16x2_rn(o[8 * k], o[8 * k + 1]), bf16x2_rn(o[8 * k + 2], o[8 * k + 3]),
                   bf16x2_rn(o[8 * k + 4], o[8 * k + 5]), bf16x2_rn(o[8 * k + 6], o[8 * k + 7]));
          continue;
        }
        // A record in fp32: 128 bytes of each row at a time.
#pragma unroll
        for (int k = 0; k < 8; ++k)
          sts128(at(lane, k), __float_as_uint(o[4 * k]), __float_as_uint(o[4 * k + 1]), __float_as_uint(o[4 * k + 2]),
                 __float_as_uint(o[4 * k + 3]));
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
      const int t0 = t_base + block(q) * kBlock + w * 8 + sub;  // >= 0
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
          elements8<kE1M2>(words[k], e);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            e[x] = mul_f16x2(e[x], k < 2 ? g0 : g1);
            if (bf16) e[x] = bf16x2_of_f16x2(e[x]);
          }
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

// ---- few rows: registers --------------------------------------------------
// HBM-bound work: every byte of K and V is needed once for a handful of rows.  A
// CTA takes 8 kN rows and a range of keys.  Warp 0 streams the keys' codes and
// scales into a two-stage ring of 128 keys; four warps take two 16-key tiles of a
// stage each, dequantize in registers (exact in f16) and multiply with mma.sync
// m16n8k16: S^T[16 keys, 8 rows] = K Q^T, O^T[128, 8 rows] += V^T P^T, for each of
// the kN groups of rows.  (tcgen05 would take a 128-row operand for these few, and
// K and V through shared memory: 64 x 16384 ragged tokens 381 us by the tiles.)
//
// Lane roles (g = lane / 4, t = lane % 4), as the fragments have them:
//   K rows g and g + 8 of the tile, channels 32t..32t+31; V rows 2t, 2t+1, 2t+8,
//   2t+9, channels 16g..16g+15; Q row g of a group, channels 32t..32t+31.
// Row m of a 16-key tile is key (m & 1) * 4 + (m >> 1 & 3) + (m & 8), so that a V
// load covers four consecutive keys.
constexpr int kRowsWarps = 4;
constexpr int kRowsThreads = 32 * (1 + kRowsWarps);
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
// The eight elements of a code word as pairs.  E2M1: (0,1) (2,3) (4,5) (6,7).
// E1M2: (0,4) (1,5) (2,6) (3,7), the second and fourth pair times 16 (a nibble in
// bits 4-7 is decoded where it stands); their scales carry the 1/16.
template <bool kE1M2>
__device__ __forceinline__ void pairs8(uint32_t w, uint32_t e[4]) {
  if (kE1M2) {
    const uint32_t t = w >> 8;
    e[0] = sub_f16x2((w & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
    e[1] = sub_f16x2((w & 0x00F000F0u) ^ 0x64806480u, 0x64806480u);
    e[2] = sub_f16x2((t & 0x000F000Fu) ^ 0x64086408u, 0x64086408u);
    e[3] = sub_f16x2((t & 0x00F000F0u) ^ 0x64806480u, 0x64806480u);
  } else {
    elements8<false>(w, e);
  }
}

template <int kN>
struct RowsShared {
  uint64_t full[kRing], empty[kRing];
  uint32_t present[kRing][4];
  Tile tile;
  Seq seq;
  int lo, hi;
  float m[kRowsWarps][8 * kN], l[kRowsWarps][8 * kN];
  uint2 q[kN > 1 ? kN : 1][8][32];  // Q fragments by group, k-step, lane (one group: in registers)
  volatile int abort;
};
constexpr uint32_t kRowsSmem = kRing * kStageBytes + kRowsWarps * 8 * kMergeRow * 4;

template <int kN, bool kE1M2, bool kMods>
__global__ void __launch_bounds__(kRowsThreads, kN == 1 ? 4 : kN == 2 ? 3 : 2) extend_rows_kernel(const ExtendArgs a) {
  extern __shared__ __align__(128) uint8_t smem_raw[];
  __shared__ RowsShared<kN> sh;
  constexpr uint32_t kRows = 8 * kN;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(&sh.full[i], 1 + 32);  // the armed bytes, and each lane's own copies
      mbar_init(&sh.empty[i], kRowsWarps);
    }
    sh.abort = 0;
    fence_mbar_init();
  }
  griddep_wait_and_release();
  const uint32_t split = blockIdx.x % a.splits, rest = blockIdx.x / a.splits;
  const uint32_t tile_id = rest / a.map.hkv, kvh = rest - tile_id * a.map.hkv, group = a.group.d;
  if (warp == 0) {
    const Tile tl = find_tile<kRows>(a, tile_id);
    Seq sq = {0, 0, 0};
    if (tl.b < a.map.batch) sq = sequence(a, tl.b);
    // The keys that the tile's rows see.
    int lo = 0x7fffffff, hi = 0;
    const uint32_t rows = tl.b < a.map.batch ? min(sq.n * group - tl.row0, kRows) : 0;
    if (lane < static_cast<int>(rows)) {
      const uint32_t tok = a.group.div(tl.row0 + lane);
      const int p = sq.len - static_cast<int>(sq.n) + static_cast<int>(tok);
      const int2 vis = visible(a, p, sq.len, a.prefix_lens ? __ldg(a.prefix_lens + tl.b) : 0,
                               a.doc_start ? __ldg(a.doc_start + sq.first + tok) : 0);
      if (p >= 0 && vis.x < vis.y) {
        lo = vis.x;
        hi = vis.y;
      }
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) {
      sh.tile = tl;
      sh.seq = sq;
      sh.lo = hi > lo ? lo : 0;
      sh.hi = hi > lo ? hi : 0;
    }
  }
  __syncthreads();
  const Tile tile = sh.tile;
  if (tile.b >= a.map.batch) return;  // more CTAs than tiles
  const Seq seq = sh.seq;
  const uint32_t rows = min(seq.n * group - tile.row0, kRows);
  // This CTA's keys, in whole stages from the tile's first.
  const int stages = (sh.hi - sh.lo + kBlock - 1) / kBlock;
  const int per = (stages + static_cast<int>(a.splits) - 1) / static_cast<int>(a.splits);
  const int s0 = min(static_cast<int>(split) * per, stages), n = min(per, stages - s0);
  const int t_base = sh.lo + s0 * kBlock, t_end = min(sh.hi, t_base + n * kBlock);

  if (warp == 0) {
    // ------------------------------------------------------------ producer ---
    // Lane i has keys i, i + 32, i + 64, i + 96 of a stage.  Codes come by bulk
    // copies, one for each run of keys within a page; scales, 8 bytes a key, by
    // the lane's own copies.  A key that is not there (past the end, or its page
    // absent) gets scales of zero, whatever its codes' bytes.
    const int64_t head = static_cast<int64_t>(kvh) * a.map.size.d;
    for (int i = 0; i < n; ++i) {
      const int st = i & 1, t0 = t_base + i * kBlock;
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
    }
    // Copies in flight land before the CTA's memory goes to another (its
    // consumers have waited for them unless a wait ran out).
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (sh.abort)
      for (int i = max(n - 2, 0); i < n; ++i) mbar_wait_bounded(&sh.full[i & 1], (i >> 1) & 1, nullptr, kDrainLimitNs);
    return;
  }

  // ------------------------------------------------------------- consumers ---
  const int cw = warp - 1, g = lane >> 2, t = lane & 3;
  // Rows of the lane's columns in a group's tile of scores: 2t and 2t + 1.
  int2 vis[kN][2];
  float mult[kN][2], slope[kN][2];
  int pos[kN][2];
  int all_lo = 0, all_hi = 0x7fffffff;  // keys that every row sees
#pragma unroll
  for (int x = 0; x < kN; ++x)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const uint32_t lr = 8 * x + 2 * t + c;
      const bool live = lr < rows;
      const uint32_t r = tile.row0 + (live ? lr : 0), tok = a.group.div(r), h = kvh * group + (r - tok * group);
      const int p = seq.len - static_cast<int>(seq.n) + static_cast<int>(tok);
      vis[x][c] = visible(a, p, seq.len, a.prefix_lens ? __ldg(a.prefix_lens + tile.b) : 0,
                          a.doc_start ? __ldg(a.doc_start + seq.first + tok) : 0);
      if (!live || p < 0) vis[x][c] = make_int2(0x7fffffff, 0);
      if (live) {
        all_lo = max(all_lo, vis[x][c].x);
        all_hi = min(all_hi, vis[x][c].y);
      }
      pos[x][c] = p;
      slope[x][c] = kMods && a.slopes && live ? __ldg(a.slopes + h) * kLog2e : 0.0f;
    }
  all_lo = __reduce_max_sync(0xffffffffu, all_lo);
  all_hi = __reduce_min_sync(0xffffffffu, all_hi);
  // Queries: f16 after an exact scaling by a power of two to below 1.
  uint32_t qf[16];
#pragma unroll
  for (int x = 0; x < kN; ++x) {
    const uint32_t lr = 8 * x + g;
    const bool live = lr < rows;
    const uint32_t r = tile.row0 + (live ? lr : 0), tok = a.group.div(r);
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
    const int e = max(-125, min(static_cast<int>(top >> 7) - 126, 126));
    const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    const float up = a.scale * kLog2e * __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
    mult[x][0] = __shfl_sync(0xffffffffu, up, (2 * t) * 4);
    mult[x][1] = __shfl_sync(0xffffffffu, up, (2 * t + 1) * 4);
    float v[32];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack_bf16x8(w[i], v + 8 * i);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // Channels of k-step j, in the order of pairs8.
      const int c0 = kE1M2 ? 8 * (j >> 1) + 2 * (j & 1) : 4 * j;
      const int c1 = kE1M2 ? c0 + 4 : c0 + 1, c2 = kE1M2 ? c0 + 1 : c0 + 2, c3 = kE1M2 ? c0 + 5 : c0 + 3;
      const uint2 f = make_uint2(f16x2_rn(v[c0] * down, v[c1] * down), f16x2_rn(v[c2] * down, v[c3] * down));
      if (kN == 1) {
        qf[2 * j] = f.x;
        qf[2 * j + 1] = f.y;
      } else if (cw == 0) {
        sh.q[x][j][lane] = f;
      }
    }
  }
  if (kN > 1) asm volatile("bar.sync 1, %0;" ::"n"(32 * kRowsWarps) : "memory");

  float o[kN][8][4], m_run[kN][2], l_run[kN][2];
#pragma unroll
  for (int x = 0; x < kN; ++x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) o[x][i][0] = o[x][i][1] = o[x][i][2] = o[x][i][3] = 0.0f;
    m_run[x][0] = m_run[x][1] = -INFINITY;
    l_run[x][0] = l_run[x][1] = 0.0f;
  }
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
#pragma unroll(kN == 1 ? 2 : 1)
    for (int sub = 0; sub < kBlock / (16 * kRowsWarps); ++sub) {
      const int r0 = 16 * (cw + kRowsWarps * sub), t0 = t_base + i * kBlock + r0;
      const uint32_t there = (sh.present[st][r0 >> 5] >> (r0 & 31)) & 0xFFFFu;
      if (!there) continue;
      // ---- S^T = K Q^T: 8 k-steps of 16 channels --------------------------
      const uint4 ka = *reinterpret_cast<const uint4*>(stage + (r0 + rk0) * 64 + 16 * t);
      const uint4 kb = *reinterpret_cast<const uint4*>(stage + (r0 + rk1) * 64 + 16 * t);
      const uint32_t ksa = kv_scales16<kE1M2>(*reinterpret_cast<const uint16_t*>(k_scales + (r0 + rk0) * 8 + 2 * t));
      const uint32_t ksb = kv_scales16<kE1M2>(*reinterpret_cast<const uint16_t*>(k_scales + (r0 + rk1) * 8 + 2 * t));
      const uint32_t sa_lo = __byte_perm(ksa, ksa, 0x1010), sa_hi = __byte_perm(ksa, ksa, 0x3232);
      const uint32_t sb_lo = __byte_perm(ksb, ksb, 0x1010), sb_hi = __byte_perm(ksb, ksb, 0x3232);
      float s[kN][4];
#pragma unroll
      for (int x = 0; x < kN; ++x) s[x][0] = s[x][1] = s[x][2] = s[x][3] = 0.0f;
      const uint32_t kaw[4] = {ka.x, ka.y, ka.z, ka.w}, kbw[4] = {kb.x, kb.y, kb.z, kb.w};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t ha[4], hb[4];
        pairs8<kE1M2>(kaw[w], ha);
        pairs8<kE1M2>(kbw[w], hb);
        const uint32_t sa = w < 2 ? sa_lo : sa_hi, sb = w < 2 ? sb_lo : sb_hi;
        const uint32_t sa1 = kE1M2 ? mul_f16x2(sa, 0x2C002C00u) : sa, sb1 = kE1M2 ? mul_f16x2(sb, 0x2C002C00u) : sb;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t f[4] = {mul_f16x2(ha[2 * h], sa), mul_f16x2(hb[2 * h], sb), mul_f16x2(ha[2 * h + 1], sa1),
                                 mul_f16x2(hb[2 * h + 1], sb1)};
          const int j = 2 * w + h;
#pragma unroll
          for (int x = 0; x < kN; ++x) {
            const uint2 b = kN == 1 ? make_uint2(qf[2 * j], qf[2 * j + 1]) : sh.q[x][j][lane];
            mma16816(s[x], f, b.x, b.y);
          }
        }
      }
      // ---- scores, masks, the running maximum ------------------------------
      const bool open = t0 >= all_lo && t0 + 16 <= all_hi && there == 0xFFFFu;
      bool up = false;
#pragma unroll
      for (int x = 0; x < kN; ++x) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int key = t0 + (c < 2 ? rk0 : rk1), col = c & 1;
          float v = s[x][c] * mult[x][col];
          if (kMods) {
            if (a.cap > 0.0f) {
              const float out = a.cap * kLog2e;
              v = fmaf(-2.0f * out, rcp(1.0f + ex2(v * (2.0f / a.cap))), out);
            }
            v = fmaf(-slope[x][col], fabsf(static_cast<float>(pos[x][col] - key)), v);
          }
          if (!open && (key < vis[x][col].x || key >= vis[x][col].y || !((there >> (key - t0)) & 1u))) v = -INFINITY;
          s[x][c] = v;
          up = up || v > m_run[x][col] + kRescaleLog2;
        }
      }
      if (__any_sync(0xffffffffu, up)) {
#pragma unroll
        for (int x = 0; x < kN; ++x)
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float top = fmaxf(s[x][c], s[x][c + 2]);
#pragma unroll
            for (int sh_ = 4; sh_ < 32; sh_ <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, sh_));
            if (top > m_run[x][c] + kRescaleLog2) {
              const float shrink = ex2(m_run[x][c] - top);
              m_run[x][c] = top;
              l_run[x][c] *= shrink;
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                o[x][k][c] *= shrink;
                o[x][k][c + 2] *= shrink;
              }
            }
          }
      }
      uint32_t pb[kN][2];
#pragma unroll
      for (int x = 0; x < kN; ++x) {
        const float b0 = (m_run[x][0] == -INFINITY ? 0.0f : -m_run[x][0]) + kWeightLog2;
        const float b1 = (m_run[x][1] == -INFINITY ? 0.0f : -m_run[x][1]) + kWeightLog2;
        const float p0 = ex2(s[x][0] + b0), p1 = ex2(s[x][1] + b1), p2 = ex2(s[x][2] + b0), p3 = ex2(s[x][3] + b1);
        l_run[x][0] += p0 + p2;
        l_run[x][1] += p1 + p3;
        pb[x][0] = transposed(f16x2_rn(p0, p1));
        pb[x][1] = transposed(f16x2_rn(p2, p3));
      }
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
#pragma unroll
          for (int x = 0; x < kN; ++x) mma16816(o[x][4 * half + k], f, pb[x][0], pb[x][1]);
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.empty[st]);
  }

  // ---- join the warps, one group of rows at a time -------------------------
  float* merge = reinterpret_cast<float*>(smem_raw + kRing * kStageBytes);
#pragma unroll
  for (int x = 0; x < kN; ++x) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
      for (int s = 4; s < 32; s <<= 1) l_run[x][c] += __shfl_xor_sync(0xffffffffu, l_run[x][c], s);
      if (g == 0) {
        sh.m[cw][8 * x + 2 * t + c] = m_run[x][c];
        sh.l[cw][8 * x + 2 * t + c] = l_run[x][c];
      }
    }
    float* mine = merge + cw * 8 * kMergeRow;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int c = 18 * g + 2 * k;  // channels 16g + 2k and the next, 2 floats of padding per 16
      *reinterpret_cast<float2*>(mine + (2 * t) * kMergeRow + c) = make_float2(o[x][k][0], o[x][k][2]);
      *reinterpret_cast<float2*>(mine + (2 * t + 1) * kMergeRow + c) = make_float2(o[x][k][1], o[x][k][3]);
    }
    asm volatile("bar.sync 1, %0;" ::"n"(32 * kRowsWarps) : "memory");
    const int left = min(8, static_cast<int>(rows) - 8 * x);
    for (int idx = threadIdx.x - 32; idx < left * (kD / 4); idx += 32 * kRowsWarps) {
      const int lr = idx / (kD / 4), c = idx % (kD / 4) * 4;
      float big = -INFINITY, sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < kRowsWarps; ++w) big = fmaxf(big, sh.m[w][8 * x + lr]);
#pragma unroll
      for (int w = 0; w < kRowsWarps; ++w) {
        const float mw = sh.m[w][8 * x + lr], f = mw == -INFINITY ? 0.0f : ex2(mw - big);
        const float2* from = reinterpret_cast<const float2*>(merge + (w * 8 + lr) * kMergeRow + c + 2 * (c >> 4));
        const float2 u = from[0], v = from[1];
        sum = fmaf(f, sh.l[w][8 * x + lr], sum);
        acc[0] = fmaf(f, u.x, acc[0]);
        acc[1] = fmaf(f, u.y, acc[1]);
        acc[2] = fmaf(f, v.x, acc[2]);
        acc[3] = fmaf(f, v.y, acc[3]);
      }
      if (a.splits > 1) {
        const uint64_t rec = ((static_cast<uint64_t>(tile_id) * a.map.hkv + kvh) * a.splits + split) * kRows + 8 * x + lr;
        if (c == 0) a.ml_ws[rec] = make_float2(big, sum);
        if (big != -INFINITY) *reinterpret_cast<float4*>(a.o_ws + rec * kD + c) = make_float4(acc[0], acc[1], acc[2], acc[3]);
      } else {
        const float f = sum > 0.0f ? a.gv / sum : 0.0f;
        const uint32_t r = tile.row0 + 8 * x + lr, tok = a.group.div(r);
        *reinterpret_cast<uint2*>(a.out + (static_cast<uint64_t>(seq.first + tok) * a.hq + kvh * group + r - tok * group) * kD + c) =
            make_uint2(bf16x2_rn(acc[0] * f, acc[1] * f), bf16x2_rn(acc[2] * f, acc[3] * f));
      }
    }
    if (x + 1 < kN) asm volatile("bar.sync 1, %0;" ::"n"(32 * kRowsWarps) : "memory");
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
  int rows;  // of a tile: kTileRows, or 8, 16, 24 by the rows kernel
  int64_t tiles, tiles_per_seq, splits;
  bool full;  // the tile kernel's exact weights
};

// Contexts of up to this many keys take the tile kernel's kFull.
constexpr int64_t kFullContext = 512;

// Which kernel, the tiles (at most), and the parts that each tile's keys are cut into.
Plan plan_for(int64_t batch, int64_t n_tokens, int64_t group, int64_t hkv, int64_t context, bool uniform) {
  Plan p;
  const int64_t sms = sm_count(), blocks = (context + kBlock - 1) / kBlock;
  const int64_t rows = (n_tokens * group + batch - 1) / batch;  // of a sequence and KV head, on average
  p.full = context <= kFullContext;
  p.rows = p.full || rows > 24 ? kTileRows : static_cast<int>((rows + 7) / 8 * 8);
  p.tiles_per_seq = (n_tokens / batch * group + p.rows - 1) / p.rows;
  const int64_t ragged = n_tokens * group / p.rows + (batch < n_tokens ? batch : n_tokens);
  p.tiles = uniform ? batch * p.tiles_per_seq : ragged;
  const int64_t items = p.tiles * hkv;
  p.splits = 1;
  if (p.rows != kTileRows) {
    // Enough CTAs for six rounds on what is resident, so that sequences of
    // different lengths even out, in parts of 512 keys or more; failing that,
    // one round in parts of a stage or more.
    const int64_t resident = sms * (p.rows == 8 ? 4 : p.rows == 16 ? 3 : 2);
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
// Raising the limit is idempotent and cheap; a failure shows at the launch.
Kernel with_smem(Kernel k, uint32_t bytes) {
  cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  return k;
}
template <bool kE1M2, bool kMods>
Kernel kernel_for(const Plan& p) {
  switch (p.rows) {
    case 8: return with_smem(extend_rows_kernel<1, kE1M2, kMods>, kRowsSmem);
    case 16: return with_smem(extend_rows_kernel<2, kE1M2, kMods>, kRowsSmem);
    case 24: return with_smem(extend_rows_kernel<3, kE1M2, kMods>, kRowsSmem);
  }
  return p.full ? with_smem(extend_tile_kernel<kE1M2, kMods, true>, kTileSmem)
                : with_smem(extend_tile_kernel<kE1M2, kMods, false>, kTileSmem);
}
Kernel combine_for(const Plan& p) {
  return p.rows == 8 ? extend_combine_kernel<8> : p.rows == 16 ? extend_combine_kernel<16>
         : p.rows == 24 ? extend_combine_kernel<24> : extend_combine_kernel<kTileRows>;
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
  const Kernel kernel = e1m2 ? (mods ? kernel_for<true, true>(p) : kernel_for<true, false>(p))
                             : (mods ? kernel_for<false, true>(p) : kernel_for<false, false>(p));
  const bool by_tiles = p.rows == kTileRows;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_pdl(kernel, dim3(static_cast<uint32_t>(grid)), dim3(by_tiles ? kTileThreads : kRowsThreads),
                 by_tiles ? kTileSmem : kRowsSmem, s, a) != cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  if (p.splits > 1) {
    if (launch_pdl(combine_for(p), dim3(a.tiles, a.map.hkv, by_tiles ? 8 : (p.rows + 7) / 8), dim3(256), 0, s, a) != cudaSuccess)
      return NVFP4_ERR_CUDA;
    count_launches(1);
  }
  return launch_status();
}
