// What the kernels of extend_attention_nvfp4 share: the arguments, who sees what,
// row tiles and work items, and the small pieces of their arithmetic.
#pragma once

#include "kv_pages.cuh"

namespace nvfp4 {
constexpr int kD = 128;
constexpr int kBlock = 128;      // keys per block
constexpr int kTileRows = 256;   // rows of a tile of the many-row kernel
constexpr float kLog2e = 1.4426950408889634f;

// A weight is 2^(score + minus), scores in the log2 domain.  `minus` is 4 - the row's
// running maximum, rounded once, and moves only where an exponent would pass 15: the
// sum that is compared is the one that becomes the weight, so that no weight passes f16's
// range whatever the scores' size (a maximum plus 11, rounded by itself past 2^24, let
// weights of 2^16 through), and old and new weights differ by exactly the two `minus`.
// The largest weight is 2^4 or more (below scores of 2^26, from which on 4 is lost in
// them), and f16's steps end at 2^-28 of it.
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
  uint32_t splits;                // parts of a tile's keys, at most
  uint32_t part_blocks;           // blocks of a part; 0: each tile's keys in `splits` equal parts
  float* o_ws;                    // [tile][kv head][split][row][128] and, behind them,
  float2* ml_ws;                  // (max, sum) of each such row; unused with one part
  // Test-only (nvfp4_debug_inject_fault): CTA 0's first K stage waits for an arrival that
  // never comes.
  int fault_lose_stage;
};
__device__ __forceinline__ uint32_t lost_arrivals(const ExtendArgs& a, int stage) {
  return a.fault_lose_stage && blockIdx.x == 0 && stage == 0 ? 1u : 0u;
}

// Bounds-checked build: a (token, head) row of the output, a row's record of a part.
__device__ __forceinline__ bool out_in_bounds(const ExtendArgs& a, uint64_t row) {
  return in_bounds(a.status, row < static_cast<uint64_t>(a.n_tokens) * a.hq);
}
template <int kRows>
__device__ __forceinline__ bool record_in_bounds(const ExtendArgs& a, uint64_t rec) {
  return in_bounds(a.status, rec < static_cast<uint64_t>(a.tiles) * a.map.hkv * a.splits * kRows);
}

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

// Keys that the query at position p >= 0 sees: [lo, hi).  (A query before its sequence's first
// token, p < 0, sees none; p is raised to 0 so that no window reaches past 32 bits.)
__device__ __forceinline__ int2 visible(const ExtendArgs& a, int p, int len, int prefix, int doc) {
  int lo = max(doc, 0);
  if (a.window) lo = max(lo, max(p, 0) - a.window + 1);
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

// Parts of fixed size: the keys that a sequence's queries may see, from `lo` (by
// the window) to its length, in parts of part_blocks.
struct Span {
  int lo;
  uint32_t parts;
};
__device__ __forceinline__ Span span_of(const ExtendArgs& a, const Seq& s) {
  const int first = max(0, s.len - static_cast<int>(s.n));  // position of the first query that sees any
  const int lo = a.window ? max(0, first + 1 - a.window) : 0;
  const uint32_t keys = static_cast<uint32_t>(max(s.len - lo, 0)), part = a.part_blocks * kBlock;
  return {lo, max(1u, (keys + part - 1) / part)};
}

// Work item `index` of all sequences' (tile, KV head, part) triples, the parts
// of a tile side by side.  By a converged warp; tile.b = batch: no such item.
struct Item {
  Tile tile;
  Seq seq;
  Span span;
  uint32_t tile_id, kvh, part;
};
template <int kRows>
__device__ __forceinline__ Item find_item(const ExtendArgs& a, uint32_t index) {
  const uint32_t lane = threadIdx.x & 31;
  Item it;
  it.tile = {a.map.batch, 0};
  uint32_t items_before = 0, tiles_before = 0;
  for (uint32_t base = 0; base < a.map.batch; base += 32) {
    const uint32_t b = base + lane;
    Seq s = {0, 0, 0};
    if (b < a.map.batch) s = sequence(a, b);
    const Span span = span_of(a, s);
    const uint32_t tiles = (s.n * a.group.d + kRows - 1) / kRows;
    uint32_t items_to = tiles * a.map.hkv * span.parts, tiles_to = tiles;
#pragma unroll
    for (int sh = 1; sh < 32; sh <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, items_to, sh), w = __shfl_up_sync(0xffffffffu, tiles_to, sh);
      if (lane >= static_cast<uint32_t>(sh)) {
        items_to += v;
        tiles_to += w;
      }
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, index < items_before + items_to);
    if (hit) {
      const int l = __ffs(hit) - 1;
      const uint32_t own = __shfl_sync(0xffffffffu, tiles, l);
      it.seq = {__shfl_sync(0xffffffffu, s.first, l), __shfl_sync(0xffffffffu, s.n, l), __shfl_sync(0xffffffffu, s.len, l)};
      it.span = {__shfl_sync(0xffffffffu, span.lo, l), __shfl_sync(0xffffffffu, span.parts, l)};
      const uint32_t items = own * a.map.hkv * it.span.parts;
      uint32_t i = index - (items_before + __shfl_sync(0xffffffffu, items_to, l) - items);
      const uint32_t first_tile = tiles_before + __shfl_sync(0xffffffffu, tiles_to, l) - own;
      it.part = i % it.span.parts;
      i /= it.span.parts;
      it.kvh = i % a.map.hkv;
      i /= a.map.hkv;
      it.tile_id = first_tile + i;
      // Counted as find_tile does.  (Overlapping q_start could give more tiles than there is room for.)
      if (it.tile_id < a.tiles) it.tile = {base + l, (own - 1 - i) * kRows};
      return it;
    }
    items_before += __shfl_sync(0xffffffffu, items_to, 31);
    tiles_before += __shfl_sync(0xffffffffu, tiles_to, 31);
  }
  return it;
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

// ---- tcgen05, kind::f16 ----------------------------------------------------
constexpr uint32_t kOperand = 32768;  // bytes of a 128 x 128 f16 operand
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
__device__ __forceinline__ uint64_t pair(float x, float y) {
  uint64_t d;
  asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y));
  return d;
}
__device__ __forceinline__ void unpair(uint64_t v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// A cap in the log2 domain: s <- out tanh(s in), out = c log2(e), for kN scores of a
// lane.  y = s in.  For |y| <= 0.5 tanh(y) / y is a polynomial in y^2 (the three
// coefficients that make the largest relative error least, 2^-20.6: a weight's is then
// below 2^-15 for caps up to 50), two scores an FMA; a score far below the cap keeps its
// own relative precision whatever the cap.  Else tanh(y) = 1 - 2 / (1 + 2^(2 log2(e) y)):
// the absolute error, some 2^-22, is then relative to more than 0.46 (and the hardware
// tanh's 2^-11 would show).  Each score takes its own form, so that a row's result does
// not go by its neighbours'; a warp without a score past 0.5 leaves the second out, since
// the special-function unit has every weight's exponential to do (a chunk of 2048 on
// 16384 keys, 64 heads, took 1565 us by the second alone).
constexpr float kTanh1 = -0.333281606f, kTanh2 = 0.132053599f, kTanh3 = -0.0447506458f;
constexpr float kTanhRange = 0.5f;
__device__ __forceinline__ float capped_far(float y, float out) { return fmaf(-2.0f * out, rcp(1.0f + ex2(y * (2.0f * kLog2e))), out); }
template <int kN>
__device__ __forceinline__ void cap_scores(float* s, float in, float out) {
  float far[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kN; i += 2) far[(i >> 1) & 1] = max3(fabsf(s[i]), fabsf(s[i + 1]), far[(i >> 1) & 1]);
  const uint64_t in2 = both(in), c0 = both(out), c1 = both(out * kTanh1), c2 = both(out * kTanh2), c3 = both(out * kTanh3);
  const auto near = [&](float a, float b) {
    const uint64_t y = mul2(pair(a, b), in2), u = mul2(y, y);
    return mul2(y, fma2(fma2(fma2(c3, u, c2), u, c1), u, c0));
  };
  if (__any_sync(0xffffffffu, fmaxf(far[0], far[1]) * in > kTanhRange)) {
#pragma unroll
    for (int i = 0; i < kN; i += 2) {
      const float a = s[i] * in, b = s[i + 1] * in;
      unpair(near(s[i], s[i + 1]), s[i], s[i + 1]);
      if (fabsf(a) > kTanhRange) s[i] = capped_far(a, out);
      if (fabsf(b) > kTanhRange) s[i + 1] = capped_far(b, out);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kN; i += 2) unpair(near(s[i], s[i + 1]), s[i], s[i + 1]);
  }
}
// The same where in = 1 / out: out y = s, and the constants are immediates, for the
// kernels that have no registers for them.
template <int kN>
__device__ __forceinline__ void cap_scores(float* s, float out) {
  const float in = 1.0f / out;
  float far = 0.0f;
#pragma unroll
  for (int i = 0; i < kN; i += 2) far = max3(fabsf(s[i]), fabsf(s[i + 1]), far);
  const auto near = [&](float x) {
    const float y = x * in, u = y * y;
    return x * fmaf(fmaf(fmaf(kTanh3, u, kTanh2), u, kTanh1), u, 1.0f);
  };
  if (__any_sync(0xffffffffu, far * in > kTanhRange)) {
#pragma unroll
    for (int i = 0; i < kN; ++i) s[i] = fabsf(s[i]) * in > kTanhRange ? capped_far(s[i] * in, out) : near(s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < kN; ++i) s[i] = near(s[i]);
  }
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

// The eight elements of a code word times their block scale (kv_scales16) as four
// f16x2.  E2M1: channels (0,1) (2,3) (4,5) (6,7).  E1M2: (0,4) (1,5) (2,6) (3,7): a
// nibble is decoded where it stands, its sign bit turned over, in the low bits of
// 1024: 1032 + n, or in bits 4-7 1152 + 16 n, where 1152 scale / 16 has no more than 8
// significant bits and one FMA gives n scale exactly.  Q is laid out in the same
// order, and O comes in V's.
template <bool kE1M2>
__device__ __forceinline__ void scaled8(uint32_t w, uint32_t scale, uint32_t e[4]) {
  if (kE1M2) {
    const uint32_t t = w >> 8, scale16 = mul_f16x2(scale, 0x2C002C00u), less = mul_f16x2(scale, 0xD480D480u);
    e[0] = mul_f16x2(sub_f16x2((w & 0x000F000Fu) ^ 0x64086408u, 0x64086408u), scale);
    e[1] = fma_f16x2((w & 0x00F000F0u) ^ 0x64806480u, scale16, less);
    e[2] = mul_f16x2(sub_f16x2((t & 0x000F000Fu) ^ 0x64086408u, 0x64086408u), scale);
    e[3] = fma_f16x2((t & 0x00F000F0u) ^ 0x64806480u, scale16, less);
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

// A query row's scaling by a power of two to below 1, from the bits of its largest |x|
// (amax_bits_bf16x8): down = 2^-e, up = 2^e, both normal numbers.  A row with an infinity
// or a NaN becomes NaN in every channel, so that all its scores are NaN, and its result
// whatever the signs of the keys that it meets.
struct RowScale {
  float down, up;
};
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  const int e = max(-125, min(static_cast<int>(top >> 7) - 126, 126));
  if (top >= 0x7F80u) return {__uint_as_float(0x7FC00000u), 1.0f};
  return {__uint_as_float(static_cast<uint32_t>(127 - e) << 23), __uint_as_float(static_cast<uint32_t>(127 + e) << 23)};
}
// What a row's products of Q and K are multiplied by.  Kept a normal number: hidden scores, minus
// infinity, may be multiplied by it, and products of 0.
__device__ __forceinline__ float score_factor(float scale, float up) { return fminf(fmaxf(scale * kLog2e * up, FLT_MIN), FLT_MAX); }
// The factor of a row's output from the sum of its weights: 0 where it sees no key (a sum
// of 0 exactly), NaN where a weight was.
__device__ __forceinline__ float per_sum(float sum, float gv) { return sum == 0.0f ? 0.0f : gv / sum; }

// Two f16 values of at most 7 significant bits, at least 2^-14 or zero -> bf16,
// exact: the 5-bit exponent moves into the 8-bit field, 2^112 makes up for the bias.
__device__ __forceinline__ uint32_t bf16x2_of_f16x2(uint32_t h) {
  uint32_t d;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(((h >> 3) & 0x0FFF0FFFu) | (h & 0x80008000u)), "r"(0x77807780u));
  return d;
}

// ---- the kernels -----------------------------------------------------------
using ExtendKernel = void (*)(const ExtendArgs);
struct ExtendLaunch {
  ExtendKernel kernel;
  uint32_t threads, smem;
};
ExtendLaunch extend_tiles(bool e1m2, bool cap, bool bias, bool full);  // kTileRows a tile
ExtendLaunch extend_rows(int rows, bool e1m2, bool cap, bool full);  // 16, 24, 32; 8 with `full`
ExtendLaunch extend_decode(bool e1m2, bool mods);                    // 8

}  // namespace nvfp4
