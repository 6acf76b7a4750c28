// The experts' linears: block-scaled FP4 x FP4 products of rows sorted by expert,
// each expert's rows with its own weight.
//   out[r, n] = bf16( g_a[e] g_w[e] sum_k a[r, k] w_e[n, k] ),  r among expert e's rows
// and the same for gate_up with h = SiLU(gate) up quantized in the epilogue.
//
// A pair of CTAs has a tile of 256 weight rows and up to 256 of one expert's rows (64
// in the form for few rows an expert) by tcgen05.mma.cta_group::2 (kind::mxf4nvf4,
// 16-element block scales).  The weight
// is the M side: its rows come in 256s whatever the router does, while an expert may
// have one row or 700, and N takes any multiple of 32.  So a few rows cost the
// weight's bytes and no more, and many leave at most 31 columns idle.  Each CTA holds
// its 128 weight rows and half of the tokens' rows; D[weight row, token] is in its
// own TMEM lanes.  Which tiles there are follows from the plan on the device: every
// CTA sums the experts' tiles (shared memory); an expert's units are next to each
// other, those of one weight tile first, so that its bytes come from DRAM once.  The
// launch has a cluster for each unit that there may be; those that run take the next
// ones that have not started (cluster launch control) and stay on their SMs: units of
// 32 to 256 tokens even out.
//   warp 0      codes; a CTA's weight rows and its half of the tokens' rows
//   warp 1      leader: MMAs; peer: block scales
//   warp 2      leader: block scales into TMEM; peer: the queue of units
//   warp 3      leader: block scales
//   warps 4-    epilogue: 32 weight rows x every second (of 8 warps) or fourth (of 16) 32 tokens each
// Output rows are bf16, the type that the rows' other calls take: the one rounding of
// the fp32 sum; quantized outputs have the recipe's own alone.  The epilogue reads 16 x
// 8 fragments of D (16x256b), in which a thread has two tokens of two weight rows, and
// of gate and up at once: bf16 rows are turned into token-major ones by a transposing
// stmatrix, quantized outputs need shuffles only.
//
// What bounds it.  Few tokens: the weights from DRAM, at 6.3 of the measured 6.78 TB/s from one size to the other, and some 4
// us around that a launch takes to start, fill and drain (means of three batches: 64 tokens on 69 of 128 experts, 2048 x
// 1536, 123 MB of codes and scales in 23.4 us; 500 on 56 of 64, 4096 x 2560, 330 MB in 56.5).  Many: the loads into the SMs.
// 8192 tokens x 4 on 64 experts, 5120 x 2048, read 1.93 GB from L2, 16.4 TB/s without the MMAs in 118 us, with them in 132 to
// 136 (5.2 PFLOP/s); one expert of 8192 rows, 5120 x 13824, 6.8 PFLOP/s in 171 us, as nvfp4_linear_swiglu_quantize.  The
// accumulator takes all TMEM that the scales leave, so a unit's end (last MMAs, drain) costs 2000 cycles of 10240 at K =
// 5120, and at K = 1024 a unit's loads, MMAs and stores run almost one after another: some 2000 cycles each of 5000, with L2
// at 46 %, DRAM at 56 and the tensor pipe at 34 (8192 x 4, 1024 x 5120: 106 us).  Tried: the tokens as the M side (half of
// the MMAs of an expert with 128 rows idle); units in a fixed order (the pairs with whole tiles ended 20 % later); weights
// asked for in L2 ahead of time (56 -> 64 us at 500 tokens); units of 32 experts mixed (132 -> 153 at 8192); two accumulators
// of 128 columns (nothing at 64 tokens, 132 -> 139 at 8192); two CTAs an SM with tiles of 128 tokens (between the two forms
// or behind both: 2048 tokens on 16 experts 28.3 with 64, 24.7 with 128, 22.8 with 256; 8192 tokens 153).
#include <cuda.h>
#include <cudaTypedefs.h>

#include <cfloat>
#include <map>
#include <mutex>

#include "moe_plan.cuh"
#include "nvfp4_quant.cuh"

namespace nvfp4 {
namespace {

constexpr int kDepth = 256;  // elements of K per stage: 128 bytes of a row
constexpr int kWRows = 256;
constexpr int kEpi0 = 4;
constexpr int kQueue = 4;  // units on their way to the warps
constexpr uint32_t kWBytes = 128 * kDepth / 2;                             // a CTA's weight codes of a stage
constexpr uint32_t kScaleTile = 128 * kDepth / 16;                         // block scales of 128 rows: four atoms
constexpr uint32_t kEpiBytes = 2048;                                       // a warp's 32 tokens x 32 bf16

// kMode: 0 bf16 rows, 1 SwiGLU to NVFP4, 2 SwiGLU to MXFP4.
// kSmall false: tiles of up to 256 tokens, one CTA an SM.  Modes 0 and 2 have 8 epilogue warps with 128 accumulator
// registers a thread; mode 1 needs no shared memory there and is bound by its own latency where K is short: 16 warps with 64.
// kSmall true: tiles of up to 64 tokens, two CTAs an SM: one's start, fill and drain under the other's loads, of the same
// launch or of the next one.
template <int kMode_, bool kSmall_>
struct Form {
  static constexpr int kMode = kMode_;
  static constexpr bool kSmall = kSmall_;
  static constexpr int kTokens = kSmall ? 64 : 256;  // of a tile
  static constexpr int kStages = !kSmall ? 5 : kMode == 1 ? 4 : 3;
  static constexpr int kXTiles = kSmall ? 1 : 2;     // scale tiles of the tokens
  static constexpr int kEpiWarps = kMode == 1 && !kSmall ? 16 : 8;
  static constexpr int kThreads = 32 * (kEpi0 + kEpiWarps);
  static constexpr int kSides = kEpiWarps / 4;             // warps with the same weight rows
  static constexpr int kChunks = kTokens / 32 / kSides;    // of 32 tokens, a warp's
  static constexpr uint32_t kXBytes = kTokens / 2 * kDepth / 2;  // a CTA's token codes of a stage
  static constexpr uint32_t kXScales = kXTiles * kScaleTile;
  static constexpr uint32_t kTmemCols = kSmall ? 256 : 512, kSfCol = kTokens, kSfCols = 16 + 16 * kXTiles;
  static constexpr int kEpiSmem = kMode == 1 ? 0 : kEpiWarps * static_cast<int>(kEpiBytes);
  static constexpr int kPer = (kMoeMaxExperts + kThreads - 1) / kThreads;  // experts of a thread
  static constexpr size_t kSmem = 1024 + kStages * (kWBytes + kXBytes + kScaleTile + kXScales) + kEpiSmem +
                                  kMoeMaxExperts * (sizeof(int) + sizeof(int2)) + 512;
  static_assert(kSfCol + kStages * kSfCols <= kTmemCols, "TMEM budget");
  static_assert(kSmem <= 227 * 1024 && (!kSmall || 2 * (kSmem + 1024 + 256) <= 228 * 1024), "shared memory budget");
};
// kind::mxf4nvf4: A and B packed E2M1, K-major; M = 256.  N >> 3 is added at bit 17, UE8M0 scales set bit 23.
constexpr uint32_t kIdesc = (1u << 7) | (1u << 10) | (static_cast<uint32_t>(kWRows >> 4) << 24);
constexpr uint32_t kUE8M0 = 1u << 23;

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
  int experts, max_rows, choices, N, K, g_a_step, g_out_step;
  int w_tiles;        // 256-row tiles of an expert's weight
  int w_scale_tiles;  // 128-row tiles of its scales
  int max_units;      // what a plan can have: one of any numbers is cut to it
  bool mx;
  bool rotate;
  int fault_skip_stage;  // test-only: pair 0 leaves its first stage neither armed nor loaded
  int reversed;          // test-only: the clusters' units from the last cluster on, as if the clusters started so
  int* status;
};

// ------------------------------------------------------------- PTX pieces ---

// K-major operand tile, 128-byte swizzle: rows of 128 B, 8-row groups 1024 B apart.
__device__ __forceinline__ uint64_t tile_desc(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (1ull << 16) | (static_cast<uint64_t>(1024 >> 4) << 32) |
         (1ull << 46) | (2ull << 61);
}
// A 512-byte scale atom: 32 rows of 16 B, no swizzle, 8-row core matrices 128 B apart.
__device__ __forceinline__ uint64_t atom_desc(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(128 >> 4) << 16) |
         (static_cast<uint64_t>(128 >> 4) << 32) | (1ull << 46);
}
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb,
                                         uint32_t accumulate) {
  asm volatile(
      "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
      " tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%5], [%6], p;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sfa), "r"(sfb)
      : "memory");
}
__device__ __forceinline__ void pair_copy_scales(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void pair_commit(uint64_t* bar, uint16_t mask) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                   smem_u32(bar)),
               "h"(mask)
               : "memory");
}
__device__ __forceinline__ void pair_tmem_alloc(uint32_t* slot, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(cols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_tmem_free(uint32_t taddr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
__device__ __forceinline__ uint32_t leader_address(const uint64_t* bar) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(bar)));
  return r;
}
// Boxes into this CTA's shared memory, counted on the leader's barrier at `bar`.
__device__ __forceinline__ void load_box(void* dst, const void* map, uint64_t* bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(leader_address(bar)), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void load_box3(void* dst, const void* map, uint64_t* bar, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(leader_address(bar)), "r"(0), "r"(y), "r"(z)
      : "memory");
}
// Arrives without release: hands back an accumulator whose TMEM loads are complete and fenced, or a place of the queue
// whose 16 bytes one load has brought into registers that the warp has used; no memory that the warp wrote is read after it.
// (With release, which waits for the epilogue's stores, down of 8192 tokens takes 143 us for 106.)
__device__ __forceinline__ void arrive_relaxed(uint32_t pair_addr) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(pair_addr) : "memory");
}
// After a pipeline gave up: lets this thread's copies land before its pair exits.
__device__ __forceinline__ void wait_for_copies() {
  const uint64_t t0 = globaltimer_ns();
  while (globaltimer_ns() - t0 < kDrainLimitNs) __nanosleep(100000);
}
// 16 lanes x 32 columns: registers 4j .. 4j + 3 are columns 8j + 2 (lane % 4) and the next one, of lane's row
// lane / 4 and of the row 8 below.
__device__ __forceinline__ void tmem_ld_fragments(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_done() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  uint32_t d;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}
__device__ __forceinline__ uint32_t e2m1x2(float lo, float hi) {
  uint32_t d;
  asm("{\n .reg .b8 b;\n .reg .b16 h;\n cvt.rn.satfinite.e2m1x2.f32 b, %2, %1;\n mov.b16 h, {b, 0};\n cvt.u32.u16 %0, h;\n}"
      : "=r"(d)
      : "f"(lo), "f"(hi));
  return d;
}
// Four transposed 8 x 8 matrices of 16-bit elements; lane l has the address of row l % 8 of matrix l / 8.
__device__ __forceinline__ void stmatrix_t(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b),
               "r"(c), "r"(d)
               : "memory");
}
// SiLU(gate) * up by the hardware's 2^x and 1 / x, within 2^-22 each; 2^x takes an argument rounded to 2^-24 of itself.
__device__ __forceinline__ float silu_mul(float gate, float up) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(gate * -1.4426950408889634f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return gate * r * up;
}
// Two warps of the epilogue meet; true where both gave true.
__device__ __forceinline__ bool both(int id, bool ok) {
  int r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.b32 p, %2, 0;\n barrier.cta.red.and.pred q, %1, 64, p;\n selp.s32 %0, 1, 0, q;\n}"
      : "=r"(r)
      : "r"(id), "r"(ok ? 1 : 0)
      : "memory");
  return r != 0;
}
// The launch's clusters that have not started are its queue: a CTA of a running cluster takes one (its first CTA's index)
// in place of a start.  The answer is 16 bytes of this CTA's shared memory.
__device__ __forceinline__ void take_cluster(void* answer, uint64_t* bar) {
  asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                   smem_u32(answer)),
               "r"(smem_u32(bar))
               : "memory");
}
// The index of the cluster that was taken, -1: none was left.
__device__ __forceinline__ int taken_cluster(const void* answer) {
  uint32_t some, x;
  asm volatile(
      "{\n .reg .pred p;\n .reg .b128 h;\n ld.shared.b128 h, [%2];\n"
      " clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, h;\n selp.u32 %0, 1, 0, p;\n mov.u32 %1, 0;\n"
      " @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, h;\n}"
      : "=r"(some), "=r"(x)
      : "r"(smem_u32(answer))
      : "memory");
  return some ? static_cast<int>(x / 2) : -1;
}
// Of what is at this offset in CTA `rank` of the pair.
__device__ __forceinline__ uint32_t pair_address(const void* p, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
  return r;
}
// 16 bytes to CTA `rank` of the pair, counted on its barrier.
__device__ __forceinline__ void send_16(const void* dst, const uint64_t* bar, uint32_t rank, int4 v) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(
                   pair_address(dst, rank)),
               "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w), "r"(pair_address(bar, rank))
               : "memory");
}
__device__ __forceinline__ void expect_in_pair(const uint64_t* bar, uint32_t rank, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" ::"r"(pair_address(bar, rank)), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void meet(int id) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(id) : "memory"); }

// ------------------------------------------------------------------ units ---

struct Unit {
  int expert, w_tile;
  int row0, tokens;  // first row, rows of the tile; tokens 0: there is no unit
  __device__ __forceinline__ int n() const { return (tokens + 31) & ~31; }  // the MMA's N
};
static_assert(sizeof(Unit) == 16, "one store of the queue, and one load");
__device__ __forceinline__ Unit load_unit(const Unit* slot) {
  Unit t;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(t.expert), "=r"(t.w_tile), "=r"(t.row0), "=r"(t.tokens)
               : "r"(smem_u32(slot))
               : "memory");
  return t;
}
// Unit u, by a converged warp.  ends: [1024] units of the experts up to each one, the total behind the last one.
template <int kTokens>
__device__ __forceinline__ Unit find_unit(int u, const int* ends, const int2* rows, int lane) {
  const int block = __popc(__ballot_sync(0xffffffffu, ends[32 * lane + 31] <= u));
  const int e = 32 * block + __popc(__ballot_sync(0xffffffffu, ends[32 * block + lane] <= u));
  const int2 r = rows[e];  // first row, rows
  const int local = u - (e ? ends[e - 1] : 0), tiles = (r.y + kTokens - 1) / kTokens;
  Unit t;
  t.expert = e;
  t.w_tile = local / tiles;
  const int token_tile = local - t.w_tile * tiles;
  t.row0 = r.x + token_tile * kTokens;
  t.tokens = min(kTokens, r.y - token_tile * kTokens);
  return t;
}

// --------------------------------------------------------------- epilogue ---
// lo, hi: the fragments of a warp's weight rows 0..15 and 16..31, 32 tokens from token0.

__device__ __forceinline__ void store_rows(const GroupedArgs& a, const void* map_out, const Unit& t, const uint32_t* lo,
                                           const uint32_t* hi, int token0, int n0, float scale, uint32_t buf, int lane) {
  auto f = [&](uint32_t v) { return __uint_as_float(v) * scale; };
  // Rows of 64 bytes in 16-byte chunks, chunk c of token t at c ^ (t / 2) % 4: no bank twice, written or read.
  // That is also the 64-byte swizzle of a box of 32 x 32, which goes out by itself while the warp turns to the next; rows
  // that are fewer go out by the lanes.
  if (lane == 0) bulk_wait_read_all();  // the last box has left the buffer
  __syncwarp();
  const uint32_t put = buf + (lane & 7) * 64 + (((lane >> 3) ^ ((lane >> 1) & 3)) << 4);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    stmatrix_t(put + j * 512, pack_pair(f(lo[4 * j]), f(lo[4 * j + 1])), pack_pair(f(lo[4 * j + 2]), f(lo[4 * j + 3])),
               pack_pair(f(hi[4 * j]), f(hi[4 * j + 1])), pack_pair(f(hi[4 * j + 2]), f(hi[4 * j + 3])));
  if (token0 + 32 <= t.tokens) {
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0 && in_bounds(a.status, t.row0 + token0 + 32 <= a.max_rows)) {
      asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                       reinterpret_cast<uint64_t>(map_out)),
                   "r"(buf), "r"(n0), "r"(t.row0 + token0)
                   : "memory");
      bulk_commit_group();
    }
    return;
  }
  __syncwarp();
  const int c = lane & 3, n = n0 + 8 * c, tk0 = lane >> 2;
  const uint32_t get = buf + tk0 * 64 + ((c ^ ((tk0 >> 1) & 3)) << 4);
  uint4 v[4];
#pragma unroll
  for (int it = 0; it < 4; ++it)
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[it].x), "=r"(v[it].y), "=r"(v[it].z), "=r"(v[it].w)
                 : "r"(get + it * 512)
                 : "memory");
  __syncwarp();
  if (n >= a.N || !in_bounds(a.status, t.row0 + min(token0 + 32, t.tokens) <= a.max_rows && n + 8 <= a.N))
    return;  // N % 16 == 0: a chunk is inside or outside
  uint16_t* dst = a.out + static_cast<int64_t>(t.row0 + token0 + tk0) * a.ldo + n;
#pragma unroll
  for (int it = 0; it < 4; ++it) {
    if (token0 + tk0 + 8 * it < t.tokens) *reinterpret_cast<uint4*>(dst) = v[it];
    dst += 8 * a.ldo;
  }
}

// h = SiLU(gate) up over lo; lane has rows lane / 4 and 8 below, tokens 2 (lane % 4) and the next.
__device__ __forceinline__ void swiglu_fragments(uint32_t* lo, const uint32_t* hi, float scale) {
#pragma unroll
  for (int i = 0; i < 16; ++i)
    lo[i] = __float_as_uint(silu_mul(__uint_as_float(lo[i]) * scale, __uint_as_float(hi[i]) * scale));
}

// Quantization of 32 tokens of 16 outputs.  A lane's own token is 8 (lane / 8) + 2 (lane % 4) + (lane / 4) % 2: what a
// token needs once (its largest magnitude, its scale, its codes' word) is with its lane.  The eight lanes with the
// same lane % 4 hold all of eight tokens' outputs: fragment 4j + p of token 8j + 2 (lane % 4) + p.

// The largest magnitude of the lane's token: each step halves the tokens that a lane keeps.
__device__ __forceinline__ float token_amax(const uint32_t* h, int lane) {
  float m[8];  // tokens 2j + p of the eight
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const int i = 4 * (s >> 1) + (s & 1);
    m[s] = fmaxf(fabsf(__uint_as_float(h[i])), fabsf(__uint_as_float(h[i + 2])));
  }
#pragma unroll
  for (int half = 4; half; half >>= 1) {
    const bool upper = lane & (4 * half);
#pragma unroll
    for (int s = 0; s < half; ++s)
      m[s] = fmaxf(upper ? m[s + half] : m[s], __shfl_xor_sync(0xffffffffu, upper ? m[s] : m[s + half], 4 * half));
  }
  return m[0];
}

// The 16 codes of the lane's token, output 0 in the lowest nibble; mult: the token's factor.
__device__ __forceinline__ uint2 token_codes(const uint32_t* h, float mult, int lane) {
  // Bytes of the eight tokens: the code of row lane / 4 in the low nibble, of 8 below in the high one.
  uint32_t byte[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) {
    const float m = __shfl_sync(0xffffffffu, mult, (lane & 3) | s << 2);
    const int i = 4 * (s >> 1) + (s & 1);
    byte[s] = e2m1x2(__fmul_rn(__uint_as_float(h[i]), m), __fmul_rn(__uint_as_float(h[i + 2]), m));
  }
  const uint32_t w0 = byte[0] | byte[1] << 8 | byte[2] << 16 | byte[3] << 24;
  const uint32_t w1 = byte[4] | byte[5] << 8 | byte[6] << 16 | byte[7] << 24;
  // Transposed over the eight lanes, a bit of lane / 4 a step: x0, y0, z0 come from the lane where it is 0.
  const bool b4 = lane & 16, b3 = lane & 8, b2 = lane & 4;
  uint32_t keep = b4 ? w1 : w0, got = __shfl_xor_sync(0xffffffffu, b4 ? w0 : w1, 16);
  const uint32_t x0 = b4 ? got : keep, x1 = b4 ? keep : got;
  keep = __byte_perm(x0, x1, b3 ? 0x7632 : 0x5410);
  got = __shfl_xor_sync(0xffffffffu, __byte_perm(x0, x1, b3 ? 0x5410 : 0x7632), 8);
  const uint32_t y0 = b3 ? got : keep, y1 = b3 ? keep : got;
  keep = __byte_perm(y0, y1, b2 ? 0x7531 : 0x6420);
  got = __shfl_xor_sync(0xffffffffu, __byte_perm(y0, y1, b2 ? 0x6420 : 0x7531), 4);
  const uint32_t z0 = b2 ? got : keep, z1 = b2 ? keep : got;
  const uint32_t a = __byte_perm(z0, z1, 0x6240), b = __byte_perm(z0, z1, 0x7351);  // rows 0-3 and 4-7
  // Nibbles of a row's byte into the words of rows 0-7 and 8-15.
  auto join = [](uint32_t x, uint32_t y) { return __byte_perm(x | x >> 4, y | y >> 4, 0x6420); };
  return make_uint2(join(a & 0x0F0F0F0Fu, b & 0x0F0F0F0Fu), join(a >> 4 & 0x0F0F0F0Fu, b >> 4 & 0x0F0F0F0Fu));
}

__device__ __forceinline__ void store_codes(const GroupedArgs& a, const Unit& t, uint2 codes, uint32_t code, int token0,
                                            uint32_t oc, int lane) {
  const int tk = token0 + 8 * (lane >> 3) + 2 * (lane & 3) + ((lane >> 2) & 1);
  if (tk >= t.tokens) return;
  const uint64_t row = t.row0 + tk;
  const uint32_t cols = static_cast<uint32_t>(a.N) >> 1;
  const uint64_t off = mma_scale_offset(row, oc >> 4, cols >> 6);
  if (!in_bounds(a.status, row < static_cast<uint64_t>(a.max_rows) && oc + 16 <= cols &&
                               off < static_cast<uint64_t>(a.max_rows) * (cols >> 4)))
    return;
  *reinterpret_cast<uint2*>(a.q_codes + row * (cols >> 1) + (oc >> 1)) = codes;
  a.q_scales[off] = static_cast<uint8_t>(code);
}

template <class F>
__global__ void __launch_bounds__(F::kThreads, F::kSmall ? 2 : 1)
    grouped_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_w_scales,
                   const __grid_constant__ CUtensorMap map_x16, const __grid_constant__ CUtensorMap map_x_mid,
                   const __grid_constant__ CUtensorMap map_x128, const __grid_constant__ CUtensorMap map_x_scales,
                   const __grid_constant__ CUtensorMap map_x_scales2, const __grid_constant__ CUtensorMap map_out,
                   const GroupedArgs a) {
  constexpr int kMode = F::kMode, kStages = F::kStages;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sW = smem;
  uint8_t* sX = sW + kStages * kWBytes;
  uint8_t* sWS = sX + kStages * F::kXBytes;
  uint8_t* sXS = sWS + kStages * kScaleTile;
  uint8_t* sEpi = sXS + kStages * F::kXScales;
  int2* expert_rows_s = reinterpret_cast<int2*>(sEpi + F::kEpiSmem);
  int* ends = reinterpret_cast<int*>(expert_rows_s + kMoeMaxExperts);
  uint64_t* full = reinterpret_cast<uint64_t*>(ends + kMoeMaxExperts);  // codes landed, scales in TMEM
  uint64_t* empty = full + kStages;                                    // the stage's MMAs are done
  uint64_t* scales_in = empty + kStages;                               // block scales landed
  uint64_t* acc_full = scales_in + kStages;
  uint64_t* acc_empty = acc_full + 1;
  uint64_t* drain = acc_empty + 1;
  uint64_t* drain_copies = drain + 1;
  uint64_t* unit_full = drain_copies + 1;
  uint64_t* unit_empty = unit_full + kQueue;  // the peer's is used
  uint64_t* unit_begun = unit_empty + kQueue;  // the peer's: its first load is about to be issued
  uint64_t* answer_in = unit_begun + kQueue;   // the peer's
  Unit* queue = reinterpret_cast<Unit*>((reinterpret_cast<uintptr_t>(answer_in + 1) + 15) & ~uintptr_t(15));
  uint8_t* answer = reinterpret_cast<uint8_t*>(queue + kQueue);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(answer + 16);
  __shared__ volatile int abort_flag, late_unit;
  __shared__ int64_t warp_sum[F::kThreads / 32];

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int kblocks = a.K / kDepth;
  const uint32_t rank = cluster_ctarank();
  const bool leader = rank == 0;
  const int clusters = gridDim.x / 2;
  const auto unit_of = [&](int cluster) { return a.reversed ? clusters - 1 - cluster : cluster; };
  int first_unit = unit_of(blockIdx.x / 2);

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      // The commit of the copies of the stage's scales into TMEM, in the leader also an expect_tx of both CTAs' codes.
      mbar_init(&full[s], leader ? 2 : 1);
      mbar_init(&empty[s], 1);
      mbar_init(&scales_in[s], 1);
    }
    mbar_init(acc_full, 1);
    mbar_init(acc_empty, 2 * F::kEpiWarps);
    mbar_init(drain, 1);
    mbar_init(drain_copies, 1);
    mbar_init(answer_in, 1);
    for (int i = 0; i < kQueue; ++i) {
      mbar_init(&unit_full[i], 1);
      mbar_init(&unit_empty[i], 4 + 2 + 2 * F::kEpiWarps);  // the leader's four first warps, the peer's two
      mbar_init(&unit_begun[i], 1);
    }
    abort_flag = 0;
    fence_mbar_init();
    prefetch_tmap(&map_w);
    prefetch_tmap(&map_w_scales);
    prefetch_tmap(&map_x16);
    prefetch_tmap(&map_x_scales);
  }
  if (warp == 1) pair_tmem_alloc(tmem_slot, F::kTmemCols);
  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  griddep_wait_and_release();

  // The experts' rows and units: a few experts a thread, summed over the CTA.
  {
    int64_t n[F::kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < F::kPer; ++i) {
      const int e = F::kPer * threadIdx.x + i;
      n[i] = 0;
      if (e < a.experts) {
        const ExpertRows r = expert_rows(a.row_start, a.rows, e, a.max_rows, a.choices);
        expert_rows_s[e] = make_int2(r.first, r.n);
        n[i] = static_cast<int64_t>((r.n + F::kTokens - 1) / F::kTokens) * a.w_tiles;
      }
      sum += n[i];
    }
    int64_t upto = sum;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, upto, s);
      if (lane >= s) upto += v;
    }
    if (lane == 31) warp_sum[warp] = upto;
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto += warp_sum[w];
    upto -= sum;
#pragma unroll
    for (int i = 0; i < F::kPer; ++i) {
      upto += n[i];
      if (F::kPer * threadIdx.x + i < kMoeMaxExperts)
        ends[F::kPer * threadIdx.x + i] = static_cast<int>(min(upto, static_cast<int64_t>(a.max_units)));
    }
    __syncthreads();
  }
  const int units = ends[kMoeMaxExperts - 1];
  const uint32_t tmem = *tmem_slot;

  auto fail = [&]() {
    set_status(a.status, NVFP4_ERR_TIMEOUT);
    abort_flag = 1;
  };
  // A warp's lanes decide together: a wait that runs out in one of them ends all.
  const auto wait = [&](uint64_t* bar, uint32_t parity) {
    return __all_sync(0xffffffffu, mbar_wait_bounded(bar, parity, &abort_flag)) != 0;
  };
  // The same for a barrier that the other CTA of the pair arrives on.
  const auto wait_pair = [&](uint64_t* bar, uint32_t parity) {
    return __all_sync(0xffffffffu, mbar_wait_bounded_cluster(bar, parity, &abort_flag)) != 0;
  };
  // The peer's warp 2: takes a cluster; the unit that it begins with, -1 where none is left (asking again is not allowed).
  // False: the wait ran out.
  uint32_t answers = 0;  // the phase of answer_in
  const auto take = [&](int64_t* u) {
    if (elect_one()) {
      mbar_arrive_expect_tx(answer_in, 16);
      take_cluster(answer, answer_in);
    }
    __syncwarp();
    if (!wait(answer_in, answers)) return false;
    answers ^= 1u;
    const int taken = __shfl_sync(0xffffffffu, taken_cluster(answer), 0);
    fence_proxy_async_smem();  // read here, then written by the next answer
    *u = taken < 0 ? -1 : unit_of(taken);
    return true;
  };
  // Clusters start in any order: a pair whose own unit is not there takes others until one has a unit, and begins with that.
  // Here, before the roles: one token's gate_up and down 6.84 and 5.27 us, for 7.01 and 5.30 with a look at each unit in the
  // roles.  Without it, which leaves the others to start and end by themselves, 6.84 and 5.14, but 100 rows of 32768 choices
  // 27.9 and 38.6 for 10.8 and 16.6.
  if (first_unit >= units) {
    if (!leader && warp == 2) {
      int64_t u;
      do
        if (!take(&u)) {
          fail();
          u = -1;
        }
      while (u >= units);
      if (lane == 0)
#pragma unroll
        for (uint32_t r = 0; r < 2; ++r)
          asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(pair_address(const_cast<int*>(&late_unit), r)),
                       "r"(static_cast<int>(u))
                       : "memory");
      __syncwarp();
    }
    cluster_sync_all();
    if (late_unit >= 0) first_unit = late_unit;
  }
  // The next unit of the pair, to each of its warps by itself (n: its count of them).  False: there is none, or, with
  // *ok false, the wait ran out.
  auto next_unit = [&](Unit* t, int* n, bool* ok) {
    const int slot = *n % kQueue;
    *ok = wait_pair(&unit_full[slot], (*n / kQueue) & 1);
    if (!*ok) {
      fail();
      return false;
    }
    ++*n;
    *t = load_unit(&queue[slot]);
    const bool some = __all_sync(0xffffffffu, t->tokens != 0);  // all lanes have their load's answer
    if (lane == 0) {
      arrive_relaxed(pair_address(&unit_empty[slot], 1));
      if (leader && warp == 0) arrive_relaxed(pair_address(&unit_begun[slot], 1));
    }
    return some;
  };
  // Walks the pair's units, the first one found without the queue; body(unit) gives false where a wait ran out.
  auto walk_units = [&](auto&& body) {
    if (first_unit >= units) return true;
    Unit t = find_unit<F::kTokens>(first_unit, ends, expert_rows_s, lane);
    int n = 0;
    bool ok = true;
    do ok = body(t);
    while (ok && next_unit(&t, &n, &ok));
    return ok;
  };
  // A producer's walk; load(stage, kb, unit), in one lane, fills a stage once `free` says so.
  auto produce = [&](uint64_t* free, auto&& load) {
    const bool issuer = elect_one();
    int stage = 0;
    uint32_t phase = 0;
    bool skip = a.fault_skip_stage && first_unit == 0;
    const bool done = walk_units([&](const Unit& t) {
      for (int kb = 0; kb < kblocks; ++kb) {
        if (!wait(&free[stage], phase ^ 1u)) {
          fail();
          return false;
        }
        if (issuer && !skip) load(stage, kb, t);
        skip = false;
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
      return true;
    });
    if (!done) wait_for_copies();
  };

  if (warp == 0) {
    // -------------------------------------------------------------- codes ---
    produce(empty, [&](int stage, int kb, const Unit& t) {
      const int half = t.n() / 2;  // this CTA's tokens: `half` of them from rank * half
      constexpr int kMid = F::kSmall ? 32 : 64;
      const int box = half <= 16 ? 16 : half <= kMid ? kMid : 128;
      const CUtensorMap* map = half <= 16 ? &map_x16 : half <= kMid ? &map_x_mid : &map_x128;
      if (leader) mbar_arrive_expect_tx(&full[stage], 2 * (kWBytes + box * (kDepth / 2)));
      load_box(sW + stage * kWBytes, &map_w, &full[stage], kb * (kDepth / 2),
               t.expert * a.N + t.w_tile * kWRows + static_cast<int>(rank) * 128);
      load_box(sX + stage * F::kXBytes, map, &full[stage], kb * (kDepth / 2), t.row0 + static_cast<int>(rank) * half);
    });
  } else if (leader ? warp == 3 : warp == 1) {
    // ------------------------------------------------------- block scales ---
    // A CTA's own weight rows' and all tokens'.  8 rows of 256 bytes are the four atoms of a (row tile, k-block).
    // A stage's buffers are free once the copies have read them (`full`).
    const int tile_rows = a.K / 32;
    produce(full, [&](int stage, int kb, const Unit& t) {
      const bool two = !F::kSmall && t.n() > 128;
      if (leader) mbar_arrive_expect_tx(&scales_in[stage], 2 * (two ? 3 : 2) * kScaleTile);
      load_box(sWS + stage * kScaleTile, &map_w_scales, &scales_in[stage], 0,
               (t.expert * a.w_scale_tiles + t.w_tile * 2 + static_cast<int>(rank)) * tile_rows + kb * 8);
      uint8_t* dst = sXS + stage * F::kXScales;
      if (two)
        load_box3(dst, &map_x_scales2, &scales_in[stage], kb * 8, t.row0 / 128);
      else
        load_box(dst, &map_x_scales, &scales_in[stage], 0, t.row0 / 128 * tile_rows + kb * 8);
    });
  } else if (warp == 1) {
    // --------------------------------------------------------------- MMAs ---
    const bool issuer = elect_one();
    int stage = 0, local = 0;
    uint32_t phase = 0;
    const uint32_t utmem = __shfl_sync(0xffffffffu, tmem, 0);
    const uint64_t w_desc0 = tile_desc(smem_u32(sW)), x_desc0 = tile_desc(smem_u32(sX));
    bool ready = false;  // the next stage was seen full
    walk_units([&](const Unit& t) {
      const uint32_t idesc = kIdesc | static_cast<uint32_t>(t.n() >> 3) << 17 | (a.mx ? kUE8M0 : 0u);
      // A scale tile's columns are of 32 rows each: tiles of 64 tokens begin with its first or its third.
      const uint32_t x_col = F::kSmall && (t.row0 & 64) ? 2 : 0;
      if (!wait_pair(acc_empty, (local & 1) ^ 1u)) {
        fail();
        return false;
      }
      ++local;
      tc_fence_after();
      for (int kb = 0; kb < kblocks; ++kb) {
        if (!ready && !wait(&full[stage], phase)) {
          fail();
          return false;
        }
        tc_fence_after();
        const uint32_t ws = utmem + F::kSfCol + stage * F::kSfCols, xs = ws + 16;
        const uint64_t w_desc = w_desc0 + static_cast<uint32_t>(stage) * (kWBytes >> 4);
        const uint64_t x_desc = x_desc0 + static_cast<uint32_t>(stage) * (F::kXBytes >> 4);
        const int next = stage + 1 == kStages ? 0 : stage + 1;
        const uint32_t next_phase = next ? phase : phase ^ 1u;
        if (issuer) {
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            pair_mma(utmem, w_desc + 2 * kk, x_desc + 2 * kk, idesc, ws + kk * 4, xs + x_col + kk * 4 * F::kXTiles,
                     (kb | kk) != 0);
          pair_commit(&empty[stage], 0x3);
        }
        ready = __all_sync(0xffffffffu, mbar_test_wait(&full[next], next_phase)) != 0;
        stage = next;
        phase = next_phase;
      }
      if (issuer) pair_commit(acc_full, 0x3);
      return true;
    });
    if (issuer) pair_commit(drain, 0x1);
    mbar_wait_bounded(drain, 0, nullptr);
  } else if (warp == 2 && leader) {
    // -------------------------------------------------- scales into TMEM ---
    const bool issuer = elect_one();
    int stage = 0;
    uint32_t phase = 0;
    const uint32_t utmem = __shfl_sync(0xffffffffu, tmem, 0);
    const uint64_t ws_desc0 = atom_desc(smem_u32(sWS)), xs_desc0 = atom_desc(smem_u32(sXS));
    walk_units([&](const Unit& t) {
      for (int kb = 0; kb < kblocks; ++kb) {
        // The scales have landed, and the MMAs that read this TMEM slot are done.
        if (!wait(&scales_in[stage], phase) || !wait(&empty[stage], phase ^ 1u)) {
          fail();
          return false;
        }
        tc_fence_after();
        const uint32_t ws = utmem + F::kSfCol + stage * F::kSfCols, xs = ws + 16;
        const uint64_t ws_desc = ws_desc0 + static_cast<uint32_t>(stage) * (kScaleTile >> 4);
        const uint64_t xs_desc = xs_desc0 + static_cast<uint32_t>(stage) * (F::kXScales >> 4);
        if (issuer) {
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            pair_copy_scales(ws + kk * 4, ws_desc + kk * (512 >> 4));
            pair_copy_scales(xs + kk * 4 * F::kXTiles, xs_desc + kk * (512 >> 4));
            if (!F::kSmall && t.n() > 128) pair_copy_scales(xs + kk * 8 + 4, xs_desc + (kScaleTile + kk * 512) / 16);
          }
          pair_commit(&full[stage], 0x3);
        }
        if (++stage == kStages) { stage = 0; phase ^= 1u; }
      }
      return true;
    });
    if (issuer) pair_commit(drain_copies, 0x1);
    mbar_wait_bounded(drain_copies, 0, nullptr);
  } else if (warp == 2) {
    // ------------------------------------------------------ peer: the queue ---
    // Cluster c of `clusters` has the units c, c + clusters, ...  A pair asks for units only so far ahead that its loads
    // never wait for one, some 8 k-blocks: with more, the first pairs take them all (224 units on 76 pairs: 2 to 4 each).
    const int ahead = max(1, min(kQueue - 1, 8 / kblocks));
    const bool issuer = elect_one();
    int n = 0;
    bool ok = true;
    auto hand_out = [&](const Unit& t) {
      const int slot = n % kQueue;
      ok = ok && wait_pair(&unit_empty[slot], ((n / kQueue) & 1) ^ 1u);
      if (ok && issuer)
#pragma unroll
        for (uint32_t r = 0; r < 2; ++r) {
          expect_in_pair(&unit_full[slot], r, sizeof(Unit));
          send_16(&queue[slot], &unit_full[slot], r, make_int4(t.expert, t.w_tile, t.row0, t.tokens));
        }
      __syncwarp();
      const int old = ++n - ahead;
      if (old >= 0) ok = ok && wait_pair(&unit_begun[old % kQueue], (old / kQueue) & 1);
    };
    for (int64_t u = static_cast<int64_t>(first_unit) + clusters; first_unit < units;) {
      for (; ok && u < units; u += clusters) hand_out(find_unit<F::kTokens>(static_cast<int>(u), ends, expert_rows_s, lane));
      ok = ok && take(&u);
      if (ok && u < 0) hand_out(Unit{});
      if (!ok) fail();
      if (!ok || u < 0) break;
    }
  } else if (warp >= kEpi0) {
    // ----------------------------------------------------------- epilogue ---
    const int quarter = warp & 3, side = (warp - kEpi0) >> 2;
    const int meeting = 1 + ((warp - kEpi0) >> 1);  // two warps with the 32 outputs of an MXFP4 block
    uint8_t* buf_ptr = sEpi + (warp - kEpi0) * kEpiBytes;
    const uint32_t buf = smem_u32(buf_ptr);
    int local = 0;
    auto finish = [&](const Unit& t) {
      const float scale =
          a.g_a ? __fmul_rn(__ldg(a.g_a + static_cast<int64_t>(t.expert) * a.g_a_step), __ldg(a.g_w + t.expert)) : 1.0f;
      const float g_in = kMode == 1 ? __ldg(a.g_out + static_cast<int64_t>(t.expert) * a.g_out_step) : 1.0f;
      // Lane 0 waits and tells, so that the warp stays converged.
      int ok = 1;
      if (lane == 0) {
        ok = !abort_flag && mbar_wait_bounded(acc_full, local & 1, &abort_flag);
        if (!ok && !abort_flag) fail();
      }
      ok = __shfl_sync(0xffffffffu, ok, 0);
      if (kMode == 2) ok = both(meeting, ok != 0);  // the two warps go on or leave together
      if (!ok) return false;
      ++local;
      tc_fence_after();
      uint32_t lo[F::kChunks][16], hi[F::kChunks][16];
      const uint32_t taddr = tmem + (static_cast<uint32_t>(quarter * 32) << 16);
#pragma unroll
      for (int i = 0; i < F::kChunks; ++i) {
        const int token0 = 32 * (F::kSides * i + side);
        if (token0 < t.tokens) {
          tmem_ld_fragments(taddr + token0, lo[i]);
          tmem_ld_fragments(taddr + (16u << 16) + token0, hi[i]);
        }
      }
      tmem_ld_done();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_relaxed(leader_address(acc_empty));
      // The next unit's MMAs run while this warp computes and stores.
      const int n0 = t.w_tile * kWRows + static_cast<int>(rank) * 128 + quarter * 32;
      if constexpr (kMode == 0) {
#pragma unroll
        for (int i = 0; i < F::kChunks; ++i) {
          const int token0 = 32 * (F::kSides * i + side);
          if (token0 < t.tokens && n0 < a.N) store_rows(a, &map_out, t, lo[i], hi[i], token0, n0, scale, buf, lane);
        }
      } else if constexpr (kMode == 1) {
        const bool g_ok = g_in > 0.0f && g_in <= FLT_MAX;
        if (!g_ok && lane == 0) set_status(a.status, NVFP4_ERR_INVALID_ARG);
        const float g = g_ok ? g_in : 1.0f, six_g = __fmul_rn(6.0f, g);
#pragma unroll
        for (int i = 0; i < F::kChunks; ++i) {
          const int token0 = 32 * (F::kSides * i + side);
          if (token0 >= t.tokens) continue;
          swiglu_fragments(lo[i], hi[i], scale);
          const BlockScale b = block_scale(token_amax(lo[i], lane), g, six_g);
          const uint2 codes = token_codes(lo[i], b.mult, lane);
          store_codes(a, t, g_ok ? codes : make_uint2(0, 0), g_ok ? b.code : 0u, token0, n0 >> 1, lane);
        }
      } else {
        float* mine = reinterpret_cast<float*>(buf_ptr);
        const float* theirs = reinterpret_cast<const float*>(sEpi + ((warp - kEpi0) ^ 1) * kEpiBytes);
#pragma unroll
        for (int i = 0; i < F::kChunks; ++i) {
          const int token0 = 32 * (F::kSides * i + side);
          if (token0 >= t.tokens) continue;
          swiglu_fragments(lo[i], hi[i], scale);
          if (a.rotate) {
            // H_32 / sqrt(32) over the outputs: strides 1, 2, 4 across lanes, 8 in the thread, 16 across the two warps,
            // in this order, as hadamard32.
            float h[16];
#pragma unroll
            for (int v = 0; v < 16; ++v) h[v] = __uint_as_float(lo[i][v]);
#pragma unroll
            for (int s = 4; s < 32; s <<= 1)
#pragma unroll
              for (int v = 0; v < 16; ++v) {
                const float o = __shfl_xor_sync(0xffffffffu, h[v], s);
                h[v] = lane & s ? __fsub_rn(o, h[v]) : __fadd_rn(h[v], o);
              }
#pragma unroll
            for (int v = 0; v < 16; v += 4)
#pragma unroll
              for (int q = 0; q < 2; ++q) {
                const float x = h[v + q], y = h[v + q + 2];
                h[v + q] = __fadd_rn(x, y);
                h[v + q + 2] = __fsub_rn(x, y);
              }
#pragma unroll
            for (int v = 0; v < 16; ++v) mine[32 * v + lane] = h[v];
            meet(meeting);
#pragma unroll
            for (int v = 0; v < 16; ++v) {
              const float o = theirs[32 * v + lane];
              h[v] = __fmul_rn(quarter & 1 ? __fsub_rn(o, h[v]) : __fadd_rn(h[v], o), __uint_as_float(kInvSqrt32Bits));
              lo[i][v] = __float_as_uint(h[v]);
            }
            meet(meeting);
          }
          const float amax = token_amax(lo[i], lane);
          mine[lane] = amax;
          meet(meeting);
          const uint32_t code = mx_scale_code(fmaxf(amax, theirs[lane]));
          meet(meeting);
          store_codes(a, t, token_codes(lo[i], mx_inv_scale(code), lane), code, token0, n0 >> 1, lane);
        }
      }
      return true;
    };
    Unit t = {};
    int n = 0;
    bool ok = true, more = first_unit < units;
    if (more) t = find_unit<F::kTokens>(first_unit, ends, expert_rows_s, lane);
    while (more && finish(t)) {
      more = next_unit(&t, &n, &ok);
      if (kMode == 2 && !both(meeting, ok)) break;
    }
    if (kMode == 0 && lane == 0) bulk_wait_all();
  }

  tc_fence_before();
  cluster_sync_all();
  tc_fence_after();
  if (warp == 1) pair_tmem_free(tmem, F::kTmemCols);
}

// ------------------------------------------------------------------- host ---

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  });
  return fn;
}

bool encode(CUtensorMap* map, const uint8_t* base, uint32_t rank, const cuuint64_t* dims, const cuuint64_t* strides,
            const cuuint32_t* box, CUtensorMapSwizzle swizzle) {
  const auto enc = encoder();
  const cuuint32_t steps[3] = {1, 1, 1};
  return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, rank, const_cast<uint8_t*>(base), dims, strides, box, steps,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// [rows, K / 2] bytes, boxes of 128 bytes x box_rows.
bool codes_map(CUtensorMap* map, const uint8_t* base, int64_t rows, int64_t K, uint32_t box_rows) {
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(K / 2), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(K / 2)};
  const cuuint32_t box[2] = {kDepth / 2, box_rows};
  return encode(map, base, 2, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
// bf16 [rows, N], rows ldo apart, boxes of 32 x 32.
bool out_map(CUtensorMap* map, void* base, int64_t rows, int64_t N, int64_t ldo) {
  const auto enc = encoder();
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(N), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(ldo * 2)};
  const cuuint32_t box[2] = {32, 32}, steps[2] = {1, 1};
  return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, base, dims, strides, box, steps,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Block scales in the tensor core's order, `tiles` tiles of 128 rows, as rows of 256 bytes, K / 32 of them a tile: boxes of
// one (tile, k-block), or of two tiles.
bool scales_map(CUtensorMap* map, const uint8_t* base, int64_t tiles, int64_t K, bool two) {
  const cuuint64_t tile_rows = static_cast<cuuint64_t>(K / 32), n = static_cast<cuuint64_t>(tiles);
  const cuuint64_t dims[3] = {256, two ? tile_rows : tile_rows * n, n};
  const cuuint64_t strides[2] = {256, 256 * tile_rows};
  const cuuint32_t box[3] = {256, 8, 2};
  return encode(map, base, two ? 3 : 2, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_NONE);
}

// The shared-memory opt-in, once for each device.
template <class F>
bool opted_in() {
  static std::mutex mu;
  static std::map<int, bool> done;
  int d = 0;
  if (cudaGetDevice(&d) != cudaSuccess) return false;
  std::lock_guard<std::mutex> lock(mu);
  if (done[d]) return true;
  if (cudaFuncSetAttribute(grouped_kernel<F>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           static_cast<int>(F::kSmem)) != cudaSuccess) {
    cudaGetLastError();
    return false;
  }
  return done[d] = true;
}

template <class F>
nvfp4_status launch_form(const moe_plan* plan, GroupedArgs& a, cudaStream_t s) {
  constexpr int kTokens = F::kTokens;
  a.row_start = plan->row_start;
  a.rows = plan->rows;
  a.experts = plan->num_experts;
  a.max_rows = static_cast<int>(moe_rows_bound(plan->n_tokens, plan->top_k, plan->num_experts));
  a.w_tiles = (a.N + kWRows - 1) / kWRows;
  a.w_scale_tiles = (a.N + 127) / 128;
  const int64_t choices = plan->n_tokens * plan->top_k, used = choices < a.experts ? choices : a.experts;
  a.choices = static_cast<int>(choices);  // below moe_rows_bound
  const int64_t units = (choices + (kTokens - 1) * used) / kTokens * a.w_tiles;  // at most
  if (units >= (1ll << 30)) return NVFP4_ERR_SHAPE;
  a.max_units = static_cast<int>(units);
  // Clusters for about as many as there are, were half of the experts' last tiles none: one too many is asked for in
  // vain, one too few gives the first clusters two units.
  const int64_t about = (choices / kTokens + used / 2) * a.w_tiles, least = (F::kSmall ? 4ll : 2ll) * sm_count();
  const int64_t clusters = units < least ? units : about < least ? least : about < units ? about : units;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(F::kThreads, 1, 1);
  cfg.dynamicSmemBytes = F::kSmem;
  cfg.attrs = attr;
  if (!opted_in<F>()) return NVFP4_ERR_CUDA;
  CUtensorMap w, ws, x16, mid_x = {}, x128 = {}, xs, xs2 = {}, out = {};
  const int64_t R = a.max_rows, K = a.K;
  // No tile has more tokens than there are choices (expert_rows cuts to them): few need no map of the larger boxes.
  const bool mid = choices > 32, wide = !F::kSmall && choices > 128;
  if (!codes_map(&w, a.w_codes, static_cast<int64_t>(a.experts) * a.N, K, 128) ||
      !scales_map(&ws, a.w_scales, static_cast<int64_t>(a.experts) * a.w_scale_tiles, K, false) ||
      !codes_map(&x16, a.a_codes, R, K, 16) || (mid && !codes_map(&mid_x, a.a_codes, R, K, F::kSmall ? 32 : 64)) ||
      (wide && !codes_map(&x128, a.a_codes, R, K, 128)) || !scales_map(&xs, a.a_scales, R / 128, K, false) ||
      (wide && !scales_map(&xs2, a.a_scales, R / 128, K, true)) ||
      (F::kMode == 0 && !out_map(&out, a.out, R, a.N, a.ldo)))
    return NVFP4_ERR_CUDA;
  a.status = status_word_dev();
  a.fault_skip_stage = take_fault(NVFP4_FAULT_GEMM_SKIP_STAGE) ? 1 : 0;
  a.reversed = take_fault(NVFP4_FAULT_GROUPED_REVERSED) ? 1 : 0;
  cfg.gridDim = dim3(static_cast<uint32_t>(2 * clusters), 1, 1);
  cfg.stream = s;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, grouped_kernel<F>, w, ws, x16, mid_x, x128, xs, xs2, out, a) !=
      cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  return launch_status();
}

// Small tiles, two CTAs an SM, where an expert has few rows on average, idle experts counted: an average hides one expert of
// many rows, which then has tiles of 64.  With SwiGLU they are ahead at 96 and behind at 192, level at (47): the rule, 64,
// stops short of the crossing.  us, small against large, rows an expert in brackets:
//   SwiGLU to NVFP4  (0.1) 1 token, 2048 x 2048, 6.7 / 7.5; (4) 128 experts, 2048 x 1536, 22.7 / 23.3; (16) 16 experts,
//                    5120 x 4096, 28.1 / 28.5; (47) 64, 4096 x 2560, 57.5 / 57.1; (58) 40, 1536 x 2560, 15.7 / 17.0; (64) 64,
//                    2048 x 2048, 28.6 / 29.5; (96) 40, 1536 x 2560, 21.2 / 22.3; (192) the same, 30.4 / 28.7
//   SwiGLU to MXFP4  (5) 40 experts, 1536 x 2560, 13.8 / 14.9; (58) 16.9 / 18.0; (96) 22.7 / 23.7; (192) 33.2 / 31.0
//   bf16 rows        (5) 40 experts, 1280 x 1536, 8.1 / 8.7; (22) 11.3 / 11.5; (32) 16, 2048 x 5120, 18.4 / 17.8, 64,
//                    1024 x 2048, 16.3 / 16.5; (47) 64, 1280 x 4096, 35.3 / 33.4; (96) 40, 1280 x 1536, 15.2 / 14.2
template <int kMode>
nvfp4_status launch_grouped(const moe_plan* plan, GroupedArgs& a, cudaStream_t s) {
  const bool small = plan->n_tokens * plan->top_k <= (kMode == 0 ? 32 : 64) * static_cast<int64_t>(plan->num_experts);
  return small ? launch_form<Form<kMode, true>>(plan, a, s) : launch_form<Form<kMode, false>>(plan, a, s);
}

constexpr int64_t kMaxSide = 1ll << 20;  // N and K

// The operands' checks that all four calls share; g: whether there are tensor scales.  Without tokens the sorted rows are
// empty buffers, whose addresses may be null.
nvfp4_status check_operands(const moe_plan* plan, const GroupedArgs& a, int64_t N, int64_t K, bool g, int64_t n_step) {
  const nvfp4_status st = check_moe_plan(plan);
  if (st != NVFP4_OK) return st;
  if ((a.g_a_step != 0 && a.g_a_step != 1) || (a.g_out_step != 0 && a.g_out_step != 1)) return NVFP4_ERR_INVALID_ARG;
  if (N <= 0 || K <= 0 || N > kMaxSide || K > kMaxSide || K % 256 || N % n_step) return NVFP4_ERR_SHAPE;
  // Box coordinates, those of a last tile that reaches past the last expert too.
  if ((plan->num_experts * ((N + 127) / 128) + 2) * (K / 32) >= (1ll << 31) || plan->num_experts * N + 256 >= (1ll << 31) ||
      moe_rows_bound(plan->n_tokens, plan->top_k, plan->num_experts) / 128 * (K / 32) >= (1ll << 31))
    return NVFP4_ERR_SHAPE;
  if (plan->n_tokens == 0) return NVFP4_OK;
  if (!a.a_codes || !a.a_scales || !a.w_codes || !a.w_scales || (g && (!a.g_a || !a.g_w))) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(a.a_codes, 16) || !aligned(a.a_scales, 16) || !aligned(a.w_codes, 16) || !aligned(a.w_scales, 16) ||
      !aligned(a.g_a, 4) || !aligned(a.g_w, 4))
    return NVFP4_ERR_ALIGN;
  return NVFP4_OK;
}

nvfp4_status linear(const moe_plan* plan, GroupedArgs a, int64_t N, int64_t K, void* out, int64_t ldo, void* stream) {
  const nvfp4_status st = check_operands(plan, a, N, K, !a.mx, 16);
  if (st != NVFP4_OK) return st;
  if (ldo < N || ldo % 8) return NVFP4_ERR_SHAPE;
  if (plan->n_tokens == 0) return NVFP4_OK;
  if (!out) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(out, 16)) return NVFP4_ERR_ALIGN;
  a.out = static_cast<uint16_t*>(out);
  a.ldo = ldo;
  a.N = static_cast<int>(N);
  a.K = static_cast<int>(K);
  return launch_grouped<0>(plan, a, static_cast<cudaStream_t>(stream));
}

nvfp4_status swiglu(const moe_plan* plan, GroupedArgs a, int64_t I, int64_t K, uint8_t* codes, uint8_t* scales,
                    void* stream) {
  const nvfp4_status st = check_operands(plan, a, 2 * I, K, !a.mx, 256);
  if (st != NVFP4_OK) return st;
  if (plan->n_tokens == 0) return NVFP4_OK;
  if (!codes || !scales || (!a.mx && !a.g_out)) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(codes, 16) || !aligned(scales, 4) || !aligned(a.g_out, 4)) return NVFP4_ERR_ALIGN;
  a.q_codes = codes;
  a.q_scales = scales;
  a.N = static_cast<int>(2 * I);
  a.K = static_cast<int>(K);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  return a.mx ? launch_grouped<2>(plan, a, s) : launch_grouped<1>(plan, a, s);
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
  a.rotate = rotate != 0;
  return swiglu(plan, a, I, K, out_codes, out_scales, stream);
}
