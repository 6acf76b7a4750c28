// Attention of new tokens (one, a few, a chunk, a whole prompt) over the 4-bit
// cache that already holds them, contiguous or paged: scores optionally capped
// and biased by distance, keys limited by causality, window, prefix, document.
//
// This file chooses the kernel (extend_tiles.cu: 256 rows a tile; extend_rows.cu:
// up to 32; extend_decode.cu: up to 8) and the parts of the keys, and joins them.
#include "extend_attention.cuh"

namespace nvfp4 {
namespace {

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
  const uint32_t parts = a.part_blocks ? span_of(a, seq).parts : a.splits;
  if (parts == 1) return;  // written by its CTA
  for (uint32_t local = blockIdx.z * 8 + (threadIdx.x >> 5); local < rows; local += gridDim.z * 8) {
    const uint64_t rec = (static_cast<uint64_t>(blockIdx.x) * a.map.hkv + kvh) * a.splits * kRows + local;
    const float2* ml = a.ml_ws + rec;
    const float4* part = reinterpret_cast<const float4*>(a.o_ws + rec * kD) + lane;
    float2 mine = lane < parts ? ml[static_cast<uint64_t>(lane) * kRows] : make_float2(-INFINITY, 0.0f);
    float big = mine.x;
    for (uint32_t s = lane + 32; s < parts; s += 32) big = fmaxf(big, ml[static_cast<uint64_t>(s) * kRows].x);
#pragma unroll
    for (int sh = 16; sh; sh >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, sh));
    float sum = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (uint32_t s0 = 0; s0 < parts; s0 += 32) {
      if (s0) mine = s0 + lane < parts ? ml[static_cast<uint64_t>(s0 + lane) * kRows] : make_float2(-INFINITY, 0.0f);
      const float w = mine.x == -INFINITY ? 0.0f : ex2(mine.x - big);  // an empty part has no O
      for (uint32_t s = s0; s < min(s0 + 32, parts); s += 8) {
        float4 v[8];
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          f[k] = __shfl_sync(0xffffffffu, w, (s + k) & 31);
          if (s + k >= parts) f[k] = 0.0f;
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
    const float f = per_sum(sum, a.gv);
    const uint32_t r = t.row0 + local, tok = a.group.div(r), head = kvh * a.group.d + (r - tok * a.group.d);
    const uint64_t row = static_cast<uint64_t>(seq.first + tok) * a.hq + head;
    if (!out_in_bounds(a, row)) continue;
    reinterpret_cast<uint2*>(a.out + row * kD)[lane] =
        make_uint2(bf16x2_rn(o.x * f, o.y * f), bf16x2_rn(o.z * f, o.w * f));
  }
}

// ---- host ----------------------------------------------------------------

struct Plan {
  int rows;  // of a tile: kTileRows, or 8, 16, 24, 32
  int64_t tiles, tiles_per_seq;
  int64_t splits;       // parts of a tile's keys, at most
  int64_t part_blocks;  // 0: `splits` equal parts
  bool full;            // weights in two terms
};

// Buffers of up to this many keys a sequence take weights in two bf16 terms: among few
// keys the heavy ones may all hold a zero in a channel, and then what f16 loses of the
// light ones is the result.  (By the buffers, since the lengths are on the device: a
// short sequence in a wide table has f16's bound, 2^-29 of its largest weight.)
constexpr int64_t kFullContext = 512;

// Which kernel, the tiles (at most), and the parts that each tile's keys are cut into.
// By a sequence's rows per KV head: up to 8 the decode kernel (64 ragged sequences of up
// to 16384 keys 143 us; by 8-row tensor-core tiles 187), up to 32 the rows kernel (32 x 4
// drafted tokens on 4001 keys 77 us; by mma.sync 148, by 256-row tiles 159), else tiles.
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
  p.part_blocks = 0;
  double best = 0.0;
  if (p.rows != kTileRows) {
    // Parts of equal size, so that sequences of any lengths fill the GPU evenly:
    // the size with the least of rounds x (part + fixed cost), and half a part for
    // the end.  In blocks of 128 keys; the fixed cost (set-up, the record written
    // and joined) is worth about this many.
    const bool decode = p.rows == 8 && !p.full;
    const int64_t resident = sms * (decode ? 4 : 2), fixed = decode ? 3 : 6;
    for (int64_t part = 1;; part += part < 8 ? 1 : part / 4) {
      if (part > blocks) part = blocks;
      const int64_t parts = (blocks + part - 1) / part;
      const double cost = static_cast<double>((items * parts + resident - 1) / resident) * static_cast<double>(part + fixed) + 0.5 * static_cast<double>(part);
      if (parts <= 1024 && (best == 0.0 || cost < best)) {
        best = cost;
        p.part_blocks = part;
        p.splits = parts;
      }
      if (part >= blocks) break;
    }
    return p;
  }
  // As many parts as make the last wave of CTAs full, against what a part costs by
  // itself (its prologue; with several, its record written and read), in blocks
  // of 128 keys.
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

ExtendKernel combine_for(const Plan& p) {
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
  // So that the kernels' factors of it and of its inverse are normal numbers.  A cap below 1e-30 makes all weights
  // equal, one above 1e37 changes no score below 1e33: neither shows the difference.
  a.cap = options->logit_cap > 0.0f ? fminf(fmaxf(options->logit_cap, 1e-30f), 1e37f) : 0.0f;
  a.gv = cache->v_gscale;
  a.status = status_word_dev();
  a.fault_lose_stage = take_fault(NVFP4_FAULT_ATTN_SKIP_STAGE) ? 1 : 0;
  const Plan p = plan_for(a.map.batch, n_tokens, a.group.d, a.map.hkv, a.map.context, !q_start);
  const int64_t grid = p.tiles * a.map.hkv * p.splits;
  if (grid >= (1ll << 31)) return NVFP4_ERR_SHAPE;
  a.tiles = static_cast<uint32_t>(p.tiles);
  a.tiles_per_seq = static_cast<uint32_t>(p.tiles_per_seq);
  a.splits = static_cast<uint32_t>(p.splits);
  a.part_blocks = static_cast<uint32_t>(p.part_blocks);
  a.o_ws = static_cast<float*>(workspace);
  a.ml_ws = reinterpret_cast<float2*>(a.o_ws + static_cast<size_t>(grid) * p.rows * kD);
  const bool e1m2 = cache->kv_format == NVFP4_KV_E1M2;
  const bool by_tiles = p.rows == kTileRows;
  const ExtendLaunch l = by_tiles                     ? extend_tiles(e1m2, a.cap > 0.0f, a.slopes != nullptr, p.full)
                         : p.rows == 8 && !p.full ? extend_decode(e1m2, a.cap > 0.0f || a.slopes)
                                                  : extend_rows(p.rows, e1m2, a.cap > 0.0f, p.full);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  // Raising the limit is idempotent.
  if (cudaFuncSetAttribute(l.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(l.smem)) != cudaSuccess ||
      launch_pdl(l.kernel, dim3(static_cast<uint32_t>(grid)), dim3(l.threads), l.smem, s, a) != cudaSuccess)
    return NVFP4_ERR_CUDA;
  count_launches(1);
  if (p.splits > 1) {
    if (launch_pdl(combine_for(p), dim3(a.tiles, a.map.hkv, by_tiles ? 8 : (p.rows + 7) / 8), dim3(256), 0, s, a) != cudaSuccess)
      return NVFP4_ERR_CUDA;
    count_launches(1);
  }
  return launch_status();
}
