// A mixture-of-experts layer's plan as the kernels see it: which row of the
// sorted buffers each token's choice of an expert has.
#pragma once

#include "common.cuh"

namespace nvfp4 {

constexpr int kMoeMaxExperts = 1024;
constexpr int kMoeMaxTopK = 32;
constexpr int kMoeRowTile = 128;  // an expert's first row: the scale tiles of the tensor core's operands

// Rows of the sorted buffers: every expert with rows leaves at most 127 behind its last one.
inline int64_t moe_rows_bound(int64_t n_tokens, int32_t top_k, int32_t num_experts) {
  const int64_t pairs = n_tokens * top_k;
  const int64_t used = pairs < num_experts ? pairs : num_experts;
  return (pairs + (kMoeRowTile - 1) * used) / kMoeRowTile * kMoeRowTile;
}

inline nvfp4_status check_moe_sizes(int64_t n_tokens, int32_t top_k, int32_t num_experts) {
  if (n_tokens < 0 || top_k < 1 || top_k > kMoeMaxTopK || num_experts < 1 || num_experts > kMoeMaxExperts)
    return NVFP4_ERR_SHAPE;
  if (n_tokens >= (1ll << 31) || moe_rows_bound(n_tokens, top_k, num_experts) >= (1ll << 31)) return NVFP4_ERR_SHAPE;
  return NVFP4_OK;
}

inline nvfp4_status check_moe_plan(const moe_plan* p) {
  if (!p) return NVFP4_ERR_INVALID_ARG;
  const nvfp4_status st = check_moe_sizes(p->n_tokens, p->top_k, p->num_experts);
  if (st != NVFP4_OK) return st;
  if (!p->row_start || !p->rows || (!p->row_of && p->n_tokens)) return NVFP4_ERR_INVALID_ARG;
  if (!aligned(p->row_start, 4) || !aligned(p->rows, 4) || !aligned(p->row_of, 4)) return NVFP4_ERR_ALIGN;
  return NVFP4_OK;
}

// An expert's rows in the sorted buffers, cut to what the buffers hold and to the tokens' choices whatever the plan says:
// the host goes by these two alone where it decides what a launch can need.
struct ExpertRows {
  int first, n;
};
__device__ __forceinline__ ExpertRows expert_rows(const int32_t* row_start, const int32_t* rows, int e, int max_rows,
                                                  int choices) {
  ExpertRows r;
  r.first = __ldg(row_start + e);
  r.n = __ldg(rows + e);
  if (r.first < 0 || r.first > max_rows || (r.first & (kMoeRowTile - 1))) r.first = r.n = 0;
  r.n = max(0, min(min(r.n, choices), max_rows - r.first));
  return r;
}

}  // namespace nvfp4
