// Indexing and clamping shared by the 8-bit cache's kernels.
#pragma once

#include "common.h"
#include "internal.h"

namespace tav2 {

constexpr int KVP = TAV2_KV_PAGE;

// Tokens of sequence s, within what its table can hold.
__device__ __forceinline__ int kv_len(const tav2_kv& c, int s) {
  const int most = c.max_blocks * KVP + KVP - 1, n = c.len[s];
  return n < 0 ? 0 : n > most ? most : n;
}

// (layer, page, head): index of a scale; times 64 D that of its codes.
__device__ __forceinline__ int64_t kv_unit(const tav2_kv& c, int layer, int page, int h) {
  return (int64_t(layer) * c.pages + page) * c.kv_heads + h;
}

// First element of sequence s's tail in a layer and head (either side).
__device__ __forceinline__ int64_t kv_tail(const tav2_kv& c, int layer, int s, int h) {
  return ((int64_t(layer) * c.num_seqs + s) * c.kv_heads + h) * KVP * c.head_dim;
}

// What kv_plan_kernel leaves for kv_compact_kernel: moves[0] pages go from[i] -> hole[i],
// moves[1] pages are used; to[page] is a moved page's new number.
struct KvPlan {
  int32_t* moves;
  int32_t* hole;
  int32_t* from;
  int32_t* to;
};

}  // namespace tav2
