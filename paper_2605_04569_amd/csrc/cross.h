// Declarations shared by the cross attention kernels (cross_fwd.hip, cross_bwd.hip, cross_f32.hip) and their host side.
#pragma once

#include "attn_mfma.h"

namespace isa {

constexpr float LOWEST = -3.402823466e38f;    // the running maximum before the first key: no finite score is below it

// What the kernels get of an isa_cross_problem.  The query heads that share a key head are one sequence of `rows` = group * S_q rows:
// row r of key head hk is query r % S_q of head hk * group + r / S_q.
struct CrossArgs {
  const void *q, *k, *v;
  void* out;
  float* lse;
  const int* kv_len;
  const uint8_t* mask;
  long long mask_stride;
  int B, H, Hkv, group, Sq, Sk;
  isa_strides sq, sk, sv, so, sdo, sdq, sdk, sdv;
  float scale, cscale;              // factor of the scores; times log2(e)
  int rows;
  int items;                        // work items of a (batch item, key head): forward and dq: row tiles
  int chunk;                        // k_cross_dq: row tiles of an item
  int parts;                        // every item runs as this many workgroups, each over its share of the keys (dk, dv: of the queries)
  long long total;                  // work items * parts of all (batch item, key head)s
  // partial results of the parts: sums before normalisation [item][part][rows of a tile][D] and, per row, {maximum, sum of the weights
  // as multiplied, their sum before they were rounded, 1 if the part had a valid key}; bf16 dq: sums of dS' k and of P k [item][part][row][2][D], {sum of dS', ..}
  float* part_o;
  float4* part_ml;
  // backward
  const void* d_out;
  const void* fwd_out;
  void *dq, *dk, *dv;
  const float* fwd_lse;
  float* side;                      // per (batch item, head) and 64 queries: 64 minus-log-sum-exps (log2), then 64 minus-deltas
  int side_tiles;                   // ceil(S_q / 64)
};

// The keys of batch item b that are valid by their number
__device__ __forceinline__ int key_count(const CrossArgs& a, int b) {
  return a.kv_len ? min(max(a.kv_len[b], 0), a.Sk) : a.Sk;
}

// The work item of a workgroup.  Workgroup ids go round-robin over the 8 XCDs: each XCD takes one eighth of the items in their
// order (all items of a key head one after the other), so that the workgroups that run together on it read the same keys.
__device__ __forceinline__ bool cross_item(const CrossArgs& a, uint32_t& item) {
  const uint32_t per = gridDim.x * gridDim.y / N_XCD, id = blockIdx.y * gridDim.x + blockIdx.x;
  item = (id & 7) * per + (id >> 3);
  return item < (uint32_t)a.total;
}
// A launch dimension stays below 2^32 threads: 2^23 workgroups of 256 in x, the others in y (2^30 fp32 rows are 2^24 workgroups).
constexpr long long GRID_X = 1ll << 23;
inline dim3 cross_grid(long long total) {
  const long long y = (total + GRID_X - 1) / GRID_X, x = ((total + y - 1) / y + N_XCD - 1) / N_XCD * N_XCD;
  return dim3((unsigned)x, (unsigned)y);
}

// How a call is cut.  Chosen from the problem alone, so that the workspace can be sized by it.
struct CrossPlan {
  bool narrow;                      // 16 rows or fewer, the waves of a workgroup share the keys
  int tile_rows;
  int items, parts;
  size_t part_rows;                 // rows of partial results
};
CrossPlan cross_forward_plan(const isa_cross_problem& p);
bool cross_states_streamed(const isa_cross_problem& p);      // narrow: keys and values are loaded past the caches
struct CrossBackwardPlan {
  int dq_rows, dq_items, dq_parts;  // query rows of a workgroup
  int kv_rows, kv_items, kv_parts;  // keys of a workgroup
  int side_tiles;
  // the workspace: side, the parts' sums (of dq, then, after these have been added up, of dk and dv), the row sums of the parts of dq
  size_t side_bytes, part_bytes, ml_bytes;
};
CrossBackwardPlan cross_backward_plan(const isa_cross_problem& p);

hipError_t launch_cross_forward(CrossArgs a, const isa_cross_problem& p, hipStream_t st);
hipError_t launch_cross_backward(CrossArgs a, const isa_cross_problem& p, hipStream_t st);
hipError_t launch_cross_forward_f32(const CrossArgs& a, int D, hipStream_t st);
hipError_t launch_cross_dq(const CrossArgs& a, int D, hipStream_t st);
hipError_t launch_cross_dkv(const CrossArgs& a, int D, hipStream_t st);
hipError_t launch_cross_dq_f32(const CrossArgs& a, int D, hipStream_t st);
hipError_t launch_cross_dkv_f32(const CrossArgs& a, int D, hipStream_t st);

}  // namespace isa
