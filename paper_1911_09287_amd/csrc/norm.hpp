// Layer norm: plan and launchers (norm.hip: plan and dispatch; norm_rows.hip:
// inner = 1; norm_maps.hip: inner > 1).
#pragma once

#include "ops.hpp"

// How rows (inner = 1) are cut.  A row's vectors of 16 bytes lie `each` a thread on
// `threads` lanes of a wave (a power of two) or, with block, on a block of so many.
struct bl_norm_rows {
  bool block;
  int threads, each;
};

struct bl_norm_plan_s {
  bl_norm_desc_t d;
  bl_norm_rows fwd, bwd;     // inner = 1, not split
  bool fwd_split, bwd_split; // inner = 1: each row by several blocks, in two launches
  int chunks;                // split: blocks a row
  long chunk;                // split: elements of one, a multiple of its tile
  int row_groups;            // split backward: blocks a chunk, over rows
  int map_threads[2];        // inner > 1, forward and backward: threads of a block,
  int map_vec[2];            //   positions of a thread, lanes along positions and
  int map_lanes[2];          //   channels of a thread (0: the channels are read again
  int map_each[2];           //   for every use)
  int parts;                 // backward: partial sums of dw and db, [parts][2][size]
  size_t off_part, off_sums, bytes;
};

namespace blc {

constexpr long kMostBlocks = 1L << 24;  // of 256 threads: a launch has fewer than 2^32
constexpr int kNormThreads = 256;  // of a block, where nothing else is said

struct NormPtrs {
  const void *x, *dy, *w, *b;
  void *y, *dx, *dw, *db;
  float* stats;
  float *part, *sums;  // workspace
};

// n weights from index i on as fp32 (`one`: without weights), fp32 or of the activations' type.
template <typename T, int N>
__device__ __forceinline__ void load_weights(const void* w, bool wide, long i, long n, float one, float (&out)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) out[j] = one;
  if (!w) return;
  if (wide) {
    const Pack<float, N> p = load_part<float, N>(static_cast<const float*>(w) + i, n, 0.f);
#pragma unroll
    for (int j = 0; j < N; ++j) out[j] = p.v[j];
  } else {
    const Pack<T, N> p = load_part<T, N>(static_cast<const T*>(w) + i, n, (T)0.f);
#pragma unroll
    for (int j = 0; j < N; ++j) out[j] = to_f32(p.v[j]);
  }
}

bl_status_t norm_rows_forward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s);
bl_status_t norm_rows_backward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s);
bl_status_t norm_maps_forward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s);
bl_status_t norm_maps_backward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s);
// dw and db from their partial sums (parts = 0: zeros).
bl_status_t norm_sum_parts(const bl_norm_plan_s* p, const NormPtrs& a, int parts, hipStream_t s);
// How a plan's calls are cut, and the workspace they need.
bl_status_t norm_rows_plan(bl_norm_plan_s* p);
bl_status_t norm_maps_plan(bl_norm_plan_s* p);

}  // namespace blc
