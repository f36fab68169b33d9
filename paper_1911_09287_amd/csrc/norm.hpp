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
  int pieces;                // split: waves a row, four of a block
  long piece;                // split: elements of one, a multiple of its tile
  int row_groups;            // split backward: blocks a chunk, over rows
  // inner > 1, forward and backward: threads of a block, positions of a thread,
  // lanes along positions and channels of a thread (0: read again for every use)
  int map_threads[2], map_vec[2], map_lanes[2], map_each[2];
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

// E vectors of N weights at from, from + step, ... of M, as fp32 (`one`: without
// weights); w holds fp32 (wide) or the activations' type.  All loads are in flight
// before the first is waited for.
template <typename T, int N, int E>
__device__ __forceinline__ void load_weights(const void* w, bool wide, long from, long step, long M, float one,
                                             float (&out)[E][N]) {
  if (!w) {
#pragma unroll
    for (int k = 0; k < E; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) out[k][j] = one;
  } else if (wide) {
    Held<float, N> r[E];
#pragma unroll
    for (int k = 0; k < E; ++k) r[k].load(static_cast<const float*>(w) + from + k * step, M - from - k * step);
#pragma unroll
    for (int k = 0; k < E; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) out[k][j] = r[k][j];
  } else {
    Held<T, N> r[E];
#pragma unroll
    for (int k = 0; k < E; ++k) r[k].load(static_cast<const T*>(w) + from + k * step, M - from - k * step);
#pragma unroll
    for (int k = 0; k < E; ++k) {
      r[k].refresh();
#pragma unroll
      for (int j = 0; j < N; ++j) out[k][j] = r[k][j];
    }
  }
}

// Backward, every operation rounded by itself: of one value u and its mean are then the
// same, and the gradient is 0 and not what a fused multiply-add would leave of u's
// rounding, times 1 / sqrt(eps).  (Of several equal u the sum and the reciprocal of
// their number round, so that their mean may differ from u by a few units of its last
// place and a row of equal values have that times 1 / sqrt(eps) for a gradient.)
__device__ __forceinline__ void add_sums(float u, float h, float& s0, float& s1) {
#pragma clang fp contract(off)
  s0 += u;
  s1 += u * h;
}
__device__ __forceinline__ float grad_of(float u, float c1, float h, float c2, float rstd) {
#pragma clang fp contract(off)
  return rstd * ((u - c1) - h * c2);
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
