// Group norm with an activation: plan, arguments and what both layouts share (gnorm.hip:
// plan, dispatch and the sums that need no values; gnorm_last.hip, gnorm_first.hip: the layouts).
#pragma once

#include "ops.hpp"

struct bl_group_norm_plan_s {
  bl_group_norm_desc_t d;
  long each;       // channels of a group
  int vec;         // channels last: values of an access, a divisor of channels
  int lanes;       // channels last: accesses of a site that a block takes; first: lanes of a channel's sites
  int tiles;       // channels last: blocks along channels
  long chunk;      // sites of a block
  int chunks;      // of them
  bool joins[2];   // channels last, forward and backward: the blocks that apply join the parts themselves
  // a block keeps whole groups of a sample in registers (threads 0: no block can)
  int whole_threads[2], whole_each[2];  // forward and backward: threads, accesses of one
  int whole_lanes;  // channels last: accesses of a site (`tile` channels); first: lanes of a channel
  int whole_tiles;  // channels last: blocks of a sample
  long slab, slabs;  // samples whose sums are added at a time, and such parts (0: all at once)
  size_t off_part, off_sums, off_own, off_slabs, bytes;
};

namespace blc {

struct GroupNormArgs {
  const void *x, *dy, *w, *b;
  void *y, *dx, *dw, *db;
  float* stats;  // [2][batch][groups] mean, rstd
  float* part;   // [batch][chunks][channels][2]: forward mean and squares, backward sums of dz and dz h
  float* sums;   // backward [batch][groups][2]: means of u and of u h
  float* own;    // backward [own_rows][channels][2]: part, summed over a sample (or not)
  long own_rows;
  float* slabs;  // backward [slabs][channels][2]: own, summed over a slab's samples
  long batch, sites, channels, groups, each;
  long x_stride, y_stride;
  long chunk;
  int chunks, lanes, tiles;
  bool wide;     // w, b, dw and db in fp32
  float eps;
};

// z of the definition.  Both directions take it from here, so that the backward call
// finds max(z, 0) where the forward call left it.
__device__ __forceinline__ float norm_z(float x, float mean, float rstd, float w, float b) {
  return fmaf((x - mean) * rstd, w, b);
}
// q = 1 / (1 + exp(-z)) and q (1 - q), its slope, of z that comes from values of type T.  What rounds in z log2(e) moves the
// exponential by |z| units, which z far below 0 would keep as a relative error: fp32 takes the corrected
// one.  Of 16 bits a result of 2^-9 or 2^-11 has no sight of it (88 units are 2^-17), and there the power of two and
// the reciprocal alone do, an ulp each.  (Instructions bound 16-bit passes: 128 x 3136 x 64 bf16 takes 36 us by the
// library's exponential and division, which are 30 of 45 a value, against 22.)
template <typename T>
__device__ __forceinline__ void norm_logistic(float z, float& q, float& slope) {
  if constexpr (sizeof(T) == 4) {
    float rest;
    logistic_of(z, q, rest, slope);
  } else {
    q = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -0x1.715476p+0f));
    slope = fmaf(-q, q, q);
  }
}
template <int ACT, typename T>
__device__ __forceinline__ float act_of(float z) {
  if (ACT == BL_ACT_RELU) return z > 0.f ? z : z != z ? z : 0.f;
  if (ACT == BL_ACT_SILU) {
    float q, slope;
    norm_logistic<T>(z, q, slope);
    return z * q;
  }
  return z;
}
// dy act'(z)
template <int ACT, typename T>
__device__ __forceinline__ float act_grad(float z, float dy) {
  if (ACT == BL_ACT_RELU) return z > 0.f ? dy : z != z ? z : 0.f;
  if (ACT == BL_ACT_SILU) {
    float q, slope;
    norm_logistic<T>(z, q, slope);
    return dy * fmaf(z, slope, q);
  }
  return dy;
}

// dx.  Every operation rounds by itself (as in the groups' means): of a group of one
// value u is its mean, and the gradient is 0 and not a rounding of u times rstd.
__device__ __forceinline__ float norm_grad(float dz, float w, float c1, float h, float c2, float rstd) {
#pragma clang fp contract(off)
  const float u = dz * w;
  return rstd * ((u - c1) - h * c2);
}

// A weight at c (NULL: `one`).
template <typename T>
__device__ __forceinline__ float weight_at(const void* w, bool wide, long c, float one) {
  return !w ? one : wide ? static_cast<const float*>(w)[c] : to_f32(static_cast<const T*>(w)[c]);
}

constexpr int kMostThreads = 512;  // of a block that keeps whole groups: 256 registers a thread

// Sum over a block of up to 16 waves, in each thread; red: 16 values that nobody else uses.
__device__ __forceinline__ float block_sum(float x, float* red) {
  x = wave_sum(x);
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = x;
  __syncthreads();
  x = 0.f;
  for (unsigned w = 0; w < blockDim.x / kWave; ++w) x += red[w];
  return x;
}

// go(E) for the least of 1, 2, 4 and 8 that is at least `each`.
template <typename Go>
void with_each(int each, Go&& go) {
  if (each <= 1) go(std::integral_constant<int, 1>());
  else if (each <= 2) go(std::integral_constant<int, 2>());
  else if (each <= 4) go(std::integral_constant<int, 4>());
  else go(std::integral_constant<int, 8>());
}
constexpr long kMostEach = 8;

// Mean and sum of squares about it, of values that come in tiles: each tile's own are
// taken in registers and joined (Chan, Golub and LeVeque, "Updating formulae and a
// pairwise algorithm for computing sample variances", 1979), so that no square of a
// value far from 0 is summed.
struct Moments {
  float n, mean, m2;
};
__device__ __forceinline__ void moments_join(Moments& a, const Moments& b) {
  // (joined to nothing b stays as it is: a group of one value is its own mean)
  const float n = a.n + b.n, d = b.mean - a.mean, share = a.n == 0.f ? 1.f : b.n * __builtin_amdgcn_rcpf(n);
  a.mean = fmaf(d, share, a.mean);
  a.m2 += fmaf(d * d, a.n * share, b.m2);
  a.n = n;
}

// Parts of a sample that blocks which apply join, and of a group.  3 x 605 x 40 fp32 forward (160
// parts) takes 14.2 us so and 17.6 with a launch that joins, 128 x 3136 x 64 bf16 (256) 34.8 and
// 37.4; but 32 x 3136 x 256 (4096, which it was tried with) 41.1 and 38.4, 100 x 1024 x 50 (650) 22.4
// and 20.1.  Backward the weights' gradients are then sums over all samples' chunks, if a thread has no more
// of these than kMostOwn: 63 each of 182 x 7250 x 5 fp32 28.1 us and 31.9, of 600 x 2600 x 8 (38) 55.7 and 59.1.
constexpr long kMostJoined = 512, kMostOfGroup = 64;
// Rows of samples' sums that a thread adds: of more, slabs are cut, in which it has two trees of 16 at least, and
// 256 of them at most (64 of a thread that adds them).  Backward, bf16: 600 x 1 x 1024 23.7 us in slabs, 24.7 in one
// launch, 4000 x 1 x 64 20.1 and 65, 65536 x 1 x 64 139 and 855.
constexpr long kMostOwn = 128, kLeastOwn = 32, kMostSlabs = 256;

bl_status_t gnorm_last_forward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s);
bl_status_t gnorm_last_backward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s);
bl_status_t gnorm_first_forward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s);
bl_status_t gnorm_first_backward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s);
// The fewest threads of a block that keeps all with at most eight accesses each, and more while
// that leaves them over four and fewer; none (0) where it cannot.  each(threads): accesses.
template <typename Each>
void gnorm_whole_threads(Each&& each, int& threads, int& found) {
  threads = 0;
  int n = kWave;
  while (n <= kMostThreads && each(n) > kMostEach) n *= 2;
  if (n > kMostThreads) return;
  while (n < kMostThreads && each(n) > 4 && each(2 * n) < each(n)) n *= 2;
  threads = n;
  found = (int)each(n);
}
// How a plan's blocks keep whole groups, if they can.
void gnorm_last_whole(bl_group_norm_plan_s* p);
void gnorm_first_whole(bl_group_norm_plan_s* p);
// Statistics from the parts; backward: means over groups and sums over samples from theirs.
bl_status_t gnorm_join_forward(const GroupNormArgs& a, hipStream_t s);
bl_status_t gnorm_join_backward(const GroupNormArgs& a, int dtype, hipStream_t s);
// dw and db from the samples' sums (batch = 0: zeros); as a launch of its own, or by the blocks
// of another one past its own, of kThreads threads.
//
// Many samples are cut into slabs, whose sums a launch before adds (gnorm_slabs), so that neither the time
// nor the rounding grows with their number: a thread takes every `slices`th row, sixteen at a time whose loads
// are in flight together and whose sum is a tree, and the slices are joined in halves.  (One value in 20000
// rows is off by up to 2 half ulps so; added one after another in four slices by 800.)
constexpr int kRowsAhead = 16;
// Channels that a block takes: a power of two, so that few leave more slices of rows.
__host__ __device__ inline int gnorm_rows_cols(long channels) {
  int cols = kWave;
  while (cols > 1 && cols / 2 >= channels) cols /= 2;
  return cols;
}
// Sums of the pairs at rows first, first + step, ... below end, `stride` apart: of AHEAD rows, of sixteen of those
// and of these.
template <int AHEAD>
__device__ __forceinline__ void gnorm_pairs_ahead(const float* at, long stride, long first, long end, long step, float (&s)[2]) {
  s[0] = s[1] = 0.f;
  float few[2] = {};
  int turn = 0;
  for (long n = first; n < end; n += AHEAD * step) {
    float v[2][AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {  // (the last row again, and not counted)
      const Pack<float, 2> got = load_pack<float, 2>(at + min(n + k * step, end - 1) * stride);
      v[0][k] = got.v[0], v[1][k] = got.v[1];
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) v[j][k] = n + k * step < end ? v[j][k] : 0.f;
#pragma unroll
      for (int half = AHEAD / 2; half; half /= 2)
#pragma unroll
        for (int k = 0; k < half; ++k) v[j][k] += v[j][k + half];
      few[j] += v[j][0];
    }
    if (++turn % kRowsAhead == 0) s[0] += few[0], s[1] += few[1], few[0] = few[1] = 0.f;
  }
  s[0] += few[0];
  s[1] += few[1];
}
// (where a thread has a row or up to four, sixteen loads would be most of a launch that joins them: 4 x 270 x 360
// fp16 backward 21.1 us, so 19.3; 1 x 1723 x 41 channels first 31.3 and 27.8)
__device__ __forceinline__ void gnorm_pairs_sum(const float* at, long stride, long first, long end, long step, long rows,
                                                float (&s)[2]) {
  if (rows <= step) gnorm_pairs_ahead<1>(at, stride, first, end, step, s);
  else if (rows <= 4 * step) gnorm_pairs_ahead<4>(at, stride, first, end, step, s);
  else gnorm_pairs_ahead<kRowsAhead>(at, stride, first, end, step, s);
}
// Sums over rows [from, to) of the pairs of this block's channels: put(c, first, second), a thread a channel.
template <typename Put>
__device__ __forceinline__ void gnorm_rows_sum(const float* own, long channels, long from, long to, unsigned block, Put&& put) {
  __shared__ float red[2][kThreads / kWave][kWave];
  const int cols = gnorm_rows_cols(channels);
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int col = threadIdx.x % cols, slice = threadIdx.x / cols, slices = kThreads / cols;
  const long c = (long)block * kWave + col, at = min(c, channels - 1);
  float s[2];
  gnorm_pairs_sum(own + at * 2, channels * 2, from + slice, to, slices, to - from, s);
  for (int d = cols; d < kWave; d *= 2) s[0] += __shfl_xor(s[0], d), s[1] += __shfl_xor(s[1], d);
  red[0][wave][lane] = s[0];
  red[1][wave][lane] = s[1];
  __syncthreads();
  if (slice || c >= channels) return;
#pragma unroll
  for (int j = 0; j < 2; ++j) s[j] = (red[j][0][col] + red[j][1][col]) + (red[j][2][col] + red[j][3][col]);
  static_assert(kThreads == 4 * kWave, "the waves above");
  put(c, s[0], s[1]);
}
template <typename T>
__device__ __forceinline__ void gnorm_weights_block(const GroupNormArgs& a, unsigned block) {
  gnorm_rows_sum(a.own, a.channels, 0, a.own_rows, block, [&](long c, float db, float dw) {
    if (a.dw) {
      if (a.wide) static_cast<float*>(a.dw)[c] = dw;
      else static_cast<T*>(a.dw)[c] = (T)dw;
    }
    if (a.db) {
      if (a.wide) static_cast<float*>(a.db)[c] = db;
      else static_cast<T*>(a.db)[c] = (T)db;
    }
  });
}
inline unsigned gnorm_weights_blocks(const GroupNormArgs& a) {
  return a.dw || a.db ? (unsigned)((a.channels + kWave - 1) / kWave) : 0;
}
bl_status_t gnorm_weights(const GroupNormArgs& a, int dtype, hipStream_t s);
// Where a plan's samples are many: the sums of its slabs, which are a.own's rows from then on.
bl_status_t gnorm_slabs(const bl_group_norm_plan_s* p, GroupNormArgs& a, hipStream_t s);

// go(act) as a constant.
template <typename Go>
void with_act(int act, Go&& go) {
  if (act == BL_ACT_RELU) go(std::integral_constant<int, BL_ACT_RELU>());
  else if (act == BL_ACT_SILU) go(std::integral_constant<int, BL_ACT_SILU>());
  else go(std::integral_constant<int, BL_ACT_NONE>());
}

}  // namespace blc
