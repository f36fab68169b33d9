// Layer norm over the channels at each position (inner > 1): x [outer][size][inner].
//
// Positions lie on lanes, up to 8 bytes of them on one, so that a channel's
// positions are read as lines of 128 bytes; the channels of a position lie on the other
// lanes and waves of a block and, `EACH` of them, in a thread's registers.  So
// every value is read once and written once, and sums over the channels cross the
// lanes by shuffles and the waves by way of LDS.  Backward, a thread keeps the
// sums of its channels' dw and db over all tiles of its block.  Bound by HBM: 64 maps
// of 256 channels and 512 positions, fp32, forward 12 us, 5.6 TB/s, backward 23 us, 4.4
// TB/s, while the tensors lie in the 256 MB cache; from memory 19 us, 3.5 TB/s, and 24
// us, 4.2 TB/s; and 4 us for the last sum over blocks.  More than 512 channels in fp32
// leave room for one block a compute unit (1024: forward 61 us at four times the size,
// 4.4 TB/s, backward 130 us, 3.1 TB/s); backward of 257 to 1024 channels in 16 bits is short
// of two or three registers a lane.
#include <algorithm>

#include "norm.hpp"

namespace blc {
namespace {

constexpr int kMostThreads = 1024;
constexpr int kMostWaves = kMostThreads / kWave;

// This thread's place in a block's tile of positions: outer slice and the first of
// its VEC positions (which divide inner), and whether there are any.
struct Place {
  long outer, at;
  bool there;
};
template <int VEC, int LANES>
__device__ __forceinline__ Place place_of(long tile, const bl_norm_desc_t& d, unsigned per_slice) {
  const unsigned q = (unsigned)tile * LANES + threadIdx.x % LANES;  // of all vectors of positions
  const unsigned o = q / per_slice;
  return Place{(long)o, (long)(q - o * per_slice) * VEC, o < (unsigned long long)d.outer};
}
// Bytes from the tile's first slice (which the block shares) to this thread's
// first value; maps_shape() sees to it that they fit 32 bits.
template <typename T, int LANES>
__device__ __forceinline__ unsigned offset_of(const Place& p, long first, long stride, long inner) {
  return p.there ? (unsigned)(((p.outer - first) * stride + p.at + threadIdx.x / LANES * inner) * (long)sizeof(T)) : 0u;
}
template <typename T, int N>
__device__ __forceinline__ void store_at(T* p, unsigned bytes, bool there, const Pack<T, N>& v) {
  if (there) store_pack<T, N>(at_bytes(p, bytes), v);
}

// Weights into LDS, w[0 ... size), `one` without them; the caller synchronises.
template <typename T>
__device__ __forceinline__ void stage_weights(const void* w, bool wide, int size, float one, float* out) {
  for (int c = threadIdx.x; c < size; c += blockDim.x)
    out[c] = !w ? one : wide ? static_cast<const float*>(w)[c] : to_f32(static_cast<const T*>(w)[c]);
}

// Sum over the channels: over the lanes that hold the same positions, then the waves.
template <int N, int LANES, int THREADS>
__device__ __forceinline__ void channel_sum(float (&x)[N], float (*red)[LANES * N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (LANES == 16) x[j] = add16(x[j]);
    if (LANES <= 32) x[j] = add32(x[j]);
  }
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % LANES, waves = THREADS / kWave;
  if ((int)(threadIdx.x % kWave) < LANES)
#pragma unroll
    for (int j = 0; j < N; ++j) red[wave][lane * N + j] = x[j];
  __syncthreads();
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = 0.f;
#pragma unroll 4
  for (int w = 0; w < waves; ++w)
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] += red[w][lane * N + j];
}

template <typename T, int VEC, int LANES, int EACH, int THREADS>
__global__ __launch_bounds__(THREADS) void k_maps_fwd(NormPtrs a, bl_norm_desc_t d, unsigned per_slice, long tiles) {
  constexpr int groups = THREADS / LANES;
  __shared__ float red[2][THREADS / kWave][LANES * VEC];
  __shared__ float w[EACH * groups], b[EACH * groups];
  const int group = threadIdx.x / LANES, size = (int)d.size;
  const long sites = d.outer * d.inner, step = groups * d.inner;
  stage_weights<T>(a.w, d.wdtype == BL_F32, size, 1.f, w);  // (the sums' barriers lie before their use)
  stage_weights<T>(a.b, d.wdtype == BL_F32, size, 0.f, b);
  for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const Place p = place_of<VEC, LANES>(tile, d, per_slice);
    const long first = (unsigned)tile * LANES / per_slice;
    const T* x = static_cast<const T*>(a.x) + first * d.x_stride;
    T* y = static_cast<T*>(a.y) + first * d.y_stride;
    const unsigned from = offset_of<T, LANES>(p, first, d.x_stride, d.inner);
    const unsigned to = offset_of<T, LANES>(p, first, d.y_stride, d.inner);
    Held<T, VEC> v[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) v[k].load_at(x + k * step, from, p.there && group + k * groups < size);
    float s[VEC] = {};
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      v[k].refresh();
#pragma unroll
      for (int j = 0; j < VEC; ++j) s[j] += v[k][j];
    }
    channel_sum<VEC, LANES, THREADS>(s, red[0]);
    float mean[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      mean[j] = s[j] / (float)size;
      s[j] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const bool there = group + k * groups < size;
      v[k].refresh();
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float c = there ? v[k][j] - mean[j] : 0.f;
        s[j] = fmaf(c, c, s[j]);
      }
      v[k].refresh();
    }
    channel_sum<VEC, LANES, THREADS>(s, red[1]);
#pragma unroll
    for (int j = 0; j < VEC; ++j) s[j] = 1.f / sqrtf(s[j] / (float)size + (float)d.eps);
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int c = group + k * groups;
      if (c >= size) break;
      const float wc = w[c], bc = b[c];
      Pack<T, VEC> o;
#pragma unroll
      for (int j = 0; j < VEC; ++j) o.v[j] = (T)fmaf((v[k][j] - mean[j]) * s[j], wc, bc);
      store_at<T, VEC>(y + k * step, to, p.there, o);
    }
    if (a.stats && group == 0 && p.there)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        a.stats[p.outer * d.inner + p.at + j] = mean[j];
        a.stats[sites + p.outer * d.inner + p.at + j] = s[j];
      }
  }
}

// dx, and in part [block][2][size] this block's sums of dy h and of dy by channel.
template <typename T, int VEC, int LANES, int EACH, int THREADS>
__global__ __launch_bounds__(THREADS, 4) void k_maps_bwd(NormPtrs a, bl_norm_desc_t d, unsigned per_slice, long tiles,
                                                      bool sums) {
  constexpr int groups = THREADS / LANES;
  __shared__ float red[2][THREADS / kWave][LANES * 2 * VEC];
  __shared__ float w[EACH * groups];
  const int group = threadIdx.x / LANES, size = (int)d.size;
  const long sites = d.outer * d.inner, step = groups * d.inner;
  const float inv = 1.f / (float)size;
  float aw[EACH] = {}, ab[EACH] = {};
  stage_weights<T>(a.w, d.wdtype == BL_F32, size, 1.f, w);
  __syncthreads();
  int turn = 0;
  for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const Place p = place_of<VEC, LANES>(tile, d, per_slice);
    const long first = (unsigned)tile * LANES / per_slice;
    const T* x = static_cast<const T*>(a.x) + first * d.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + first * d.y_stride;
    T* dx = static_cast<T*>(a.dx) + first * d.x_stride;
    const unsigned at_x = offset_of<T, LANES>(p, first, d.x_stride, d.inner);
    const unsigned at_y = offset_of<T, LANES>(p, first, d.y_stride, d.inner);
    Held<T, VEC> v[EACH], g[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const bool there = p.there && group + k * groups < size;
      v[k].load_at(x + k * step, at_x, there);
      g[k].load_at(dy + k * step, at_y, there);
    }
    const long site = p.outer * d.inner + p.at;
    Held<float, VEC> mean, rstd;
    mean.load_at(a.stats + site, 0, p.there);
    rstd.load_at(a.stats + sites + site, 0, p.there);
    float s[2 * VEC] = {};
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int c = group + k * groups;
      const float wc = c < size ? w[c] : 0.f;
      v[k].refresh();
      g[k].refresh();
#pragma unroll
      for (int j = 0; j < VEC; ++j) {  // (where there is no value dy is 0)
        const float h = (v[k][j] - mean[j]) * rstd[j], dyj = g[k][j], u = dyj * wc;
        add_sums(u, h, s[2 * j], s[2 * j + 1]);
        aw[k] = fmaf(dyj, h, aw[k]);
        ab[k] += dyj;
      }
      v[k].refresh();
      g[k].refresh();
      __builtin_amdgcn_sched_barrier(0);  // (the scheduler would hold all channels' h at once)
    }
    channel_sum<2 * VEC, LANES, THREADS>(s, red[turn]);
    turn ^= 1;
#pragma unroll
    for (int j = 0; j < 2 * VEC; ++j) s[j] *= inv;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int c = group + k * groups;
      if (c >= size) break;
      const float wc = w[c];
      Pack<T, VEC> o;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float h = (v[k][j] - mean[j]) * rstd[j];
        o.v[j] = (T)grad_of(g[k][j] * wc, s[2 * j], h, s[2 * j + 1], rstd[j]);
      }
      store_at<T, VEC>(dx + k * step, at_x, p.there, o);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  if (!sums) return;
  float* part = a.part + (size_t)blockIdx.x * 2 * size;
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    const int c = group + k * groups;
    if (c >= size) break;
    aw[k] = wave_sum(aw[k], LANES);
    ab[k] = wave_sum(ab[k], LANES);
    if (threadIdx.x % LANES == 0) {
      part[c] = aw[k];
      part[size + c] = ab[k];
    }
  }
}

// More channels than a block's registers hold (over 1024): they are read again for
// the squares and for the result (from L2).  One position a lane, and one load of a lane
// in flight: 8 maps of 2000 channels and 512 positions, 64 blocks, take 102 us forward
// and 162 us backward, 0.6 TB/s.
constexpr int kStreamThreads = 1024;
__device__ __forceinline__ void stream_sum(float (&x)[2], float (*red)[2 * kWave]) { channel_sum<2, kWave, kStreamThreads>(x, red); }

template <typename T>
__global__ __launch_bounds__(kStreamThreads) void k_maps_fwd_stream(NormPtrs a, bl_norm_desc_t d, long tiles) {
  __shared__ float red[2][kMostWaves][2 * kWave];
  const int groups = blockDim.x / kWave, group = threadIdx.x / kWave;
  const bool wide = d.wdtype == BL_F32;
  const long sites = d.outer * d.inner;
  for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const Place p = place_of<1, kWave>(tile, d, (unsigned)d.inner);
    const T* x = static_cast<const T*>(a.x) + p.outer * d.x_stride + p.at;
    T* y = static_cast<T*>(a.y) + p.outer * d.y_stride + p.at;
    float s[2] = {};
    if (p.there)
      for (long c = group; c < d.size; c += groups) s[0] += to_f32(x[c * d.inner]);
    stream_sum(s, red[0]);
    const float mean = s[0] / (float)d.size;
    s[0] = s[1] = 0.f;
    if (p.there)
      for (long c = group; c < d.size; c += groups) {
        const float t = to_f32(x[c * d.inner]) - mean;
        s[0] = fmaf(t, t, s[0]);
      }
    stream_sum(s, red[1]);
    const float rstd = 1.f / sqrtf(s[0] / (float)d.size + (float)d.eps);
    if (!p.there) continue;
    for (long c = group; c < d.size; c += groups) {
      float w[1][1], b[1][1];
      load_weights<T, 1, 1>(a.w, wide, c, 0, d.size, 1.f, w);
      load_weights<T, 1, 1>(a.b, wide, c, 0, d.size, 0.f, b);
      y[c * d.inner] = (T)fmaf((to_f32(x[c * d.inner]) - mean) * rstd, w[0][0], b[0][0]);
    }
    if (a.stats && group == 0) {
      a.stats[p.outer * d.inner + p.at] = mean;
      a.stats[sites + p.outer * d.inner + p.at] = rstd;
    }
  }
}

template <typename T>
__global__ __launch_bounds__(kStreamThreads) void k_maps_bwd_stream(NormPtrs a, bl_norm_desc_t d, long tiles,
                                                                    bool sums) {
  __shared__ float red[2][kMostWaves][2 * kWave];
  const int groups = blockDim.x / kWave, group = threadIdx.x / kWave;
  const bool wide = d.wdtype == BL_F32;
  const long sites = d.outer * d.inner;
  float* part = a.part + (size_t)blockIdx.x * 2 * d.size;  // a wave's channels are its own
  int turn = 0;
  for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const Place p = place_of<1, kWave>(tile, d, (unsigned)d.inner);
    const T* x = static_cast<const T*>(a.x) + p.outer * d.x_stride + p.at;
    const T* dy = static_cast<const T*>(a.dy) + p.outer * d.y_stride + p.at;
    T* dx = static_cast<T*>(a.dx) + p.outer * d.x_stride + p.at;
    const long site = p.outer * d.inner + p.at;
    const float mean = p.there ? a.stats[site] : 0.f, rstd = p.there ? a.stats[sites + site] : 0.f;
    float s[2] = {};
    if (p.there)
      for (long c = group; c < d.size; c += groups) {
        float w[1][1];
        load_weights<T, 1, 1>(a.w, wide, c, 0, d.size, 1.f, w);
        const float u = to_f32(dy[c * d.inner]) * w[0][0];
        add_sums(u, (to_f32(x[c * d.inner]) - mean) * rstd, s[0], s[1]);
      }
    stream_sum(s, red[turn]);
    turn ^= 1;
    const float c1 = s[0] / (float)d.size, c2 = s[1] / (float)d.size;
    for (long c = group; c < d.size; c += groups) {
      float w[1][1], h = 0.f, g = 0.f;
      load_weights<T, 1, 1>(a.w, wide, c, 0, d.size, 1.f, w);
      if (p.there) {
        h = (to_f32(x[c * d.inner]) - mean) * rstd;
        g = to_f32(dy[c * d.inner]);
        dx[c * d.inner] = (T)grad_of(g * w[0][0], c1, h, c2, rstd);
      }
      if (!sums) continue;
      const float dw = wave_sum(g * h), db = wave_sum(g);
      if (threadIdx.x % kWave == 0) {
        const bool first = tile == (long)blockIdx.x;
        part[c] = dw + (first ? 0.f : part[c]);
        part[d.size + c] = db + (first ? 0.f : part[d.size + c]);
      }
    }
  }
}

// The shapes that the kernels are compiled for, by the channels they hold: channels
// of a thread and threads of a block.  Backward a thread holds twice the values and
// two sums for each channel, so half the channels.
struct Shape {
  int threads, vec, lanes, each;
};
constexpr int kForward[][2] = {{4, 256}, {8, 256}, {16, 256}, {16, 512}, {16, 1024}};
constexpr int kBackward[][2] = {{4, 256}, {8, 256}, {8, 512}, {8, 1024}, {16, 1024}};

// A lane holds the most positions that divide the map's, up to `most` (forward 8
// bytes, backward two), and as many lanes lie along positions as fill a line of 128
// bytes; 16, where those do not leave enough for the channels.  The last backward
// shape has registers for single positions only.  More channels, or slices too far
// apart for 32-bit offsets in a tile: the channels are read again for every use.
Shape maps_shape(const bl_norm_desc_t& d, const int (&shapes)[5][2], int most, bool halve_last) {
  const int wide = dtype_bytes(d.dtype);
  const long stride = std::max(d.x_stride, d.y_stride);
  int vec = most;
  while (d.inner % vec) vec /= 2;
  Shape got{kStreamThreads, 1, kWave, 0};
  for (int lanes = 128 / (vec * wide); !got.each && lanes >= 16; lanes = lanes > 16 ? 16 : 0)
    for (int i = 0; i < 5 && !got.each; ++i)
      if ((long)shapes[i][0] * (shapes[i][1] / lanes) >= d.size)
        got = Shape{shapes[i][1], i == 4 && halve_last ? 1 : vec, lanes, shapes[i][0]};
  // a tile spans at most this many slices
  const long span = ((long)got.lanes * got.vec + d.inner - 1) / d.inner + 1;
  if (got.each && (span * stride + d.size * d.inner) * wide >= 1L << 32) got = Shape{kStreamThreads, 1, kWave, 0};
  return got;
}

long tiles_of(const bl_norm_desc_t& d, int vec, int lanes, unsigned* per_slice) {
  *per_slice = (unsigned)(d.inner / vec);
  return ((long)d.outer * *per_slice + lanes - 1) / lanes;
}

// go(vec, lanes, each, threads) of the plan's shape, as constants.
template <typename T, bool BACKWARD, typename Go>
bl_status_t dispatch(const bl_norm_plan_s* p, Go&& go) {
  constexpr const int(&shapes)[5][2] = BACKWARD ? kBackward : kForward;
  const int vec = p->map_vec[BACKWARD], on = p->map_lanes[BACKWARD];
  const int each = p->map_each[BACKWARD], threads = p->map_threads[BACKWARD];
#define BL_MAPS(V, L, I)                                                                       \
  if (vec == V && on == L && each == shapes[I][0] && threads == shapes[I][1])                  \
  return go(std::integral_constant<int, V>(), std::integral_constant<int, L>(),                \
            std::integral_constant<int, shapes[I][0]>(), std::integral_constant<int, shapes[I][1]>())
#define BL_MAPS4(V, L) \
  BL_MAPS(V, L, 0);    \
  BL_MAPS(V, L, 1);    \
  BL_MAPS(V, L, 2);    \
  BL_MAPS(V, L, 3)
#define BL_MAPS5(V, L) \
  BL_MAPS4(V, L);      \
  BL_MAPS(V, L, 4)
  if constexpr (sizeof(T) == 4) {
    if constexpr (BACKWARD) { BL_MAPS4(2, 16); } else { BL_MAPS5(2, 16); }
    BL_MAPS5(1, 32);
  } else {
    if constexpr (BACKWARD) { BL_MAPS4(2, 32); } else { BL_MAPS5(4, 16); BL_MAPS5(2, 32); }
    BL_MAPS5(1, 64);
    if constexpr (BACKWARD) { BL_MAPS(1, 32, 4); } else { BL_MAPS(2, 16, 4); }
    BL_MAPS(1, 16, 3);
  }
  BL_MAPS(1, 16, 4);
#undef BL_MAPS5
#undef BL_MAPS4
#undef BL_MAPS
  return BL_ERR_INVALID_ARG;
}

template <typename T>
bl_status_t forward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  unsigned per_slice;
  const long tiles = tiles_of(p->d, p->map_vec[0], p->map_lanes[0], &per_slice);
  const dim3 grid((unsigned)std::min<long>(tiles, 1L << 20)), block(p->map_threads[0]);
  const double bytes = 2.0 * p->d.outer * p->d.size * p->d.inner * sizeof(T);
  bl_status_t shape = BL_OK;
  const bl_status_t st = timed_launch("norm_fwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    if (!p->map_each[0]) {
      hipExtLaunchKernelGGL(k_maps_fwd_stream<T>, grid, block, 0, s, e0, e1, 0, a, p->d, tiles);
      return;
    }
    shape = dispatch<T, false>(p, [&](auto v, auto l, auto e, auto n) {
      hipExtLaunchKernelGGL((k_maps_fwd<T, decltype(v)::value, decltype(l)::value, decltype(e)::value, decltype(n)::value>), grid,
                            block, 0, s, e0, e1, 0, a, p->d, per_slice, tiles);
      return BL_OK;
    });
  });
  return shape != BL_OK ? shape : st;
}

template <typename T>
bl_status_t backward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  unsigned per_slice;
  const long tiles = tiles_of(p->d, p->map_vec[1], p->map_lanes[1], &per_slice);
  const dim3 grid((unsigned)p->parts), block(p->map_threads[1]);
  const bool sums = a.dw || a.db;
  const double bytes = 3.0 * p->d.outer * p->d.size * p->d.inner * sizeof(T);
  bl_status_t shape = BL_OK;
  const bl_status_t st = timed_launch("norm_bwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    if (!p->map_each[1]) {
      hipExtLaunchKernelGGL(k_maps_bwd_stream<T>, grid, block, 0, s, e0, e1, 0, a, p->d, tiles, sums);
      return;
    }
    shape = dispatch<T, true>(p, [&](auto v, auto l, auto e, auto n) {
      hipExtLaunchKernelGGL((k_maps_bwd<T, decltype(v)::value, decltype(l)::value, decltype(e)::value, decltype(n)::value>), grid,
                            block, 0, s, e0, e1, 0, a, p->d, per_slice, tiles, sums);
      return BL_OK;
    });
  });
  if (shape != BL_OK) return shape;
  return st == BL_OK && sums ? norm_sum_parts(p, a, p->parts, s) : st;
}

}  // namespace

bl_status_t norm_maps_plan(bl_norm_plan_s* p) {
  const Shape shapes[2] = {maps_shape(p->d, kForward, 8 / dtype_bytes(p->d.dtype), false),
                           maps_shape(p->d, kBackward, 2, true)};
  for (int i = 0; i < 2; ++i) {
    p->map_threads[i] = shapes[i].threads;
    p->map_vec[i] = shapes[i].vec;
    p->map_lanes[i] = shapes[i].lanes;
    p->map_each[i] = shapes[i].each;
  }
  unsigned per_slice;
  const long tiles = tiles_of(p->d, shapes[1].vec, shapes[1].lanes, &per_slice);
  // as many blocks as are on the GPU at once: each gives a row of partial sums (half of
  // them / these / twice, with the last sum, fp32 at 512 positions: 64 maps of 256
  // channels 25 + 4 / 23 + 4 / 26.5 + 6.5 us, of 512 63 + 4 / 45 + 4 / 47 + 4; on blocks
  // of 1024 of 1024 channels 177 + 4 / 129 + 4 / 130 + 5)
  p->parts = (int)std::min<long>(tiles, shapes[1].threads == kMostThreads ? 256 : 512);
  p->off_part = 0;
  p->bytes = (size_t)p->parts * 2 * p->d.size * sizeof(float);
  return BL_OK;
}

bl_status_t norm_maps_forward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  if (p->d.dtype == BL_F32) return forward<float>(p, a, s);
  if (p->d.dtype == BL_BF16) return forward<bf16_t>(p, a, s);
  return forward<f16_t>(p, a, s);
}

bl_status_t norm_maps_backward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  if (p->d.dtype == BL_F32) return backward<float>(p, a, s);
  if (p->d.dtype == BL_BF16) return backward<bf16_t>(p, a, s);
  return backward<f16_t>(p, a, s);
}

}  // namespace blc
