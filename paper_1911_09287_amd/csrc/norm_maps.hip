// Layer norm over the channels at each position (inner > 1): x [outer][size][inner].
//
// Positions lie on lanes, 8 or 16 bytes of them on one, so that a channel's
// positions are read as whole lines; the channels of a position lie on the other
// lanes and waves of a block and, `EACH` of them, in a thread's registers.  So
// every value is read once and written once, and sums over the channels cross the
// lanes by shuffles and the waves by way of LDS.  Backward, a thread keeps the
// sums of its channels' dw and db over all tiles of its block.  Bound by HBM.
#include <algorithm>

#include "norm.hpp"

namespace blc {
namespace {

constexpr int kMostThreads = 1024;
constexpr int kMostWaves = kMostThreads / kWave;

// A block's tile of positions, and this thread's place in it: its first position's
// offset in a channel, the outer slice and how many of VEC positions there are.
struct Place {
  long outer, at;
  int n;
};
template <int VEC, int LANES>
__device__ __forceinline__ Place place_of(long tile, const bl_norm_desc_t& d, unsigned per_slice) {
  const unsigned q = (unsigned)tile * LANES + threadIdx.x % LANES;  // of all vectors of positions
  const unsigned o = q / per_slice, i = (q - o * per_slice) * VEC;
  Place p{(long)o, (long)i, 0};
  if (o < (unsigned long long)d.outer) p.n = (int)min((long)VEC, (long)d.inner - p.at);
  return p;
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
  const int group = threadIdx.x / LANES;
  const bool wide = d.wdtype == BL_F32;
  const long sites = d.outer * d.inner, step = groups * d.inner;
  for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const Place p = place_of<VEC, LANES>(tile, d, per_slice);
    const T* x = static_cast<const T*>(a.x) + p.outer * d.x_stride + p.at + group * d.inner;
    T* y = static_cast<T*>(a.y) + p.outer * d.y_stride + p.at + group * d.inner;
    Held<T, VEC> v[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k, x += step) v[k].load(x, group + k * groups < d.size ? p.n : 0);
    float w[EACH][1], b[EACH][1];
    load_weights<T, 1, EACH>(a.w, wide, group, groups, d.size, 1.f, w);
    load_weights<T, 1, EACH>(a.b, wide, group, groups, d.size, 0.f, b);
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
      mean[j] = s[j] / (float)d.size;
      s[j] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const bool there = group + k * groups < d.size;
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
    for (int j = 0; j < VEC; ++j) s[j] = 1.f / sqrtf(s[j] / (float)d.size + (float)d.eps);
#pragma unroll
    for (int k = 0; k < EACH; ++k, y += step) {
      const int c = group + k * groups;
      if (c >= d.size) break;
      Pack<T, VEC> o;
#pragma unroll
      for (int j = 0; j < VEC; ++j) o.v[j] = (T)fmaf((v[k][j] - mean[j]) * s[j], w[k][0], b[k][0]);
      store_part<T, VEC>(y, p.n, o);
    }
    if (a.stats && group == 0)
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (j < p.n) {
          a.stats[p.outer * d.inner + p.at + j] = mean[j];
          a.stats[sites + p.outer * d.inner + p.at + j] = s[j];
        }
  }
}

// dx, and in part [block][2][size] this block's sums of dy h and of dy by channel.
template <typename T, int VEC, int LANES, int EACH, int THREADS>
__global__ __launch_bounds__(THREADS) void k_maps_bwd(NormPtrs a, bl_norm_desc_t d, unsigned per_slice, long tiles,
                                                      bool sums) {
  constexpr int groups = THREADS / LANES;
  __shared__ float red[2][THREADS / kWave][LANES * 2 * VEC];
  const int group = threadIdx.x / LANES;
  const bool wide = d.wdtype == BL_F32;
  const long sites = d.outer * d.inner, step = groups * d.inner;
  const float inv = 1.f / (float)d.size;
  float w[EACH][1], aw[EACH] = {}, ab[EACH] = {};
  load_weights<T, 1, EACH>(a.w, wide, group, groups, d.size, 1.f, w);
  int turn = 0;
  for (long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
    const Place p = place_of<VEC, LANES>(tile, d, per_slice);
    const T* x = static_cast<const T*>(a.x) + p.outer * d.x_stride + p.at + group * d.inner;
    const T* dy = static_cast<const T*>(a.dy) + p.outer * d.y_stride + p.at + group * d.inner;
    T* dx = static_cast<T*>(a.dx) + p.outer * d.x_stride + p.at + group * d.inner;
    Held<T, VEC> v[EACH], g[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k, x += step, dy += step) {
      const int n = group + k * groups < d.size ? p.n : 0;
      v[k].load(x, n);
      g[k].load(dy, n);
    }
    const long site = p.outer * d.inner + p.at;
    const Pack<float, VEC> mean = load_part<float, VEC>(a.stats + site, p.n, 0.f);
    const Pack<float, VEC> rstd = load_part<float, VEC>(a.stats + sites + site, p.n, 0.f);
    float s[2 * VEC] = {};
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      v[k].refresh();
      g[k].refresh();
#pragma unroll
      for (int j = 0; j < VEC; ++j) {  // (where there is no value dy is 0)
        const float h = (v[k][j] - mean.v[j]) * rstd.v[j], dyj = g[k][j], u = dyj * w[k][0];
        s[2 * j] += u;
        s[2 * j + 1] = fmaf(u, h, s[2 * j + 1]);
        aw[k] = fmaf(dyj, h, aw[k]);
        ab[k] += dyj;
      }
      v[k].refresh();
      g[k].refresh();
    }
    channel_sum<2 * VEC, LANES, THREADS>(s, red[turn]);
    turn ^= 1;
#pragma unroll
    for (int k = 0; k < EACH; ++k, dx += step) {
      const int c = group + k * groups;
      if (c >= d.size) break;
      Pack<T, VEC> o;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float h = (v[k][j] - mean.v[j]) * rstd.v[j];
        o.v[j] = (T)(rstd.v[j] * (fmaf(g[k][j], w[k][0], -s[2 * j] * inv) - h * (s[2 * j + 1] * inv)));
      }
      store_part<T, VEC>(dx, p.n, o);
    }
  }
  if (!sums) return;
  float* part = a.part + (size_t)blockIdx.x * 2 * d.size;
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    const int c = group + k * groups;
    if (c >= d.size) break;
    aw[k] = wave_sum(aw[k], LANES);
    ab[k] = wave_sum(ab[k], LANES);
    if (threadIdx.x % LANES == 0) {
      part[c] = aw[k];
      part[d.size + c] = ab[k];
    }
  }
}

// More channels than a block's registers hold: they are read again for the
// squares and for the result (from L2).  One position a lane.
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
    if (p.n)
      for (long c = group; c < d.size; c += groups) s[0] += to_f32(x[c * d.inner]);
    stream_sum(s, red[0]);
    const float mean = s[0] / (float)d.size;
    s[0] = s[1] = 0.f;
    if (p.n)
      for (long c = group; c < d.size; c += groups) {
        const float t = to_f32(x[c * d.inner]) - mean;
        s[0] = fmaf(t, t, s[0]);
      }
    stream_sum(s, red[1]);
    const float rstd = 1.f / sqrtf(s[0] / (float)d.size + (float)d.eps);
    if (!p.n) continue;
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
    const float mean = p.n ? a.stats[site] : 0.f, rstd = p.n ? a.stats[sites + site] : 0.f;
    float s[2] = {};
    if (p.n)
      for (long c = group; c < d.size; c += groups) {
        float w[1][1];
        load_weights<T, 1, 1>(a.w, wide, c, 0, d.size, 1.f, w);
        const float u = to_f32(dy[c * d.inner]) * w[0][0];
        s[0] += u;
        s[1] = fmaf(u, (to_f32(x[c * d.inner]) - mean) * rstd, s[1]);
      }
    stream_sum(s, red[turn]);
    turn ^= 1;
    const float c1 = s[0] / (float)d.size, c2 = s[1] / (float)d.size;
    for (long c = group; c < d.size; c += groups) {
      float w[1][1], h = 0.f, g = 0.f;
      load_weights<T, 1, 1>(a.w, wide, c, 0, d.size, 1.f, w);
      if (p.n) {
        h = (to_f32(x[c * d.inner]) - mean) * rstd;
        g = to_f32(dy[c * d.inner]);
        dx[c * d.inner] = (T)(rstd * (fmaf(g, w[0][0], -c1) - h * c2));
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

// The shapes that the kernels are compiled for, by the channels they hold: threads
// of a block and channels of a thread.  On 16 lanes along positions a block of 256
// has 16 groups for channels, on 32 it has 8, on 64 4.
struct Shape {
  int threads, vec, lanes, each;
};
constexpr int kShapes[][2] = {{256, 4}, {256, 8}, {256, 16}, {512, 16}, {1024, 16}};

// `full`: positions of a vector (forward 16 bytes, backward, with twice the
// values to hold, 8).  Where the map's positions fill vectors (or only the last of
// many is cut) lanes hold vectors, 32 backward and 16 forward, which are 256 bytes
// of a channel; else single positions, 64 lanes.  Many channels: 16 lanes.
Shape maps_shape(const bl_norm_desc_t& d, int full, int lanes) {
  const int vec = d.inner % full == 0 || d.inner >= 8 * full ? full : 1;
  for (const auto& s : kShapes) {
    const int on = vec > 1 ? lanes : kWave;
    if ((long)s[1] * (s[0] / on) >= d.size) return Shape{s[0], vec, on, s[1]};
  }
  if (16L * (kMostThreads / 16) >= d.size) return Shape{kMostThreads, vec, 16, 16};
  return Shape{kStreamThreads, 1, kWave, 0};
}

long tiles_of(const bl_norm_desc_t& d, int vec, int lanes, unsigned* per_slice) {
  *per_slice = (unsigned)((d.inner + vec - 1) / vec);
  return ((long)d.outer * *per_slice + lanes - 1) / lanes;
}

template <typename T, bool BACKWARD, typename Go>
bl_status_t dispatch(const bl_norm_plan_s* p, Go&& go) {
  constexpr int full = (BACKWARD ? 8 : 16) / sizeof(T), lanes = 16;
  const int vec = p->map_vec[BACKWARD], on = p->map_lanes[BACKWARD], each = p->map_each[BACKWARD];
  const int threads = p->map_threads[BACKWARD];
#define BL_MAPS(V, L, E, N)                                            \
  if (vec == V && on == L && each == E && threads == N)                \
  return go(std::integral_constant<int, V>(), std::integral_constant<int, L>(), std::integral_constant<int, E>(), \
            std::integral_constant<int, N>())
#define BL_MAPS5(V, L)      \
  BL_MAPS(V, L, 4, 256);    \
  BL_MAPS(V, L, 8, 256);    \
  BL_MAPS(V, L, 16, 256);   \
  BL_MAPS(V, L, 16, 512);   \
  BL_MAPS(V, L, 16, 1024)
  BL_MAPS5(full, lanes);
  BL_MAPS5(1, 64);
  BL_MAPS(1, 16, 16, 1024);
#undef BL_MAPS5
#undef BL_MAPS
  return BL_ERR_INVALID_ARG;
}

template <typename T>
bl_status_t forward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  unsigned per_slice;
  const long tiles = tiles_of(p->d, p->map_vec[0], p->map_lanes[0], &per_slice);
  const dim3 grid((unsigned)std::min<long>(tiles, 1L << 20)), block(p->map_threads[0]);
  const double bytes = 2.0 * p->d.outer * p->d.size * p->d.inner * sizeof(T);
  return timed_launch("norm_fwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    if (!p->map_each[0]) {
      hipExtLaunchKernelGGL(k_maps_fwd_stream<T>, grid, block, 0, s, e0, e1, 0, a, p->d, tiles);
      return;
    }
    (void)dispatch<T, false>(p, [&](auto v, auto l, auto e, auto n) {
      hipExtLaunchKernelGGL((k_maps_fwd<T, decltype(v)::value, decltype(l)::value, decltype(e)::value, decltype(n)::value>), grid,
                            block, 0, s, e0, e1, 0, a, p->d, per_slice, tiles);
      return BL_OK;
    });
  });
}

template <typename T>
bl_status_t backward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  unsigned per_slice;
  const long tiles = tiles_of(p->d, p->map_vec[1], p->map_lanes[1], &per_slice);
  const dim3 grid((unsigned)p->parts), block(p->map_threads[1]);
  const bool sums = a.dw || a.db;
  const double bytes = 3.0 * p->d.outer * p->d.size * p->d.inner * sizeof(T);
  const bl_status_t st = timed_launch("norm_bwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    if (!p->map_each[1]) {
      hipExtLaunchKernelGGL(k_maps_bwd_stream<T>, grid, block, 0, s, e0, e1, 0, a, p->d, tiles, sums);
      return;
    }
    (void)dispatch<T, true>(p, [&](auto v, auto l, auto e, auto n) {
      hipExtLaunchKernelGGL((k_maps_bwd<T, decltype(v)::value, decltype(l)::value, decltype(e)::value, decltype(n)::value>), grid,
                            block, 0, s, e0, e1, 0, a, p->d, per_slice, tiles, sums);
      return BL_OK;
    });
  });
  return st == BL_OK && sums ? norm_sum_parts(p, a, p->parts, s) : st;
}

}  // namespace

bl_status_t norm_maps_plan(bl_norm_plan_s* p) {
  const int wide = dtype_bytes(p->d.dtype);
  const Shape f = maps_shape(p->d, 16 / wide, 16), b = maps_shape(p->d, 8 / wide, 16);
  const Shape both[2] = {f, b};
  for (int i = 0; i < 2; ++i) {
    p->map_threads[i] = both[i].threads;
    p->map_vec[i] = both[i].vec;
    p->map_lanes[i] = both[i].lanes;
    p->map_each[i] = both[i].each;
  }
  unsigned per_slice;
  const long tiles = tiles_of(p->d, b.vec, b.lanes, &per_slice);
  // as many blocks as are on the GPU at once: each gives a row of partial sums
  p->parts = (int)std::min<long>(tiles, 256L * (kMostThreads / b.threads));
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
