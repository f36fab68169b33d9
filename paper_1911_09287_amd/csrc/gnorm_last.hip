// Group norm with an activation, channels last: x [batch][sites][channels].
//
// A thread keeps an access of channels (`vec` of them, a divisor of their number) and walks
// sites, so that neighbouring threads read neighbouring memory whatever the channels'
// number, and what belongs to its channels (weights, statistics) stays in registers.
//
// Two blocks a compute unit with the next sites' loads in flight: the sums of 51 MB take 13.9 us
// (3.7 TB/s, from memory) and the launch that applies them 20.6 (5.0 TB/s, x from the cache).
#include <algorithm>

#include "gnorm.hpp"

namespace blc {
namespace {

// Sites of a thread whose loads are in flight while as many are worked on; backward, of x and dy.
// (With twice as many the sums above take 15.7 us and those of 32 x 3136 x 256 backward 35, not 32.)
template <typename T, int V>
constexpr int kAhead = V * sizeof(T) >= 16 ? 4 : 8;
template <typename T, int V>
constexpr int kAheadBoth = kAhead<T, V> / 2;
constexpr int kFew = 16;       // turns whose sums are taken by themselves
constexpr int kMostWholeParts = 16;
constexpr int kMostParts = 8;  // of a channel's slices, which threads sum side by side

// Where a thread stands: sample, chunk, its first channel and its sites begin + slice, begin +
// slice + slices, ... below end.
struct LastPlace {
  long n, chunk, c, begin, end;
  int lane, slice, slices;
  bool there;
  template <int V>
  __device__ __forceinline__ static LastPlace make(const GroupNormArgs& a, unsigned block) {
    LastPlace p;
    const long q = (long)block / a.tiles, tile = (long)block - q * a.tiles;
    p.n = q / a.chunks;
    p.chunk = q - p.n * a.chunks;
    p.slices = kThreads / a.lanes;
    p.slice = threadIdx.x / a.lanes;
    p.lane = threadIdx.x - p.slice * a.lanes;
    p.c = (tile * kThreads + p.lane) * V;
    p.there = p.slice < p.slices && p.c < a.channels;
    p.begin = p.chunk * a.chunk;
    p.end = min(a.sites, p.begin + a.chunk);
    return p;
  }
  // COUNT sites of a thread at a time: load(held, site) for them while work(held, site, the
  // sites that there are) goes through those before.  Sites behind the last one are read as the
  // last one, so that loads have no branch around them and can be told from those after.
  template <int COUNT, typename H, typename Load, typename Work>
  __device__ __forceinline__ void walk(Load&& load, Work&& work) const {
    const long step = (long)COUNT * slices;
    H now[COUNT], next[COUNT];
    auto fetch = [&](H (&to)[COUNT], long from) {
#pragma unroll
      for (int k = 0; k < COUNT; ++k) load(to[k], min(from + (long)k * slices + slice, end - 1));
    };
    long t = begin;
    fetch(now, t);
    for (; t + step <= end; t += step) {
      fetch(next, t + step);
      work(now, t + slice, std::integral_constant<int, COUNT>());
#pragma unroll
      for (int k = 0; k < COUNT; ++k) now[k] = next[k];
    }
    const long left = end - t - slice;
    if (left > 0) work(now, t + slice, (int)((left + slices - 1) / slices));
  }
};

// Sums over the slices of a thread's N values, in each thread.  red: [kThreads][N].
template <int N>
__device__ __forceinline__ void slices_sum(float (&v)[N], float* red, const LastPlace& p, int lanes) {
  if (p.slices == 1) return;
  const int width = lanes * N, parts = max(1, min(min(kMostParts, p.slices), kThreads / width));
#pragma unroll
  for (int j = 0; j < N; ++j) red[threadIdx.x * N + j] = v[j];
  __syncthreads();
  // (a part's threads alone read the place that its sum goes to)
  for (int i = threadIdx.x; i < parts * width; i += kThreads) {
    const int q = i / width, c = i - q * width;
    float s = 0.f;
    for (int k = q; k < p.slices; k += parts) s += red[k * width + c];
    red[i] = s;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < N; ++j) v[j] = 0.f;
  for (int q = 0; q < parts; ++q)
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] += red[q * width + p.lane * N + j];
}

// Each channel's moments over the block's sites.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void k_last_part(GroupNormArgs a) {
  __shared__ float red[kThreads * V];
  const LastPlace p = LastPlace::make<V>(a, blockIdx.x);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c;
  float n = 0.f, mean[V] = {}, m2[V] = {};
  if (p.there)
    p.walk<kAhead<T, V>, Held<T, V>>(
        [&](Held<T, V>& to, long site) { to.load(x + site * a.channels, V); },
        [&](Held<T, V>(&v)[kAhead<T, V>], long, auto count) {
          const float inv = 1.f / (float)count, share = (float)count / (n + (float)count);
          const float old = n * share;
#pragma unroll
          for (int k = 0; k < kAhead<T, V>; ++k) v[k].refresh();
#pragma unroll
          for (int j = 0; j < V; ++j) {
            float m = 0.f, s = 0.f;
#pragma unroll
            for (int k = 0; k < kAhead<T, V>; ++k) m += k < count ? v[k][j] : 0.f;
            m *= inv;
#pragma unroll
            for (int k = 0; k < kAhead<T, V>; ++k) {
              const float d = k < count ? v[k][j] - m : 0.f;
              s = fmaf(d, d, s);
            }
            const float d = m - mean[j];
            m2[j] += fmaf(d * d, old, s);
            mean[j] = fmaf(d, share, mean[j]);
          }
          n += (float)count;
        });
  // the block's means, then the squares about them
  float sum[V];
  const float inv = 1.f / (float)(p.end - p.begin);
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = n * mean[j];
  slices_sum(sum, red, p, a.lanes);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < V; ++j) {
    sum[j] = p.slices == 1 ? mean[j] : sum[j] * inv;
    const float d = mean[j] - sum[j];
    m2[j] = fmaf(n * d, d, m2[j]);
  }
  slices_sum(m2, red, p, a.lanes);
  if (p.slice || !p.there) return;
  float* to = a.part + ((p.n * a.chunks + p.chunk) * a.channels + p.c) * 2;
#pragma unroll
  for (int j = 0; j < V; ++j) to[2 * j] = sum[j], to[2 * j + 1] = m2[j];
}

// Two sums over each group's parts in a sample, of one chunk and channel each, by as many lanes of
// a wave as there are parts: first(part), then second(part, the first sum), and done(group, both).
// Every thread calls it.
template <typename Value, typename First, typename Second, typename Done>
__device__ __forceinline__ void join_parts(const GroupNormArgs& a, long n, First&& first, Second&& second, Done&& done) {
  const int parts = (int)a.each * a.chunks, each = (int)a.each;
  int on = 1;
  while (on < parts) on *= 2;
  const int lane = threadIdx.x % on, k = lane / each, c = lane - k * each;
  for (long g0 = 0; g0 < a.groups; g0 += kThreads / on) {
    const long g = g0 + threadIdx.x / on;
    const bool there = g < a.groups && lane < parts;
    Value v;
    v.load(a, there, there ? a.part + ((n * a.chunks + k) * a.channels + g * each + c) * 2 : a.part,
           there ? g * each + c : 0, k);
    const float s1 = wave_sum(first(v), on), s2 = wave_sum(second(v, s1), on);
    if (there && lane == 0) done(g, s1, s2);
  }
}
// A part's sites (0: there is none), mean and squares about it.
struct PartMoments {
  float sites, mean, m2;
  __device__ __forceinline__ void load(const GroupNormArgs& a, bool there, const float* from, long, int chunk) {
    const Pack<float, 2> v = load_pack<float, 2>(from);
    sites = there ? (float)min(a.chunk, a.sites - (long)chunk * a.chunk) : 0.f;
    mean = there ? v.v[0] : 0.f;
    m2 = there ? v.v[1] : 0.f;
  }
};
// A part's sums of u = dz w and of u h; every product and sum rounds by itself, so that a group
// of one value, whose u is its mean, has a gradient of 0.
template <typename T>
struct PartSums {
  float u, uh;
  __device__ __forceinline__ void load(const GroupNormArgs& a, bool there, const float* from, long c, int) {
#pragma clang fp contract(off)
    const Pack<float, 2> v = load_pack<float, 2>(from);
    const float w = weight_at<T>(a.w, a.wide, c, 1.f);
    u = there ? v.v[0] * w : 0.f;
    uh = there ? v.v[1] * w : 0.f;
  }
};

// What a thread's channels need: statistics and weights.
template <typename T, int V>
struct LastChannels {
  float mean[V], rstd[V], w[V], b[V];
  // stats: of the sample's groups, rstd `all` behind mean
  __device__ __forceinline__ void load(const GroupNormArgs& a, const LastPlace& p, const float* stats, long all) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const long c = p.there ? p.c + j : 0, q = c / a.each;
      mean[j] = stats[q];
      rstd[j] = stats[all + q];
      w[j] = weight_at<T>(a.w, a.wide, c, 1.f);
      b[j] = weight_at<T>(a.b, a.wide, c, 0.f);
    }
  }
  __device__ __forceinline__ void load(const GroupNormArgs& a, const LastPlace& p) {
    load(a, p, a.stats + p.n * a.groups, a.batch * a.groups);
  }
};

// JOINS: the statistics are joined here, by each block for itself (the first of a sample leaves them).
template <typename T, int V, int ACT, bool JOINS>
__global__ __launch_bounds__(kThreads) void k_last_apply(GroupNormArgs a) {
  const LastPlace p = LastPlace::make<V>(a, blockIdx.x);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c;
  T* y = static_cast<T*>(a.y) + p.n * a.y_stride + p.c;
  LastChannels<T, V> own;
  if constexpr (JOINS) {
    __shared__ float stats[2 * kMostJoined];
    const float size = (float)a.sites * (float)a.each;
    join_parts<PartMoments>(
        a, p.n, [](const PartMoments& v) { return v.sites * v.mean; },
        [&](const PartMoments& v, float sum) {
          const float d = v.mean - sum / size;
          return fmaf(v.sites * d, d, v.m2);
        },
        [&](long g, float sum, float m2) {
          const float mean = sum / size, rstd = 1.f / sqrtf(m2 / size + a.eps);
          stats[g] = mean;
          stats[kMostJoined + g] = rstd;
          if (p.chunk) return;
          a.stats[p.n * a.groups + g] = mean;
          a.stats[(a.batch + p.n) * a.groups + g] = rstd;
        });
    __syncthreads();
    own.load(a, p, stats, kMostJoined);
  } else {
    own.load(a, p);
  }
  if (!p.there) return;
  p.walk<kAhead<T, V>, Held<T, V>>(
      [&](Held<T, V>& to, long site) { to.load(x + site * a.channels, V); },
      [&](Held<T, V>(&v)[kAhead<T, V>], long site, auto count) {
#pragma unroll
        for (int k = 0; k < kAhead<T, V>; ++k, site += p.slices) {
          v[k].refresh();
          Pack<T, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j)
            o.v[j] = (T)act_of<ACT, T>(norm_z(v[k][j], own.mean[j], own.rstd[j], own.w[j], own.b[j]));
          if (k < count) store_pack(y + site * a.channels, o);
        }
      });
}

// A site's x and dy.
template <typename T, int V>
struct HeldBoth {
  Held<T, V> v, g;
  __device__ __forceinline__ void load(const T* x, const T* dy) {
    v.load(x, V);
    g.load(dy, V);
  }
  __device__ __forceinline__ void refresh() {
    v.refresh();
    g.refresh();
  }
};

// Each channel's sums of dz and of dz h over the block's sites.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_last_bwd_part(GroupNormArgs a) {
  __shared__ float red[kThreads * 2 * V];
  const LastPlace p = LastPlace::make<V>(a, blockIdx.x);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c;
  const T* dy = static_cast<const T*>(a.dy) + p.n * a.y_stride + p.c;
  LastChannels<T, V> own;
  own.load(a, p);
  // Sums of kFew turns' sites, and of those before: one chain over all of a long sample's would round too much
  // (512 x 32768 x 64 fp32, one value throughout: db off by 2e-5, and 1e-6 so)
  float s[2 * V] = {}, before[2 * V] = {};
  int turn = 0;
  if (p.there)
    p.walk<kAheadBoth<T, V>, HeldBoth<T, V>>(
        [&](HeldBoth<T, V>& to, long site) { to.load(x + site * a.channels, dy + site * a.channels); },
        [&](HeldBoth<T, V>(&at)[kAheadBoth<T, V>], long, auto count) {
#pragma unroll
          for (int k = 0; k < kAheadBoth<T, V>; ++k) {
            at[k].refresh();
            if (k >= count) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) {
              const float h = (at[k].v[j] - own.mean[j]) * own.rstd[j];
              const float dz = act_grad<ACT, T>(norm_z(at[k].v[j], own.mean[j], own.rstd[j], own.w[j], own.b[j]), at[k].g[j]);
              s[2 * j] += dz;
              s[2 * j + 1] = fmaf(dz, h, s[2 * j + 1]);
            }
          }
          if (++turn % kFew == 0)
#pragma unroll
            for (int j = 0; j < 2 * V; ++j) before[j] += s[j], s[j] = 0.f;
        });
#pragma unroll
  for (int j = 0; j < 2 * V; ++j) s[j] += before[j];
  slices_sum(s, red, p, a.lanes);
  if (p.slice || !p.there) return;
  float* to = a.part + ((p.n * a.chunks + p.chunk) * a.channels + p.c) * 2;
#pragma unroll
  for (int j = 0; j < 2 * V; ++j) to[j] = s[j];
}

// (the blocks past the values' own sum the weights' gradients)
template <typename T, int V, int ACT, bool JOINS>
__global__ __launch_bounds__(kThreads) void k_last_bwd_apply(GroupNormArgs a, unsigned blocks) {
  // (JOINS: these come first, as they have more to sum)
  const unsigned sums = gridDim.x - blocks, block = JOINS ? blockIdx.x - sums : blockIdx.x;
  if (block >= blocks) {
    gnorm_weights_block<T>(a, JOINS ? blockIdx.x : blockIdx.x - blocks);
    return;
  }
  const LastPlace p = LastPlace::make<V>(a, block);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c;
  const T* dy = static_cast<const T*>(a.dy) + p.n * a.y_stride + p.c;
  T* dx = static_cast<T*>(a.dx) + p.n * a.x_stride + p.c;
  LastChannels<T, V> own;
  own.load(a, p);
  const float* means = a.sums + 2 * p.n * a.groups;
  if constexpr (JOINS) {
    __shared__ float joined[2 * kMostJoined];
    const float size = (float)a.sites * (float)a.each;
    join_parts<PartSums<T>>(
        a, p.n, [](const PartSums<T>& v) { return v.u; }, [](const PartSums<T>& v, float) { return v.uh; },
        [&](long g, float u, float uh) {
          joined[2 * g] = u / size;
          joined[2 * g + 1] = uh / size;
        });
    __syncthreads();
    means = joined;
  }
  float c1[V], c2[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const long q = (p.there ? p.c + j : 0) / a.each;
    c1[j] = means[2 * q];
    c2[j] = means[2 * q + 1];
  }
  if (!p.there) return;
  p.walk<kAheadBoth<T, V>, HeldBoth<T, V>>(
      [&](HeldBoth<T, V>& to, long site) { to.load(x + site * a.channels, dy + site * a.channels); },
      [&](HeldBoth<T, V>(&at)[kAheadBoth<T, V>], long site, auto count) {
#pragma unroll
        for (int k = 0; k < kAheadBoth<T, V>; ++k, site += p.slices) {
          at[k].refresh();
          Pack<T, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float dz = act_grad<ACT, T>(norm_z(at[k].v[j], own.mean[j], own.rstd[j], own.w[j], own.b[j]), at[k].g[j]);
            o.v[j] = (T)norm_grad(dz, own.w[j], c1[j], (at[k].v[j] - own.mean[j]) * own.rstd[j], c2[j], own.rstd[j]);
          }
          if (k < count) store_pack(dx + site * a.channels, o);
        }
      });
}

// A block keeps all sites of a tile of whole groups of a sample: accesses of V channels on
// `lanes` lanes (any number), sites on the other threads' slices, E of them each.  x (and dy)
// are read once, and no sums cross blocks but the weights' gradients.  (2 x 64 x 32 fp32 forward:
// 6.2 us, in three launches 14.)
template <int V>
struct WholePlace {
  long n, first, c;  // sample, tile's first channel, this thread's in the tile
  int width, lanes, slices, slice;  // width: channels of the tile that there are
  bool there;
  __device__ __forceinline__ WholePlace(const GroupNormArgs& a, int on, int tiles) : lanes(on) {
    n = (long)blockIdx.x / tiles;
    first = ((long)blockIdx.x - n * tiles) * lanes * V;
    width = (int)min((long)lanes * V, a.channels - first);
    slices = blockDim.x / lanes;
    slice = threadIdx.x / lanes;
    c = (threadIdx.x - slice * lanes) * V;
    there = slice < slices && c < width;
  }
  __device__ __forceinline__ bool site(const GroupNormArgs& a, int e, long& at) const {
    at = (long)e * slices + slice;
    return there && at < a.sites;
  }
};
// Sums over slices and a group's channels of what each thread has for its channels, a wave a
// group: sums[g] of the tile's groups.  all: [slices][lanes V].
template <int V>
__device__ __forceinline__ void group_sums(const GroupNormArgs& a, const WholePlace<V>& p, const float (&x)[V], float* all,
                                           float* sums) {
  const int row = p.lanes * V, each = (int)a.each;
  __syncthreads();  // (what was there has been read)
  if (p.slice < p.slices)
#pragma unroll
    for (int j = 0; j < V; ++j) all[p.slice * row + p.c + j] = p.there ? x[j] : 0.f;
  __syncthreads();
  const unsigned lane = threadIdx.x % kWave, waves = blockDim.x / kWave;
  for (unsigned g = threadIdx.x / kWave; g < (unsigned)(p.width / each); g += waves) {
    float s = 0.f;
    for (unsigned i = lane; i < (unsigned)(p.slices * each); i += kWave) {
      const unsigned k = i / (unsigned)each;
      s += all[k * row + g * each + (i - k * each)];
    }
    s = wave_sum(s);
    if (lane == 0) sums[g] = s;
  }
  __syncthreads();
}

template <typename T, int V, int ACT, int E>
__global__ __launch_bounds__(kMostThreads) void k_last_whole_fwd(GroupNormArgs a, int lanes, int tiles) {
  extern __shared__ float all[];  // [slices][lanes V], then the groups' sums
  const WholePlace<V> p(a, lanes, tiles);
  float* sums = all + p.slices * lanes * V;
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.first + p.c;
  T* y = static_cast<T*>(a.y) + p.n * a.y_stride + p.first + p.c;
  Held<T, V> v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    long at;
    const bool there = p.site(a, e, at);
    v[e].load(x + at * a.channels, there ? V : 0);
  }
  float w[V], b[V], s[V] = {};
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const long c = p.first + (p.there ? p.c + j : 0);
    w[j] = weight_at<T>(a.w, a.wide, c, 1.f);
    b[j] = weight_at<T>(a.b, a.wide, c, 0.f);
  }
  int group[V];  // of the tile
#pragma unroll
  for (int j = 0; j < V; ++j) group[j] = p.there ? (int)(p.c + j) / (int)a.each : 0;
  const float size = (float)a.sites * (float)a.each, inv = 1.f / size;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    v[e].refresh();
#pragma unroll
    for (int j = 0; j < V; ++j) s[j] += v[e][j];  // (0 where there is none)
  }
  group_sums<V>(a, p, s, all, sums);
  float mean[V], rstd[V];
#pragma unroll
  for (int j = 0; j < V; ++j) mean[j] = sums[group[j]] / size, s[j] = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    long at;
    const bool there = p.site(a, e, at);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float d = there ? v[e][j] - mean[j] : 0.f;
      s[j] = fmaf(d, d, s[j]);
    }
  }
  group_sums<V>(a, p, s, all, sums);
#pragma unroll
  for (int j = 0; j < V; ++j) rstd[j] = 1.f / sqrtf(sums[group[j]] * inv + a.eps);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    long at;
    if (!p.site(a, e, at)) continue;
    Pack<T, V> o;
#pragma unroll
    for (int j = 0; j < V; ++j) o.v[j] = (T)act_of<ACT, T>(norm_z(v[e][j], mean[j], rstd[j], w[j], b[j]));
    store_pack(y + at * a.channels, o);
  }
  if (a.stats && p.slice == 0 && p.there)
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const long q = p.n * a.groups + (p.first + p.c + j) / a.each;
      if ((p.c + j) % a.each == 0) a.stats[q] = mean[j], a.stats[a.batch * a.groups + q] = rstd[j];
    }
}

template <typename T, int V, int ACT, int E>
__global__ __launch_bounds__(kMostThreads) void k_last_whole_bwd(GroupNormArgs a, int lanes, int tiles) {
  extern __shared__ float all[];  // [slices][lanes V], then [lanes V][2] of channels and [groups][2]
  const WholePlace<V> p(a, lanes, tiles);
  const int row = lanes * V, each = (int)a.each;
  float *chan = all + p.slices * row, *sums = chan + 2 * row;
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.first + p.c;
  const T* dy = static_cast<const T*>(a.dy) + p.n * a.y_stride + p.first + p.c;
  T* dx = static_cast<T*>(a.dx) + p.n * a.x_stride + p.first + p.c;
  Held<T, V> v[E], d[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    long at;
    const bool there = p.site(a, e, at);
    v[e].load(x + at * a.channels, there ? V : 0);
    d[e].load(dy + at * a.channels, there ? V : 0);
  }
  float w[V], b[V], mean[V], rstd[V], s[2][V] = {};
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const long c = p.first + (p.there ? p.c + j : 0), q = p.n * a.groups + c / a.each;
    mean[j] = a.stats[q];
    rstd[j] = a.stats[a.batch * a.groups + q];
    w[j] = weight_at<T>(a.w, a.wide, c, 1.f);
    b[j] = weight_at<T>(a.b, a.wide, c, 0.f);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    v[e].refresh();
    d[e].refresh();
    long at;
    const bool there = p.site(a, e, at);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float h = (v[e][j] - mean[j]) * rstd[j];
      const float dz = act_grad<ACT, T>(norm_z(v[e][j], mean[j], rstd[j], w[j], b[j]), d[e][j]);
      s[0][j] += there ? dz : 0.f;
      s[1][j] = there ? fmaf(dz, h, s[1][j]) : s[1][j];
    }
    v[e].refresh();
    d[e].refresh();
  }
  // over the slices: many in a few parts first, then a thread a channel
  const int parts = min(p.slices, kMostWholeParts);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (k) __syncthreads();
    if (p.slice < p.slices)
#pragma unroll
      for (int j = 0; j < V; ++j) all[p.slice * row + p.c + j] = p.there ? s[k][j] : 0.f;
    __syncthreads();
    if (p.slices > parts) {
      // (a part's thread alone reads the place that its sum goes to)
      for (int i = threadIdx.x; i < parts * row; i += blockDim.x) {
        float sum = 0.f;
        for (int at = i; at < p.slices * row; at += parts * row) sum += all[at];
        all[i] = sum;
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < p.width; c += blockDim.x) {
      float sum = 0.f;
      for (int i = 0; i < parts; ++i) sum += all[i * row + c];
      chan[2 * c + k] = sum;
      a.own[(p.n * a.channels + p.first + c) * 2 + k] = sum;
    }
  }
  __syncthreads();
  {
#pragma clang fp contract(off)
    const unsigned lane = threadIdx.x % kWave, waves = blockDim.x / kWave;
    const float size = (float)a.sites * (float)a.each;
    for (unsigned g = threadIdx.x / kWave; g < (unsigned)(p.width / each); g += waves) {
      float c1 = 0.f, c2 = 0.f;
      for (int c = lane; c < each; c += kWave) {
        const int at = g * each + c;
        const float wc = weight_at<T>(a.w, a.wide, p.first + at, 1.f);
        c1 += wc * chan[2 * at];
        c2 += wc * chan[2 * at + 1];
      }
      c1 = wave_sum(c1);
      c2 = wave_sum(c2);
      if (lane == 0) sums[2 * g] = c1 / size, sums[2 * g + 1] = c2 / size;
    }
  }
  __syncthreads();
  float c1[V], c2[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int g = p.there ? (int)(p.c + j) / each : 0;
    c1[j] = sums[2 * g];
    c2[j] = sums[2 * g + 1];
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    long at;
    if (!p.site(a, e, at)) continue;
    Pack<T, V> o;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float dz = act_grad<ACT, T>(norm_z(v[e][j], mean[j], rstd[j], w[j], b[j]), d[e][j]);
      o.v[j] = (T)norm_grad(dz, w[j], c1[j], (v[e][j] - mean[j]) * rstd[j], c2[j], rstd[j]);
    }
    store_pack(dx + at * a.channels, o);
  }
}

// Bytes of LDS of a block.
unsigned whole_lds(const bl_group_norm_plan_s* p, bool backward) {
  const long row = (long)p->whole_lanes * p->vec, slices = p->whole_threads[backward] / p->whole_lanes;
  const long groups = std::max<long>(1, row / p->each);
  return (unsigned)((slices * row + (backward ? 2 * row + 2 * groups : groups)) * sizeof(float));
}

// go(T, V) of a plan.
template <typename Go>
void dispatch(const bl_group_norm_plan_s* p, Go&& go) {
  using std::integral_constant;
  auto with = [&](auto t) {
    using T = decltype(t);
    if constexpr (sizeof(T) == 2)
      if (p->vec == 8) return go(t, integral_constant<int, 8>());
    if (p->vec == 4) return go(t, integral_constant<int, 4>());
    if (p->vec == 2) return go(t, integral_constant<int, 2>());
    return go(t, integral_constant<int, 1>());
  };
  if (p->d.dtype == BL_F32) with(float());
  else if (p->d.dtype == BL_BF16) with(bf16_t());
  else with(f16_t());
}

}  // namespace

void gnorm_last_whole(bl_group_norm_plan_s* p) {
  const bl_group_norm_desc_t& d = p->d;
  // whole groups and whole accesses, in lines of 128 bytes where there are as many
  long step = p->each;
  while (step % p->vec) step += p->each;
  long width = step;
  while (width < d.channels && (width + step) * dtype_bytes(d.dtype) <= 128) width += step;
  const long lanes = width / p->vec;
  if (lanes > kThreads) return;
  p->whole_lanes = (int)lanes;
  p->whole_tiles = (int)((d.channels + width - 1) / width);
  for (int i = 0; i < 2; ++i) {
    const auto each = [&](int threads) {
      const long slices = threads / lanes;
      return slices ? (d.sites + slices - 1) / slices : kMostEach + 1L;
    };
    gnorm_whole_threads(each, p->whole_threads[i], p->whole_each[i]);
  }
}

bl_status_t gnorm_last_forward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.batch * a.chunks * a.tiles)), block(kThreads);
  const double bytes = (double)a.batch * a.sites * a.channels * dtype_bytes(p->d.dtype);
  if (p->whole_threads[0])
    return timed_launch("gnorm_fwd", 2.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      with_act(p->d.act, [&](auto act) {
        with_each(p->whole_each[0], [&](auto e) {
          dispatch(p, [&](auto t, auto v) {
            hipExtLaunchKernelGGL((k_last_whole_fwd<decltype(t), decltype(v)::value, decltype(act)::value, decltype(e)::value>),
                                  dim3((unsigned)(a.batch * p->whole_tiles)), dim3(p->whole_threads[0]),
                                  whole_lds(p, false), s, e0, e1, 0, a, p->whole_lanes, p->whole_tiles);
          });
        });
      });
    });
  bl_status_t st = timed_launch("gnorm_part", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    dispatch(p, [&](auto t, auto v) {
      hipExtLaunchKernelGGL((k_last_part<decltype(t), decltype(v)::value>), grid, block, 0, s, e0, e1, 0, a);
    });
  });
  if (st == BL_OK && !p->joins[0]) st = gnorm_join_forward(a, s);
  if (st != BL_OK) return st;
  return timed_launch("gnorm_fwd", 2.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    with_act(p->d.act, [&](auto act) {
      dispatch(p, [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, A = decltype(act)::value;
        hipExtLaunchKernelGGL((p->joins[0] ? k_last_apply<T, V, A, true> : k_last_apply<T, V, A, false>), grid, block, 0, s,
                              e0, e1, 0, a);
      });
    });
  });
}

bl_status_t gnorm_last_backward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.batch * a.chunks * a.tiles)), block(kThreads);
  const double bytes = (double)a.batch * a.sites * a.channels * dtype_bytes(p->d.dtype);
  if (p->whole_threads[1]) {
    bl_status_t st = timed_launch("gnorm_bwd", 3.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      with_act(p->d.act, [&](auto act) {
        with_each(p->whole_each[1], [&](auto e) {
          dispatch(p, [&](auto t, auto v) {
            hipExtLaunchKernelGGL((k_last_whole_bwd<decltype(t), decltype(v)::value, decltype(act)::value, decltype(e)::value>),
                                  dim3((unsigned)(a.batch * p->whole_tiles)), dim3(p->whole_threads[1]),
                                  whole_lds(p, true), s, e0, e1, 0, a, p->whole_lanes, p->whole_tiles);
          });
        });
      });
    });
    GroupNormArgs rest = a;
    if (st == BL_OK) st = gnorm_slabs(p, rest, s);
    return st == BL_OK ? gnorm_weights(rest, p->d.dtype, s) : st;
  }
  bl_status_t st = timed_launch("gnorm_bwd_part", 2.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    with_act(p->d.act, [&](auto act) {
      dispatch(p, [&](auto t, auto v) {
        hipExtLaunchKernelGGL((k_last_bwd_part<decltype(t), decltype(v)::value, decltype(act)::value>), grid, block, 0,
                              s, e0, e1, 0, a);
      });
    });
  });
  if (st == BL_OK && !p->joins[1]) st = gnorm_join_backward(a, p->d.dtype, s);
  GroupNormArgs rest = a;
  if (p->joins[1]) rest.own = a.part, rest.own_rows = a.batch * a.chunks;
  else if (st == BL_OK) st = gnorm_slabs(p, rest, s);
  if (st != BL_OK) return st;
  return timed_launch("gnorm_bwd", 3.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    with_act(p->d.act, [&](auto act) {
      dispatch(p, [&](auto t, auto v) {
        using T = decltype(t);
        constexpr int V = decltype(v)::value, A = decltype(act)::value;
        hipExtLaunchKernelGGL((p->joins[1] ? k_last_bwd_apply<T, V, A, true> : k_last_bwd_apply<T, V, A, false>),
                              dim3(grid.x + gnorm_weights_blocks(a)), block, 0, s, e0, e1, 0, rest, grid.x);
      });
    });
  });
}

}  // namespace blc
