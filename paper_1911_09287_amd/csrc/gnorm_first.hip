// Group norm with an activation, channels first: x [batch][channels][sites].
//
// A channel's sites lie side by side, on `lanes` lanes of a wave (a power of two) or a
// block, and what belongs to the channel is the same for all of them.
#include "gnorm.hpp"

namespace blc {
namespace {

constexpr int kAhead = 4;  // accesses of a thread that are in flight together
constexpr int kWaves = kThreads / kWave;

// Where a thread stands: its sample and channel, and its accesses of V sites begin,
// begin + lanes V, ...
struct FirstPlace {
  long row, n, c, chunk, begin, end;
  int lane;
  bool there;
  template <int V>
  __device__ __forceinline__ static FirstPlace make(const GroupNormArgs& a) {
    FirstPlace p;
    const long q = (long)blockIdx.x / a.chunks;
    p.chunk = (long)blockIdx.x - q * a.chunks;
    const int rows = kThreads / a.lanes, mine = threadIdx.x / a.lanes;
    p.lane = threadIdx.x - mine * a.lanes;
    p.row = q * rows + mine;
    p.there = p.row < a.batch * a.channels;
    p.n = p.there ? p.row / a.channels : 0;
    p.c = p.there ? p.row - p.n * a.channels : 0;
    p.begin = p.chunk * a.chunk + p.lane * V;
    p.end = p.there ? min(a.sites, (p.chunk + 1) * a.chunk) : 0;
    return p;
  }
};

// Sums over the lanes of a channel (a block of them: by way of LDS), in each of them.
__device__ __forceinline__ float lanes_sum(float x, int lanes, float (&red)[kWaves]) {
  x = wave_sum(x, min(lanes, kWave));
  if (lanes <= kWave) return x;
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = x;
  __syncthreads();
  x = 0.f;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) x += red[w];
  return x;
}

template <typename T, int V>
__global__ __launch_bounds__(kThreads) void k_first_part(GroupNormArgs a) {
  __shared__ float red[2][kWaves];
  const FirstPlace p = FirstPlace::make<V>(a);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c * a.sites;
  const long step = (long)a.lanes * V;
  Moments m{0.f, 0.f, 0.f};
  for (long t = p.begin; t < p.end; t += kAhead * step) {
    Held<T, V> v[kAhead];
    float count = 0.f;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      v[k].load(x + t + k * step, p.end - t - k * step);
      count += (float)min(max(p.end - t - k * step, 0L), (long)V);
    }
    Moments own{count, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      v[k].refresh();
#pragma unroll
      for (int j = 0; j < V; ++j) own.mean += v[k][j];  // (0 where there is none)
    }
    own.mean /= count;
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float d = t + k * step + j < p.end ? v[k][j] - own.mean : 0.f;
        own.m2 = fmaf(d, d, own.m2);
      }
    moments_join(m, own);
  }
  const float mean = lanes_sum(m.n * m.mean, a.lanes, red[0]) / (float)max(min(a.sites - p.chunk * a.chunk, a.chunk), 1L);
  const float d = m.mean - mean, m2 = lanes_sum(fmaf(m.n * d, d, m.m2), a.lanes, red[1]);
  if (p.lane || !p.there) return;
  float* to = a.part + ((p.n * a.chunks + p.chunk) * a.channels + p.c) * 2;
  to[0] = mean;
  to[1] = m2;
}

// What a channel needs: statistics and weights.
template <typename T>
struct FirstChannel {
  float mean, rstd, w, b;
  __device__ __forceinline__ FirstChannel(const GroupNormArgs& a, const FirstPlace& p) {
    const long q = p.n * a.groups + p.c / a.each;
    mean = a.stats[q];
    rstd = a.stats[a.batch * a.groups + q];
    w = weight_at<T>(a.w, a.wide, p.c, 1.f);
    b = weight_at<T>(a.b, a.wide, p.c, 0.f);
  }
  __device__ __forceinline__ float z(float x) const { return norm_z(x, mean, rstd, w, b); }
  __device__ __forceinline__ float h(float x) const { return (x - mean) * rstd; }
};

template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_first_apply(GroupNormArgs a) {
  const FirstPlace p = FirstPlace::make<V>(a);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c * a.sites;
  T* y = static_cast<T*>(a.y) + p.n * a.y_stride + p.c * a.sites;
  const FirstChannel<T> own(a, p);
  const long step = (long)a.lanes * V;
  for (long t = p.begin; t < p.end; t += kAhead * step) {
    Held<T, V> v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k].load(x + t + k * step, p.end - t - k * step);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      v[k].refresh();
      Pack<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.v[j] = (T)act_of<ACT, T>(own.z(v[k][j]));
      store_part(y + t + k * step, p.end - t - k * step, o);
    }
  }
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_first_bwd_part(GroupNormArgs a) {
  __shared__ float red[2][kWaves];
  const FirstPlace p = FirstPlace::make<V>(a);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c * a.sites;
  const T* dy = static_cast<const T*>(a.dy) + p.n * a.y_stride + p.c * a.sites;
  const FirstChannel<T> own(a, p);
  const long step = (long)a.lanes * V;
  float s1 = 0.f, s2 = 0.f;
  for (long t = p.begin; t < p.end; t += kAhead * step) {
    Held<T, V> v[kAhead], g[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      v[k].load(x + t + k * step, p.end - t - k * step);
      g[k].load(dy + t + k * step, p.end - t - k * step);
    }
    // (these few by themselves first: a chain of all of a long channel's would round too much)
    float few1 = 0.f, few2 = 0.f;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      v[k].refresh();
      g[k].refresh();
#pragma unroll
      for (int j = 0; j < V; ++j) {
        // (where there is no value z may be anything)
        const float dz = t + k * step + j < p.end ? act_grad<ACT, T>(own.z(v[k][j]), g[k][j]) : 0.f;
        few1 += dz;
        few2 = t + k * step + j < p.end ? fmaf(dz, own.h(v[k][j]), few2) : few2;
      }
    }
    s1 += few1;
    s2 += few2;
  }
  s1 = lanes_sum(s1, a.lanes, red[0]);
  s2 = lanes_sum(s2, a.lanes, red[1]);
  if (p.lane || !p.there) return;
  float* to = a.part + ((p.n * a.chunks + p.chunk) * a.channels + p.c) * 2;
  to[0] = s1;
  to[1] = s2;
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_first_bwd_apply(GroupNormArgs a, unsigned blocks) {
  if (blockIdx.x >= blocks) {
    gnorm_weights_block<T>(a, blockIdx.x - blocks);
    return;
  }
  const FirstPlace p = FirstPlace::make<V>(a);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c * a.sites;
  const T* dy = static_cast<const T*>(a.dy) + p.n * a.y_stride + p.c * a.sites;
  T* dx = static_cast<T*>(a.dx) + p.n * a.x_stride + p.c * a.sites;
  const FirstChannel<T> own(a, p);
  const long q = p.n * a.groups + p.c / a.each;
  const float c1 = a.sums[2 * q], c2 = a.sums[2 * q + 1];
  const long step = (long)a.lanes * V;
  for (long t = p.begin; t < p.end; t += kAhead * step) {
    Held<T, V> v[kAhead], g[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      v[k].load(x + t + k * step, p.end - t - k * step);
      g[k].load(dy + t + k * step, p.end - t - k * step);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      v[k].refresh();
      g[k].refresh();
      Pack<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float dz = act_grad<ACT, T>(own.z(v[k][j]), g[k][j]);
        o.v[j] = (T)norm_grad(dz, own.w, c1, own.h(v[k][j]), c2, own.rstd);
      }
      store_part(dx + t + k * step, p.end - t - k * step, o);
    }
  }
}

// A block keeps a group of a sample: each channel's sites on `lanes` lanes of a wave, so that
// a thread has accesses k of the channels pass rows + its row (entry e = pass per + k of E).
// x (and dy) are read once, and no sums cross blocks but the weights' gradients.  (64 x 256 x 512
// fp32 backward: 27.8 us, 3.6 TB/s, in three launches over 90.)
template <int V>
struct WholePlace {
  long n, g, c, site;  // of an entry: its channel in the group and its first site
  int lanes, rows, row, lane, per;
  __device__ __forceinline__ WholePlace(const GroupNormArgs& a, int on) : lanes(on) {
    n = (long)blockIdx.x / a.groups;
    g = (long)blockIdx.x - n * a.groups;
    rows = blockDim.x / lanes;
    row = threadIdx.x / lanes;
    lane = threadIdx.x % lanes;
    per = (int)((a.sites + lanes * V - 1) / (lanes * V));
  }
  // entry e: values of it that there are (<= 0: none)
  __device__ __forceinline__ long at(const GroupNormArgs& a, int e) {
    const int pass = e / per;
    c = (long)pass * rows + row;
    site = (long)((e - pass * per) * lanes + lane) * V;
    return c < a.each ? a.sites - site : 0;
  }
  __device__ __forceinline__ long offset(const GroupNormArgs& a) const { return (g * a.each + c) * a.sites + site; }
};

template <typename T, int V, int ACT, int E>
__global__ __launch_bounds__(kMostThreads) void k_first_whole_fwd(GroupNormArgs a, int lanes) {
  __shared__ float red[2][kMostThreads / kWave];
  WholePlace<V> p(a, lanes);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride;
  T* y = static_cast<T*>(a.y) + p.n * a.y_stride;
  Held<T, V> v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const long there = p.at(a, e);
    v[e].load(x + p.offset(a), there);
  }
  float w[E], b[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const bool there = p.at(a, e) > 0;
    w[e] = there ? weight_at<T>(a.w, a.wide, p.g * a.each + p.c, 1.f) : 0.f;
    b[e] = there ? weight_at<T>(a.b, a.wide, p.g * a.each + p.c, 0.f) : 0.f;
  }
  const float size = (float)a.sites * (float)a.each;
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    v[e].refresh();
#pragma unroll
    for (int j = 0; j < V; ++j) s += v[e][j];  // (0 where there is none)
  }
  const float mean = block_sum(s, red[0]) / size;
  s = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const long there = p.at(a, e);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float d = j < there ? v[e][j] - mean : 0.f;
      s = fmaf(d, d, s);
    }
  }
  const float rstd = 1.f / sqrtf(block_sum(s, red[1]) * (1.f / size) + a.eps);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const long there = p.at(a, e);
    Pack<T, V> o;
#pragma unroll
    for (int j = 0; j < V; ++j) o.v[j] = (T)act_of<ACT, T>(norm_z(v[e][j], mean, rstd, w[e], b[e]));
    store_part(y + p.offset(a), there, o);
  }
  if (a.stats && threadIdx.x == 0) {
    a.stats[blockIdx.x] = mean;
    a.stats[a.batch * a.groups + blockIdx.x] = rstd;
  }
}

template <typename T, int V, int ACT, int E>
__global__ __launch_bounds__(kMostThreads) void k_first_whole_bwd(GroupNormArgs a, int lanes) {
  extern __shared__ float chan[];  // [each][2]: sums of dz and of dz h
  __shared__ float both[2];
  WholePlace<V> p(a, lanes);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride;
  const T* dy = static_cast<const T*>(a.dy) + p.n * a.y_stride;
  T* dx = static_cast<T*>(a.dx) + p.n * a.x_stride;
  Held<T, V> v[E], d[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const long there = p.at(a, e);
    v[e].load(x + p.offset(a), there);
    d[e].load(dy + p.offset(a), there);
  }
  const float mean = a.stats[blockIdx.x], rstd = a.stats[a.batch * a.groups + blockIdx.x];
  float w[E], b[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const bool there = p.at(a, e) > 0;
    w[e] = there ? weight_at<T>(a.w, a.wide, p.g * a.each + p.c, 1.f) : 0.f;
    b[e] = there ? weight_at<T>(a.b, a.wide, p.g * a.each + p.c, 0.f) : 0.f;
  }
  float s1 = 0.f, s2 = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const long there = p.at(a, e);
    v[e].refresh();
    d[e].refresh();
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float dz = act_grad<ACT, T>(norm_z(v[e][j], mean, rstd, w[e], b[e]), d[e][j]), h = (v[e][j] - mean) * rstd;
      s1 += j < there ? dz : 0.f;
      s2 = j < there ? fmaf(dz, h, s2) : s2;
    }
    v[e].refresh();
    d[e].refresh();
    if ((e + 1) % p.per == 0) {  // the channel's last
      s1 = wave_sum(s1, lanes);
      s2 = wave_sum(s2, lanes);
      if (p.lane == 0 && p.c < a.each) chan[2 * p.c] = s1, chan[2 * p.c + 1] = s2;
      s1 = s2 = 0.f;
    }
  }
  __syncthreads();
  if (threadIdx.x < kWave) {
#pragma clang fp contract(off)
    float c1 = 0.f, c2 = 0.f;
    for (long c = threadIdx.x; c < a.each; c += kWave) {
      const long at = p.g * a.each + c;
      a.own[(p.n * a.channels + at) * 2] = chan[2 * c];
      a.own[(p.n * a.channels + at) * 2 + 1] = chan[2 * c + 1];
      const float wc = weight_at<T>(a.w, a.wide, at, 1.f);
      c1 += wc * chan[2 * c];
      c2 += wc * chan[2 * c + 1];
    }
    c1 = wave_sum(c1);
    c2 = wave_sum(c2);
    if (threadIdx.x == 0) {
      const float size = (float)a.sites * (float)a.each;
      both[0] = c1 / size;
      both[1] = c2 / size;
    }
  }
  __syncthreads();
  const float c1 = both[0], c2 = both[1];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const long there = p.at(a, e);
    Pack<T, V> o;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float dz = act_grad<ACT, T>(norm_z(v[e][j], mean, rstd, w[e], b[e]), d[e][j]);
      o.v[j] = (T)norm_grad(dz, w[e], c1, (v[e][j] - mean) * rstd, c2, rstd);
    }
    store_part(dx + p.offset(a), there, o);
  }
}

// go(T, V) of a plan.
template <typename Go>
void dispatch(const bl_group_norm_plan_s* p, Go&& go) {
  if (p->d.dtype == BL_F32) go(float(), std::integral_constant<int, 4>());
  else if (p->d.dtype == BL_BF16) go(bf16_t(), std::integral_constant<int, 8>());
  else go(f16_t(), std::integral_constant<int, 8>());
}

dim3 grid_of(const GroupNormArgs& a) {
  const long rows = kThreads / a.lanes;
  return dim3((unsigned)((a.batch * a.channels + rows - 1) / rows * a.chunks));
}

}  // namespace

void gnorm_first_whole(bl_group_norm_plan_s* p) {
  const bl_group_norm_desc_t& d = p->d;
  const long vec = 16 / dtype_bytes(d.dtype);
  int lanes = kWave;
  while (lanes > 1 && lanes / 2 * vec >= d.sites) lanes /= 2;
  const long per = (d.sites + lanes * vec - 1) / (lanes * vec);
  p->whole_lanes = lanes;
  p->whole_tiles = (int)d.groups;
  for (int i = 0; i < 2; ++i) {
    const auto each = [&](int threads) { return (p->each + threads / lanes - 1) / (threads / lanes) * per; };
    gnorm_whole_threads(each, p->whole_threads[i], p->whole_each[i]);
  }
}

bl_status_t gnorm_first_forward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s) {
  const dim3 grid = grid_of(a), block(kThreads);
  const double bytes = (double)a.batch * a.sites * a.channels * dtype_bytes(p->d.dtype);
  if (p->whole_threads[0])
    return timed_launch("gnorm_fwd", 2.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      with_act(p->d.act, [&](auto act) {
        with_each(p->whole_each[0], [&](auto e) {
          dispatch(p, [&](auto t, auto v) {
            hipExtLaunchKernelGGL((k_first_whole_fwd<decltype(t), decltype(v)::value, decltype(act)::value, decltype(e)::value>),
                                  dim3((unsigned)(a.batch * a.groups)), dim3(p->whole_threads[0]), 0, s, e0, e1, 0, a,
                                  p->whole_lanes);
          });
        });
      });
    });
  bl_status_t st = timed_launch("gnorm_part", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    dispatch(p, [&](auto t, auto v) {
      hipExtLaunchKernelGGL((k_first_part<decltype(t), decltype(v)::value>), grid, block, 0, s, e0, e1, 0, a);
    });
  });
  if (st == BL_OK) st = gnorm_join_forward(a, s);
  if (st != BL_OK) return st;
  return timed_launch("gnorm_fwd", 2.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    with_act(p->d.act, [&](auto act) {
      dispatch(p, [&](auto t, auto v) {
        hipExtLaunchKernelGGL((k_first_apply<decltype(t), decltype(v)::value, decltype(act)::value>), grid, block, 0, s,
                              e0, e1, 0, a);
      });
    });
  });
}

bl_status_t gnorm_first_backward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s) {
  const dim3 grid = grid_of(a), block(kThreads);
  const double bytes = (double)a.batch * a.sites * a.channels * dtype_bytes(p->d.dtype);
  if (p->whole_threads[1]) {
    bl_status_t st = timed_launch("gnorm_bwd", 3.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      with_act(p->d.act, [&](auto act) {
        with_each(p->whole_each[1], [&](auto e) {
          dispatch(p, [&](auto t, auto v) {
            hipExtLaunchKernelGGL((k_first_whole_bwd<decltype(t), decltype(v)::value, decltype(act)::value, decltype(e)::value>),
                                  dim3((unsigned)(a.batch * a.groups)), dim3(p->whole_threads[1]),
                                  (unsigned)(p->each * 2 * sizeof(float)), s, e0, e1, 0, a, p->whole_lanes);
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
        hipExtLaunchKernelGGL((k_first_bwd_part<decltype(t), decltype(v)::value, decltype(act)::value>), grid, block, 0,
                              s, e0, e1, 0, a);
      });
    });
  });
  if (st == BL_OK) st = gnorm_join_backward(a, p->d.dtype, s);
  GroupNormArgs rest = a;
  if (st == BL_OK) st = gnorm_slabs(p, rest, s);
  if (st != BL_OK) return st;
  // (the blocks past the values' own sum the weights' gradients)
  return timed_launch("gnorm_bwd", 3.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    with_act(p->d.act, [&](auto act) {
      dispatch(p, [&](auto t, auto v) {
        hipExtLaunchKernelGGL((k_first_bwd_apply<decltype(t), decltype(v)::value, decltype(act)::value>),
                              dim3(grid.x + gnorm_weights_blocks(a)), block, 0, s, e0, e1, 0, rest, grid.x);
      });
    });
  });
}

}  // namespace blc
