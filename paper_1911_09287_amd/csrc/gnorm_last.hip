// Group norm with an activation, channels last: x [batch][sites][channels].
//
// A thread keeps an access of channels (`vec` of them, a divisor of their number) and walks
// sites, so that neighbouring threads read neighbouring memory whatever the channels'
// number, and what belongs to its channels (weights, statistics) stays in registers.
#include "gnorm.hpp"

namespace blc {
namespace {

constexpr int kAhead = 4;  // sites of a thread whose loads are in flight together

// Where a thread stands: sample, chunk, its first channel and its sites begin, begin +
// slices, ...
struct LastPlace {
  long n, chunk, c, begin, end;
  int lane, slice, slices;
  bool there;
  template <int V>
  __device__ __forceinline__ static LastPlace make(const GroupNormArgs& a) {
    LastPlace p;
    const long q = (long)blockIdx.x / a.tiles, tile = (long)blockIdx.x - q * a.tiles;
    p.n = q / a.chunks;
    p.chunk = q - p.n * a.chunks;
    p.slices = kThreads / a.lanes;
    p.slice = threadIdx.x / a.lanes;
    p.lane = threadIdx.x - p.slice * a.lanes;
    p.c = (tile * kThreads + p.lane) * V;
    p.there = p.slice < p.slices && p.c < a.channels;
    p.begin = p.chunk * a.chunk + p.slice;
    p.end = p.there ? min(a.sites, (p.chunk + 1) * a.chunk) : 0;
    return p;
  }
};

// Each channel's moments over the block's sites.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void k_last_part(GroupNormArgs a) {
  __shared__ Moments red[kThreads][V];
  const LastPlace p = LastPlace::make<V>(a);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c;
  Moments m[V];
#pragma unroll
  for (int j = 0; j < V; ++j) m[j] = Moments{0.f, 0.f, 0.f};
  for (long t = p.begin; t < p.end; t += (long)kAhead * p.slices) {
    Held<T, V> v[kAhead];
    int count = 0;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long site = t + (long)k * p.slices;
      v[k].load(x + site * a.channels, site < p.end ? V : 0);
      count += site < p.end;
    }
    const float inv = 1.f / (float)count;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v[k].refresh();
#pragma unroll
    for (int j = 0; j < V; ++j) {
      Moments own{(float)count, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < kAhead; ++k) own.mean += v[k][j];
      own.mean *= inv;
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const float d = k < count ? v[k][j] - own.mean : 0.f;
        own.m2 = fmaf(d, d, own.m2);
      }
      moments_join(m[j], own);
    }
  }
  // over the slices, by halves
  int span = 1;
  while (span < p.slices) span *= 2;
#pragma unroll
  for (int j = 0; j < V; ++j) red[threadIdx.x][j] = m[j];
  for (span /= 2; span; span /= 2) {
    __syncthreads();
    if (p.slice < span && p.slice + span < p.slices)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        moments_join(m[j], red[threadIdx.x + span * a.lanes][j]);
        red[threadIdx.x][j] = m[j];
      }
  }
  if (p.slice || !p.there) return;
  float* to = a.part + ((p.n * a.chunks + p.chunk) * a.channels + p.c) * 2;
#pragma unroll
  for (int j = 0; j < V; ++j) to[2 * j] = m[j].mean, to[2 * j + 1] = m[j].m2;
}

// What a thread's channels need: statistics and weights.
template <typename T, int V>
struct LastChannels {
  float mean[V], rstd[V], w[V], b[V];
  __device__ __forceinline__ void load(const GroupNormArgs& a, const LastPlace& p) {
    const long all = a.batch * a.groups;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const long c = p.there ? p.c + j : 0, q = p.n * a.groups + c / a.each;
      mean[j] = a.stats[q];
      rstd[j] = a.stats[all + q];
      w[j] = weight_at<T>(a.w, a.wide, c, 1.f);
      b[j] = weight_at<T>(a.b, a.wide, c, 0.f);
    }
  }
};

template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_last_apply(GroupNormArgs a) {
  const LastPlace p = LastPlace::make<V>(a);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c;
  T* y = static_cast<T*>(a.y) + p.n * a.y_stride + p.c;
  LastChannels<T, V> own;
  own.load(a, p);
  for (long t = p.begin; t < p.end; t += (long)kAhead * p.slices) {
    Held<T, V> v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long site = t + (long)k * p.slices;
      v[k].load(x + site * a.channels, site < p.end ? V : 0);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long site = t + (long)k * p.slices;
      v[k].refresh();
      Pack<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.v[j] = (T)act_of<ACT>(norm_z(v[k][j], own.mean[j], own.rstd[j], own.w[j], own.b[j]));
      if (site < p.end) store_pack(y + site * a.channels, o);
    }
  }
}

// Each channel's sums of dz and of dz h over the block's sites.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_last_bwd_part(GroupNormArgs a) {
  __shared__ float red[kThreads][2 * V];
  const LastPlace p = LastPlace::make<V>(a);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c;
  const T* dy = static_cast<const T*>(a.dy) + p.n * a.y_stride + p.c;
  LastChannels<T, V> own;
  own.load(a, p);
  float s[2 * V] = {};
  for (long t = p.begin; t < p.end; t += (long)kAhead * p.slices) {
    Held<T, V> v[kAhead], g[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long site = t + (long)k * p.slices;
      v[k].load(x + site * a.channels, site < p.end ? V : 0);
      g[k].load(dy + site * a.channels, site < p.end ? V : 0);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      v[k].refresh();
      g[k].refresh();
      if (t + (long)k * p.slices >= p.end) continue;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float h = (v[k][j] - own.mean[j]) * own.rstd[j];
        const float dz = act_grad<ACT>(norm_z(v[k][j], own.mean[j], own.rstd[j], own.w[j], own.b[j]), g[k][j]);
        s[2 * j] += dz;
        s[2 * j + 1] = fmaf(dz, h, s[2 * j + 1]);
      }
    }
  }
  int span = 1;
  while (span < p.slices) span *= 2;
#pragma unroll
  for (int j = 0; j < 2 * V; ++j) red[threadIdx.x][j] = s[j];
  for (span /= 2; span; span /= 2) {
    __syncthreads();
    if (p.slice < span && p.slice + span < p.slices)
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) red[threadIdx.x][j] = s[j] += red[threadIdx.x + span * a.lanes][j];
  }
  if (p.slice || !p.there) return;
  float* to = a.part + ((p.n * a.chunks + p.chunk) * a.channels + p.c) * 2;
#pragma unroll
  for (int j = 0; j < 2 * V; ++j) to[j] = s[j];
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_last_bwd_apply(GroupNormArgs a) {
  const LastPlace p = LastPlace::make<V>(a);
  const T* x = static_cast<const T*>(a.x) + p.n * a.x_stride + p.c;
  const T* dy = static_cast<const T*>(a.dy) + p.n * a.y_stride + p.c;
  T* dx = static_cast<T*>(a.dx) + p.n * a.x_stride + p.c;
  LastChannels<T, V> own;
  own.load(a, p);
  float c1[V], c2[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const long q = p.n * a.groups + (p.there ? p.c + j : 0) / a.each;
    c1[j] = a.sums[2 * q];
    c2[j] = a.sums[2 * q + 1];
  }
  for (long t = p.begin; t < p.end; t += (long)kAhead * p.slices) {
    Held<T, V> v[kAhead], g[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long site = t + (long)k * p.slices;
      v[k].load(x + site * a.channels, site < p.end ? V : 0);
      g[k].load(dy + site * a.channels, site < p.end ? V : 0);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const long site = t + (long)k * p.slices;
      v[k].refresh();
      g[k].refresh();
      Pack<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float dz = act_grad<ACT>(norm_z(v[k][j], own.mean[j], own.rstd[j], own.w[j], own.b[j]), g[k][j]);
        o.v[j] = (T)norm_grad(dz, own.w[j], c1[j], (v[k][j] - own.mean[j]) * own.rstd[j], c2[j], own.rstd[j]);
      }
      if (site < p.end) store_pack(dx + site * a.channels, o);
    }
  }
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

bl_status_t gnorm_last_forward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.batch * a.chunks * a.tiles)), block(kThreads);
  const double bytes = (double)a.batch * a.sites * a.channels * dtype_bytes(p->d.dtype);
  bl_status_t st = timed_launch("gnorm_part", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    dispatch(p, [&](auto t, auto v) {
      hipExtLaunchKernelGGL((k_last_part<decltype(t), decltype(v)::value>), grid, block, 0, s, e0, e1, 0, a);
    });
  });
  if (st == BL_OK) st = gnorm_join_forward(a, s);
  if (st != BL_OK) return st;
  return timed_launch("gnorm_fwd", 2.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    with_act(p->d.act, [&](auto act) {
      dispatch(p, [&](auto t, auto v) {
        hipExtLaunchKernelGGL((k_last_apply<decltype(t), decltype(v)::value, decltype(act)::value>), grid, block, 0, s,
                              e0, e1, 0, a);
      });
    });
  });
}

bl_status_t gnorm_last_backward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.batch * a.chunks * a.tiles)), block(kThreads);
  const double bytes = (double)a.batch * a.sites * a.channels * dtype_bytes(p->d.dtype);
  bl_status_t st = timed_launch("gnorm_bwd_part", 2.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    with_act(p->d.act, [&](auto act) {
      dispatch(p, [&](auto t, auto v) {
        hipExtLaunchKernelGGL((k_last_bwd_part<decltype(t), decltype(v)::value, decltype(act)::value>), grid, block, 0,
                              s, e0, e1, 0, a);
      });
    });
  });
  if (st == BL_OK) st = gnorm_join_backward(a, p->d.dtype, s);
  if (st != BL_OK) return st;
  st = timed_launch("gnorm_bwd", 3.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    with_act(p->d.act, [&](auto act) {
      dispatch(p, [&](auto t, auto v) {
        hipExtLaunchKernelGGL((k_last_bwd_apply<decltype(t), decltype(v)::value, decltype(act)::value>), grid, block, 0,
                              s, e0, e1, 0, a);
      });
    });
  });
  return st == BL_OK ? gnorm_weights(a, p->d.dtype, s) : st;
}

}  // namespace blc
