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
      for (int j = 0; j < V; ++j) o.v[j] = (T)act_of<ACT>(own.z(v[k][j]));
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
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      v[k].refresh();
      g[k].refresh();
#pragma unroll
      for (int j = 0; j < V; ++j) {
        // (where there is no value z may be anything)
        const float dz = t + k * step + j < p.end ? act_grad<ACT>(own.z(v[k][j]), g[k][j]) : 0.f;
        s1 += dz;
        s2 = t + k * step + j < p.end ? fmaf(dz, own.h(v[k][j]), s2) : s2;
      }
    }
  }
  s1 = lanes_sum(s1, a.lanes, red[0]);
  s2 = lanes_sum(s2, a.lanes, red[1]);
  if (p.lane || !p.there) return;
  float* to = a.part + ((p.n * a.chunks + p.chunk) * a.channels + p.c) * 2;
  to[0] = s1;
  to[1] = s2;
}

template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void k_first_bwd_apply(GroupNormArgs a) {
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
        const float dz = act_grad<ACT>(own.z(v[k][j]), g[k][j]);
        o.v[j] = (T)norm_grad(dz, own.w, c1, own.h(v[k][j]), c2, own.rstd);
      }
      store_part(dx + t + k * step, p.end - t - k * step, o);
    }
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

bl_status_t gnorm_first_forward(const bl_group_norm_plan_s* p, const GroupNormArgs& a, hipStream_t s) {
  const dim3 grid = grid_of(a), block(kThreads);
  const double bytes = (double)a.batch * a.sites * a.channels * dtype_bytes(p->d.dtype);
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
  bl_status_t st = timed_launch("gnorm_bwd_part", 2.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    with_act(p->d.act, [&](auto act) {
      dispatch(p, [&](auto t, auto v) {
        hipExtLaunchKernelGGL((k_first_bwd_part<decltype(t), decltype(v)::value, decltype(act)::value>), grid, block, 0,
                              s, e0, e1, 0, a);
      });
    });
  });
  if (st == BL_OK) st = gnorm_join_backward(a, p->d.dtype, s);
  if (st != BL_OK) return st;
  st = timed_launch("gnorm_bwd", 3.0 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    with_act(p->d.act, [&](auto act) {
      dispatch(p, [&](auto t, auto v) {
        hipExtLaunchKernelGGL((k_first_bwd_apply<decltype(t), decltype(v)::value, decltype(act)::value>), grid, block, 0,
                              s, e0, e1, 0, a);
      });
    });
  });
  return st == BL_OK ? gnorm_weights(a, p->d.dtype, s) : st;
}

}  // namespace blc
