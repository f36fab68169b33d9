// Layer norm over the middle axis of [outer][size][inner]: forward and backward.
#include <cmath>
#include <new>

#include "ops.hpp"

struct bl_norm_plan_s {
  bl_norm_desc_t d;
};

namespace blc {
namespace {

constexpr int kT = 256;

__device__ float block_sum(float x, float* red) {
  x = wave_sum(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  float t = 0.f;
  for (int w = 0; w < kT / 64; ++w) t += red[w];
  return t;
}

__device__ float load_w(const void* w, int dtype, long i) {
  return dtype == BL_F32 ? static_cast<const float*>(w)[i]
                         : dtype == BL_BF16 ? to_f32(static_cast<const bf16_t*>(w)[i])
                                            : to_f32(static_cast<const f16_t*>(w)[i]);
}
__device__ void store_w(void* w, int dtype, long i, float x) {
  if (dtype == BL_F32) static_cast<float*>(w)[i] = x;
  else if (dtype == BL_BF16) static_cast<bf16_t*>(w)[i] = (bf16_t)x;
  else static_cast<f16_t*>(w)[i] = (f16_t)x;
}

template <typename T>
__global__ void k_norm_fwd(const T* x, const void* w, const void* b, T* y, float* stats, bl_norm_desc_t d) {
  __shared__ float red[kT / 64];
  const long site = blockIdx.x, o = site / d.inner, i = site % d.inner, sites = d.outer * d.inner;
  const T* xr = x + o * d.x_stride + i;
  float s = 0.f;
  for (long j = threadIdx.x; j < d.size; j += kT) s += to_f32(xr[j * d.inner]);
  const float mean = block_sum(s, red) / d.size;
  s = 0.f;
  for (long j = threadIdx.x; j < d.size; j += kT) {
    const float c = to_f32(xr[j * d.inner]) - mean;
    s += c * c;
  }
  const float rstd = 1.f / sqrtf(block_sum(s, red) / d.size + (float)d.eps);
  for (long j = threadIdx.x; j < d.size; j += kT) {
    const float h = (to_f32(xr[j * d.inner]) - mean) * rstd;
    y[o * d.y_stride + j * d.inner + i] = (T)(h * (w ? load_w(w, d.wdtype, j) : 1.f) + (b ? load_w(b, d.wdtype, j) : 0.f));
  }
  if (stats && threadIdx.x == 0) {
    stats[site] = mean;
    stats[sites + site] = rstd;
  }
}

template <typename T>
__global__ void k_norm_dx(const T* dy, const T* x, const void* w, const float* stats, T* dx, bl_norm_desc_t d) {
  __shared__ float red[kT / 64];
  const long site = blockIdx.x, o = site / d.inner, i = site % d.inner, sites = d.outer * d.inner;
  const float mean = stats[site], rstd = stats[sites + site];
  float s1 = 0.f, s2 = 0.f;
  for (long j = threadIdx.x; j < d.size; j += kT) {
    const float h = (to_f32(x[o * d.x_stride + j * d.inner + i]) - mean) * rstd;
    const float u = to_f32(dy[o * d.y_stride + j * d.inner + i]) * (w ? load_w(w, d.wdtype, j) : 1.f);
    s1 += u;
    s2 += u * h;
  }
  s1 = block_sum(s1, red) / d.size;
  s2 = block_sum(s2, red) / d.size;
  for (long j = threadIdx.x; j < d.size; j += kT) {
    const float h = (to_f32(x[o * d.x_stride + j * d.inner + i]) - mean) * rstd;
    const float u = to_f32(dy[o * d.y_stride + j * d.inner + i]) * (w ? load_w(w, d.wdtype, j) : 1.f);
    dx[o * d.x_stride + j * d.inner + i] = (T)(rstd * (u - s1 - h * s2));
  }
}

template <typename T>
__global__ void k_norm_dw(const T* dy, const T* x, const float* stats, void* dw, void* db, bl_norm_desc_t d) {
  __shared__ float red[kT / 64];
  const long j = blockIdx.x, sites = d.outer * d.inner;
  float s1 = 0.f, s2 = 0.f;
  for (long site = threadIdx.x; site < sites; site += kT) {
    const long o = site / d.inner, i = site % d.inner;
    const float h = (to_f32(x[o * d.x_stride + j * d.inner + i]) - stats[site]) * stats[sites + site];
    const float g = to_f32(dy[o * d.y_stride + j * d.inner + i]);
    s1 += g * h;
    s2 += g;
  }
  s1 = block_sum(s1, red);
  s2 = block_sum(s2, red);
  if (threadIdx.x == 0) {
    if (dw) store_w(dw, d.wdtype, j, s1);
    if (db) store_w(db, d.wdtype, j, s2);
  }
}

}  // namespace
}  // namespace blc

using namespace blc;

extern "C" bl_status_t bl_norm_plan_create(bl_norm_plan_t* out, const bl_norm_desc_t* desc) {
  if (!out || !desc) return BL_ERR_INVALID_ARG;
  *out = nullptr;
  bl_norm_desc_t d = *desc;
  if (d.outer < 0 || d.size < 1 || d.inner < 1 || !known_dtype(d.dtype)) return BL_ERR_INVALID_ARG;
  if (d.wdtype != BL_F32 && d.wdtype != d.dtype) return BL_ERR_INVALID_ARG;
  if (!(d.eps >= 0.0) || !std::isfinite(d.eps)) return BL_ERR_INVALID_ARG;
  if (d.x_stride < 0 || d.y_stride < 0) return BL_ERR_INVALID_ARG;
  const long long most = (1LL << 31) - 1;
  if (d.size > most || d.inner > most || d.size * d.inner > most) return BL_ERR_UNSUPPORTED;
  if (d.outer > most || d.outer * d.inner > most) return BL_ERR_UNSUPPORTED;
  if (!d.x_stride) d.x_stride = d.size * d.inner;
  if (!d.y_stride) d.y_stride = d.size * d.inner;
  if (d.outer > 1 && (d.x_stride < d.size * d.inner || d.y_stride < d.size * d.inner)) return BL_ERR_INVALID_ARG;
  bl_norm_plan_s* p = new (std::nothrow) bl_norm_plan_s{d};
  if (!p) return BL_ERR_OOM;
  *out = p;
  return BL_OK;
}

extern "C" bl_status_t bl_norm_plan_destroy(bl_norm_plan_t p) {
  if (!p) return BL_ERR_INVALID_ARG;
  delete p;
  return BL_OK;
}

extern "C" bl_status_t bl_norm_workspace_size(bl_norm_plan_t p, size_t* bytes) {
  if (!p || !bytes) return BL_ERR_INVALID_ARG;
  *bytes = 0;
  return BL_OK;
}

namespace {
template <typename T>
bl_status_t forward(const bl_norm_plan_s* p, const void* x, const void* w, const void* b, void* y, float* stats,
                    hipStream_t s) {
  const bl_norm_desc_t& d = p->d;
  const double n = (double)d.outer * d.size * d.inner;
  if (!d.outer) return BL_OK;
  return timed_launch("norm_fwd", 2 * n * sizeof(T), 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL(k_norm_fwd<T>, dim3((unsigned)(d.outer * d.inner)), dim3(kT), 0, s, e0, e1, 0,
                          static_cast<const T*>(x), w, b, static_cast<T*>(y), stats, d);
  });
}
template <typename T>
bl_status_t backward(const bl_norm_plan_s* p, const void* dy, const void* x, const void* w, const float* stats,
                     void* dx, void* dw, void* db, hipStream_t s) {
  const bl_norm_desc_t& d = p->d;
  const double n = (double)d.outer * d.size * d.inner;
  const T* dyt = static_cast<const T*>(dy);
  const T* xt = static_cast<const T*>(x);
  if (dw || db) {
    const bl_status_t st = timed_launch("norm_dw", 2 * n * sizeof(T), 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      hipExtLaunchKernelGGL(k_norm_dw<T>, dim3((unsigned)d.size), dim3(kT), 0, s, e0, e1, 0, dyt, xt, stats, dw, db, d);
    });
    if (st != BL_OK) return st;
  }
  if (!d.outer) return BL_OK;
  return timed_launch("norm_dx", 3 * n * sizeof(T), 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL(k_norm_dx<T>, dim3((unsigned)(d.outer * d.inner)), dim3(kT), 0, s, e0, e1, 0, dyt, xt, w,
                          stats, static_cast<T*>(dx), d);
  });
}
}  // namespace

extern "C" bl_status_t bl_norm_forward(bl_norm_plan_t p, const void* x, const void* w, const void* b, void* y,
                                       float* stats, void* ws, void* stream) {
  if (!p || (p->d.outer && (!x || !y))) return BL_ERR_INVALID_ARG;
  (void)ws;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p->d.dtype == BL_F32) return forward<float>(p, x, w, b, y, stats, s);
  if (p->d.dtype == BL_BF16) return forward<bf16_t>(p, x, w, b, y, stats, s);
  return forward<f16_t>(p, x, w, b, y, stats, s);
}

extern "C" bl_status_t bl_norm_backward(bl_norm_plan_t p, const void* dy, const void* x, const void* w,
                                        const float* stats, void* dx, void* dw, void* db, void* ws, void* stream) {
  if (!p || (p->d.outer && (!dy || !x || !stats || !dx))) return BL_ERR_INVALID_ARG;
  (void)ws;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p->d.dtype == BL_F32) return backward<float>(p, dy, x, w, stats, dx, dw, db, s);
  if (p->d.dtype == BL_BF16) return backward<bf16_t>(p, dy, x, w, stats, dx, dw, db, s);
  return backward<f16_t>(p, dy, x, w, stats, dx, dw, db, s);
}
