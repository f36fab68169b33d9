// Log probabilities of given classes, entropies and likeliest classes of rows of
// logits, and the gradient of the logits.
#include <new>

#include "ops.hpp"

struct bl_logprob_plan_s {
  bl_logprob_desc_t d;
};

namespace blc {
namespace {

constexpr int kT = 256;

// A value and its class as one number: larger values first, then lower classes;
// -0 as 0, NaN above every number.
__device__ unsigned long long order_key(float z, unsigned j) {
  z += 0.f;
  unsigned u = __float_as_uint(z);
  u = z != z ? 0xFFFFFFFFu : u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
  return ((unsigned long long)u << 32) | (0xFFFFFFFFu - j);
}

template <typename V, typename Op>
__device__ V block_reduce(V x, V* red, Op op) {
  for (int o = 32; o > 0; o >>= 1) x = op(x, __shfl_xor(x, o));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = red[0];
  for (int w = 1; w < kT / 64; ++w) x = op(x, red[w]);
  return x;
}

template <typename T>
__global__ void k_logprob_fwd(const T* logits, const long long* targets, float* logp, float* stats, float* top_logp,
                              long long* top_index, bl_logprob_desc_t d) {
  __shared__ float redf[kT / 64];
  __shared__ unsigned long long redk[kT / 64];
  const long row = blockIdx.x;
  const T* z = logits + row * d.stride;
  auto add = [](float a, float b) { return a + b; };
  auto large = [](float a, float b) { return fmaxf(a, b); };
  float m = -INFINITY;
  for (long j = threadIdx.x; j < d.classes; j += kT) m = fmaxf(m, to_f32(z[j]));
  m = block_reduce(m, redf, large);
  const float base = m == -INFINITY ? 0.f : m;
  float a = 0.f, b = 0.f;
  for (long j = threadIdx.x; j < d.classes; j += kT) {
    const float t = to_f32(z[j]) - base, e = expf(t);
    a += e;
    if (e != 0.f) b += e * t;
  }
  a = block_reduce(a, redf, add);
  b = block_reduce(b, redf, add);
  const bool none = m == -INFINITY && a == 0.f;  // (a NaN beside it is not ruled out)
  const float log_sum = logf(a);
  if (threadIdx.x == 0) {
    const long long t = targets ? targets[row] : -1;
    const bool there = t >= 0 && t < d.classes;
    if (logp) logp[row] = !there ? 0.f : none ? -INFINITY : to_f32(z[t]) - base - log_sum;
    if (stats) {
      stats[row] = m;
      stats[d.rows + row] = log_sum;
      stats[2 * d.rows + row] = none ? 0.f : log_sum - b / a;
    }
  }
  auto larger = [](unsigned long long a, unsigned long long b) { return a > b ? a : b; };
  unsigned long long last = ~0ull;
  for (int k = 0; k < d.top; ++k) {
    unsigned long long best = 0;
    for (long j = threadIdx.x; j < d.classes; j += kT) {
      const unsigned long long key = order_key(to_f32(z[j]), (unsigned)j);
      if (key < last && key > best) best = key;
    }
    last = block_reduce(best, redk, larger);
    if (threadIdx.x == 0) {
      const long j = last ? (long)(0xFFFFFFFFu - (unsigned)last) : -1;
      top_index[row * d.top + k] = j;
      top_logp[row * d.top + k] = j < 0 || none ? -INFINITY : to_f32(z[j]) - base - log_sum;
    }
  }
}

template <typename T>
__global__ void k_logprob_bwd(const T* logits, const long long* targets, const float* stats, const float* g_logp,
                              const float* g_entropy, T* dlogits, bl_logprob_desc_t d) {
  const long row = blockIdx.x;
  const float m = stats[row], log_sum = stats[d.rows + row], entropy = stats[2 * d.rows + row];
  const long long t = targets ? targets[row] : -1;
  const bool none = m == -INFINITY && log_sum == -INFINITY;
  const float g = g_logp && t >= 0 && t < d.classes ? g_logp[row] : 0.f, ge = g_entropy ? g_entropy[row] : 0.f;
  for (long j = threadIdx.x; j < d.classes; j += kT) {
    const float lq = to_f32(logits[row * d.stride + j]) - m - log_sum, q = expf(lq);
    float dz = (j == t ? g : 0.f) - g * q;
    if (g_entropy && q != 0.f) dz -= ge * q * (lq + entropy);
    dlogits[row * d.grad_stride + j] = (T)(none ? 0.f : dz);
  }
}

}  // namespace
}  // namespace blc

using namespace blc;

extern "C" bl_status_t bl_logprob_plan_create(bl_logprob_plan_t* out, const bl_logprob_desc_t* desc) {
  if (!out || !desc) return BL_ERR_INVALID_ARG;
  *out = nullptr;
  bl_logprob_desc_t d = *desc;
  if (d.rows < 0 || d.classes < 1 || d.top < 0 || !known_dtype(d.dtype)) return BL_ERR_INVALID_ARG;
  if (d.stride < 0 || d.grad_stride < 0) return BL_ERR_INVALID_ARG;
  if (!d.stride) d.stride = d.classes;
  if (!d.grad_stride) d.grad_stride = d.classes;
  if (d.rows > 1 && (d.stride < d.classes || d.grad_stride < d.classes)) return BL_ERR_INVALID_ARG;
  const long long most = (1LL << 31) - 1;
  if (d.top > 64 || d.classes > most || d.rows > most) return BL_ERR_UNSUPPORTED;
  bl_logprob_plan_s* p = new (std::nothrow) bl_logprob_plan_s{d};
  if (!p) return BL_ERR_OOM;
  *out = p;
  return BL_OK;
}

extern "C" bl_status_t bl_logprob_plan_destroy(bl_logprob_plan_t p) {
  if (!p) return BL_ERR_INVALID_ARG;
  delete p;
  return BL_OK;
}

extern "C" bl_status_t bl_logprob_workspace_size(bl_logprob_plan_t p, size_t* bytes) {
  if (!p || !bytes) return BL_ERR_INVALID_ARG;
  *bytes = 0;
  return BL_OK;
}

namespace {
template <typename T>
bl_status_t forward(const bl_logprob_plan_s* p, const void* logits, const long long* targets, float* logp,
                    float* stats, float* top_logp, long long* top_index, hipStream_t s) {
  const bl_logprob_desc_t& d = p->d;
  return timed_launch("logprob_fwd", (double)d.rows * d.classes * sizeof(T), 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL(k_logprob_fwd<T>, dim3((unsigned)d.rows), dim3(kT), 0, s, e0, e1, 0,
                          static_cast<const T*>(logits), targets, logp, stats, top_logp, top_index, d);
  });
}
template <typename T>
bl_status_t backward(const bl_logprob_plan_s* p, const void* logits, const long long* targets, const float* stats,
                     const float* g_logp, const float* g_entropy, void* dlogits, hipStream_t s) {
  const bl_logprob_desc_t& d = p->d;
  return timed_launch("logprob_bwd", 2.0 * d.rows * d.classes * sizeof(T), 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL(k_logprob_bwd<T>, dim3((unsigned)d.rows), dim3(kT), 0, s, e0, e1, 0,
                          static_cast<const T*>(logits), targets, stats, g_logp, g_entropy,
                          static_cast<T*>(dlogits), d);
  });
}
}  // namespace

extern "C" bl_status_t bl_logprob_forward(bl_logprob_plan_t p, const void* logits, const long long* targets,
                                          float* logp, float* stats, float* top_logp, long long* top_index, void* ws,
                                          void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (!p->d.rows) return BL_OK;
  if (!logits || (p->d.top && (!top_logp || !top_index))) return BL_ERR_INVALID_ARG;
  (void)ws;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p->d.dtype == BL_F32) return forward<float>(p, logits, targets, logp, stats, top_logp, top_index, s);
  if (p->d.dtype == BL_BF16) return forward<bf16_t>(p, logits, targets, logp, stats, top_logp, top_index, s);
  return forward<f16_t>(p, logits, targets, logp, stats, top_logp, top_index, s);
}

extern "C" bl_status_t bl_logprob_backward(bl_logprob_plan_t p, const void* logits, const long long* targets,
                                           const float* stats, const float* g_logp, const float* g_entropy,
                                           void* dlogits, void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (!p->d.rows) return BL_OK;
  if (!logits || !stats || !dlogits) return BL_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p->d.dtype == BL_F32) return backward<float>(p, logits, targets, stats, g_logp, g_entropy, dlogits, s);
  if (p->d.dtype == BL_BF16) return backward<bf16_t>(p, logits, targets, stats, g_logp, g_entropy, dlogits, s);
  return backward<f16_t>(p, logits, targets, stats, g_logp, g_entropy, dlogits, s);
}
