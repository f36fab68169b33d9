// AdamW over many tensors at once, moments in 32 bits or in 8.
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "ops.hpp"

struct bl_adamw_plan_s {
  int param_dtype, grad_dtype, bits;
  std::vector<long long> sizes;
  std::vector<unsigned char> decay;
  std::vector<long long> first;  // first chunk of each tensor; [count] = all chunks
  size_t off_m, off_v, off_ms, off_vs, bytes;
};

namespace blc {
namespace {

constexpr int kT = 256;
constexpr int kChunk = 1024;  // elements that a block handles; tensors start at multiples of it
constexpr int kBlock = 128;   // elements that share a power of two
constexpr int kTensors = 120; // of one launch: their list is part of the kernel's arguments (4 KB at most)

// The tensors of a launch; tensor i has chunks first[i] ... first[i + 1] - 1 of
// the layout, `tail` elements in the last one, decay in the sign of tail.
struct TensorList {
  void* p[kTensors];
  const void* g[kTensors];
  unsigned first[kTensors + 1];
  short tail[kTensors];
  int count;
};

struct StepArgs {
  float b1, r1, b2, r2;    // beta, 1 - beta
  float eps, keep;         // keep: 1 - lr weight_decay
  float rate, root;        // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  unsigned key;            // of the dither
  unsigned seed;
  double beta1, beta2, wd;
  const float* grad_scale;
  const double* live;
  float *m, *v;            // 32-bit moments
  unsigned char *mc, *vc;  // 8-bit codes
  float *ms, *vs;          // powers of two of their blocks
};

// What follows from lr and the step (on the device for a live step).
__host__ __device__ void step_scalars(StepArgs& a, double lr, double t) {
  a.rate = (float)(lr / (1.0 - pow(a.beta1, t)));
  a.root = (float)(1.0 / sqrt(1.0 - pow(a.beta2, t)));
  a.keep = (float)(1.0 - lr * a.wd);
  a.key = a.seed * 0x6A09E667u + (unsigned)(long long)t * 0xBB67AE85u;
}

__device__ __forceinline__ unsigned dither(unsigned long long place, unsigned key) {
  unsigned x = (unsigned)place * 0x9E3779B9u + key;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}

// 8-bit values: the block's power of two S is divided out exactly, and a power
// of two that turns the code's lowest exponents into fp32's subnormals leaves
// exponent and fraction of the code in the bits above 20 (m: 2^-113, v: 2^-97),
// where the dither is added.
constexpr float kDownM = 0x1p-113f, kUpM = 0x1p113f, kDownV = 0x1p-97f, kUpV = 0x1p97f;
__device__ __forceinline__ float power_of(float largest) {
  return fmaxf(__uint_as_float(__float_as_uint(largest) & 0x7F800000u), 0x1p-96f);
}
// For moments set from values: half of it where the largest is itself a power of
// two (which the code above all fractions then holds), so that values which
// codes stood for are held again as they are, however their block's S was.
__device__ __forceinline__ float power_below(float largest) {
  const unsigned u = __float_as_uint(largest);
  return power_of(__uint_as_float(u ? u - 1 : 0));
}
__device__ __forceinline__ unsigned encode(float a, float scale, float down, unsigned d16) {
  return (__float_as_uint(a / scale * down) + (d16 << 4)) >> 20;
}
__device__ __forceinline__ unsigned encode_m(float m, float scale, unsigned d16) {
  if (!isfinite(m)) return 0x7F;
  return encode(fabsf(m), scale, kDownM, d16) | (__float_as_uint(m) >> 31 << 7);
}
__device__ __forceinline__ unsigned encode_v(float v, float scale, unsigned d16) {
  if (!isfinite(v)) return 0xFF;
  const unsigned c = encode(v, scale, kDownV, d16);
  return v > 0.f && c == 0 ? 1 : c;
}
__device__ __forceinline__ float decode_m(unsigned c, float scale) {
  const unsigned e = c & 0x7F;
  if (e == 0x7F) return NAN;
  return copysignf(__uint_as_float(e << 20) * kUpM * scale, c & 0x80 ? -1.f : 1.f);
}
__device__ __forceinline__ float decode_v(unsigned c, float scale) {
  return c == 0xFF ? NAN : __uint_as_float(c << 20) * kUpV * scale;
}
__device__ __forceinline__ float finite_or_zero(float x) { return isfinite(x) ? x : 0.f; }
// Largest over the 32 lanes that hold a block of 128 values.
__device__ __forceinline__ float block_largest(const float (&x)[4]) {
  float l = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) l = fmaxf(l, finite_or_zero(fabsf(x[j])));
  return wave_max(l, 32);
}

// s b + x r, every operation rounded by itself, so that the codes of moments are
// those of the formula in fp32.
__device__ __forceinline__ float decayed(float s, float b, float x, float r) {
#pragma clang fp contract(off)
  return s * b + x * r;
}

template <typename P>
__device__ P round_param(float x, unsigned h);
template <>
__device__ float round_param<float>(float x, unsigned) {
  return x;
}
template <>
__device__ bf16_t round_param<bf16_t>(float x, unsigned h) {
  if (x != x) return (bf16_t)x;
  const unsigned u = (__float_as_uint(x) + (h * 0x6A09E667u >> 16)) & 0xFFFF0000u;
  return (bf16_t)__uint_as_float(u);
}

template <typename P, typename G, int BITS>
__global__ __launch_bounds__(kT) void k_adamw(const TensorList list, StepArgs a) {
  int t = 0;
  while (t + 1 < list.count && list.first[t + 1] <= blockIdx.x + list.first[0]) ++t;
  const unsigned chunk = blockIdx.x + list.first[0];
  const unsigned in = chunk - list.first[t];
  const int tail = list.tail[t];
  const bool last = chunk + 1 == list.first[t + 1];
  const int n = (last ? abs(tail) : kChunk) - (int)threadIdx.x * 4;  // of this thread's four
  if (a.live) step_scalars(a, a.live[0], a.live[1]);
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const float keep = tail < 0 ? a.keep : 1.f;
  const size_t off = (size_t)in * kChunk + threadIdx.x * 4;       // in the tensor
  const size_t at = (size_t)chunk * kChunk + threadIdx.x * 4;     // in the layout
  P* pp = static_cast<P*>(list.p[t]) + off;
  const Pack<P, 4> p = load_part<P, 4>(pp, n, (P)0.f);
  const Pack<G, 4> g = load_part<G, 4>(static_cast<const G*>(list.g[t]) + off, n, (G)0.f);
  float m[4], v[4];
  if (BITS == 32) {
    const Pack<float, 4> m0 = load_pack<float, 4>(a.m + at), v0 = load_pack<float, 4>(a.v + at);
#pragma unroll
    for (int j = 0; j < 4; ++j) m[j] = m0.v[j], v[j] = v0.v[j];
  } else {
    const unsigned mc = *reinterpret_cast<const unsigned*>(a.mc + at), vc = *reinterpret_cast<const unsigned*>(a.vc + at);
    const float ms = a.ms[at / kBlock], vs = a.vs[at / kBlock];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = decode_m(mc >> (8 * j) & 0xFF, ms);
      v[j] = decode_v(vc >> (8 * j) & 0xFF, vs);
    }
  }
  Pack<P, 4> out;
  unsigned h[4] = {};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (BITS == 8 || sizeof(P) == 2) h[j] = dither(at + j, a.key);
    const float gj = to_f32(g.v[j]) * gs;
    m[j] = decayed(m[j], a.b1, gj, a.r1);
    v[j] = decayed(v[j], a.b2, gj * gj, a.r2);
    const float pj = to_f32(p.v[j]) * keep - m[j] * a.rate / (sqrtf(v[j]) * a.root + a.eps);
    out.v[j] = round_param<P>(pj, h[j]);
  }
  store_part<P, 4>(pp, n, out);
  if (BITS == 32) {
    store_part<float, 4>(a.m + at, n, Pack<float, 4>{{m[0], m[1], m[2], m[3]}});
    store_part<float, 4>(a.v + at, n, Pack<float, 4>{{v[0], v[1], v[2], v[3]}});
  } else {
    const float ms = power_of(block_largest(m)), vs = power_of(block_largest(v));
    unsigned mc = 0, vc = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      mc |= encode_m(m[j], ms, h[j] & 0xFFFF) << (8 * j);
      vc |= encode_v(v[j], vs, h[j] >> 16) << (8 * j);
    }
    *reinterpret_cast<unsigned*>(a.mc + at) = mc;
    *reinterpret_cast<unsigned*>(a.vc + at) = vc;
    if (threadIdx.x % 32 == 0) {
      a.ms[at / kBlock] = ms;
      a.vs[at / kBlock] = vs;
    }
  }
}

__global__ __launch_bounds__(kT) void k_get8(const StepArgs a, bf16_t* m, bf16_t* v) {
  const size_t at = ((size_t)blockIdx.x * kT + threadIdx.x) * 4;
  const unsigned mc = *reinterpret_cast<const unsigned*>(a.mc + at), vc = *reinterpret_cast<const unsigned*>(a.vc + at);
  const float ms = a.ms[at / kBlock], vs = a.vs[at / kBlock];
  Pack<bf16_t, 4> mo, vo;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    mo.v[j] = (bf16_t)decode_m(mc >> (8 * j) & 0xFF, ms);
    vo.v[j] = (bf16_t)decode_v(vc >> (8 * j) & 0xFF, vs);
  }
  store_pack<bf16_t, 4>(m + at, mo);
  store_pack<bf16_t, 4>(v + at, vo);
}

__global__ __launch_bounds__(kT) void k_set8(StepArgs a, const float* m, const float* v) {
  const size_t at = ((size_t)blockIdx.x * kT + threadIdx.x) * 4;
  const Pack<float, 4> mi = load_pack<float, 4>(m + at), vi = load_pack<float, 4>(v + at);
  const float ms = power_below(block_largest(mi.v)), vs = power_below(block_largest(vi.v));
  unsigned mc = 0, vc = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    mc |= encode_m(mi.v[j], ms, 1u << 15) << (8 * j);
    vc |= encode_v(vi.v[j], vs, 1u << 15) << (8 * j);
  }
  *reinterpret_cast<unsigned*>(a.mc + at) = mc;
  *reinterpret_cast<unsigned*>(a.vc + at) = vc;
  if (threadIdx.x % 32 == 0) {
    a.ms[at / kBlock] = ms;
    a.vs[at / kBlock] = vs;
  }
}

__global__ __launch_bounds__(kT) void k_copy2(const float* m, const float* v, float* mo, float* vo) {
  const size_t at = ((size_t)blockIdx.x * kT + threadIdx.x) * 4;
  store_pack<float, 4>(mo + at, load_pack<float, 4>(m + at));
  store_pack<float, 4>(vo + at, load_pack<float, 4>(v + at));
}

StepArgs state_of(const bl_adamw_plan_s* p, const void* state) {
  StepArgs a{};
  char* s = static_cast<char*>(const_cast<void*>(state));
  a.m = reinterpret_cast<float*>(s + p->off_m);
  a.v = reinterpret_cast<float*>(s + p->off_v);
  a.mc = reinterpret_cast<unsigned char*>(s + p->off_m);
  a.vc = reinterpret_cast<unsigned char*>(s + p->off_v);
  a.ms = reinterpret_cast<float*>(s + p->off_ms);
  a.vs = reinterpret_cast<float*>(s + p->off_vs);
  return a;
}

template <typename P, typename G, int BITS>
bl_status_t step(const bl_adamw_plan_s* p, void* const* params, const void* const* grads, const StepArgs& a,
                 hipStream_t s) {
  const int count = (int)p->sizes.size();
  for (int at = 0; at < count;) {
    TensorList list;
    list.count = 0;
    long long values = 0;
    list.first[0] = (unsigned)p->first[at];
    for (; at < count && list.count < kTensors; ++at) {
      if (!p->sizes[at]) continue;
      const int i = list.count++;
      list.p[i] = params[at];
      list.g[i] = grads[at];
      list.first[i] = (unsigned)p->first[at];
      list.first[i + 1] = (unsigned)p->first[at + 1];
      const int tail = (int)((p->sizes[at] - 1) % kChunk + 1);
      list.tail[i] = (short)(p->decay[at] ? -tail : tail);
      values += p->sizes[at];
    }
    if (!list.count) break;
    const unsigned blocks = list.first[list.count] - list.first[0];
    const double bytes = (double)values * (2 * sizeof(P) + sizeof(G) + (BITS == 32 ? 16 : 4 + 16.0 / kBlock));
    const bl_status_t st = timed_launch("adamw", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      hipExtLaunchKernelGGL((k_adamw<P, G, BITS>), dim3(blocks), dim3(kT), 0, s, e0, e1, 0, list, a);
    });
    if (st != BL_OK) return st;
  }
  return BL_OK;
}

template <typename P, typename G>
bl_status_t step_bits(const bl_adamw_plan_s* p, void* const* params, const void* const* grads, const StepArgs& a,
                      hipStream_t s) {
  return p->bits == 32 ? step<P, G, 32>(p, params, grads, a, s) : step<P, G, 8>(p, params, grads, a, s);
}

template <typename P>
bl_status_t step_grad(const bl_adamw_plan_s* p, void* const* params, const void* const* grads, const StepArgs& a,
                      hipStream_t s) {
  if (p->grad_dtype == BL_F32) return step_bits<P, float>(p, params, grads, a, s);
  if (p->grad_dtype == BL_BF16) return step_bits<P, bf16_t>(p, params, grads, a, s);
  return step_bits<P, f16_t>(p, params, grads, a, s);
}

}  // namespace
}  // namespace blc

using namespace blc;

extern "C" bl_status_t bl_adamw_plan_create(bl_adamw_plan_t* out, const bl_adamw_desc_t* d) {
  if (!out || !d) return BL_ERR_INVALID_ARG;
  *out = nullptr;
  if (d->count < 0 || (d->count && !d->sizes)) return BL_ERR_INVALID_ARG;
  if (d->param_dtype != BL_F32 && d->param_dtype != BL_BF16) return BL_ERR_INVALID_ARG;
  if (!known_dtype(d->grad_dtype) || (d->bits != 32 && d->bits != 8)) return BL_ERR_INVALID_ARG;
  long long chunks = 0;
  for (int i = 0; i < d->count; ++i) {
    if (d->sizes[i] < 0) return BL_ERR_INVALID_ARG;
    if (d->sizes[i] >= 1LL << 40) return BL_ERR_UNSUPPORTED;
    chunks += (d->sizes[i] + kChunk - 1) / kChunk;
    if (chunks >= 1LL << 31) return BL_ERR_UNSUPPORTED;
  }
  bl_adamw_plan_s* p = new (std::nothrow) bl_adamw_plan_s();
  if (!p) return BL_ERR_OOM;
  p->param_dtype = d->param_dtype;
  p->grad_dtype = d->grad_dtype;
  p->bits = d->bits;
  try {
    p->first.assign(1, 0);
    for (int i = 0; i < d->count; ++i) {
      p->sizes.push_back(d->sizes[i]);
      p->decay.push_back(!d->decay || d->decay[i]);
      p->first.push_back(p->first.back() + (d->sizes[i] + kChunk - 1) / kChunk);
    }
  } catch (const std::bad_alloc&) {
    delete p;
    return BL_ERR_OOM;
  }
  const size_t total = (size_t)chunks * kChunk, wide = d->bits / 8;
  p->off_m = 0;
  p->off_v = total * wide;
  p->off_ms = 2 * total * wide;
  p->off_vs = p->off_ms + (d->bits == 8 ? total / kBlock * 4 : 0);
  p->bytes = p->off_vs + (d->bits == 8 ? total / kBlock * 4 : 0);
  *out = p;
  return BL_OK;
}

extern "C" bl_status_t bl_adamw_plan_destroy(bl_adamw_plan_t p) {
  if (!p) return BL_ERR_INVALID_ARG;
  delete p;
  return BL_OK;
}

extern "C" bl_status_t bl_adamw_state_size(bl_adamw_plan_t p, size_t* bytes, long long* total, long long* start) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (bytes) *bytes = p->bytes;
  if (total) *total = p->first.back() * kChunk;
  if (start)
    for (size_t i = 0; i < p->sizes.size(); ++i) start[i] = p->first[i] * kChunk;
  return BL_OK;
}

extern "C" bl_status_t bl_adamw_state_layout(bl_adamw_plan_t p, size_t* off_m, size_t* off_v, size_t* off_m_scale,
                                             size_t* off_v_scale) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (off_m) *off_m = p->off_m;
  if (off_v) *off_v = p->off_v;
  if (off_m_scale) *off_m_scale = p->off_ms;
  if (off_v_scale) *off_v_scale = p->off_vs;
  return BL_OK;
}

extern "C" bl_status_t bl_adamw_step(bl_adamw_plan_t p, void* const* params, const void* const* grads, void* state,
                                     const bl_adamw_args_t* args, void* stream) {
  if (!p || !args) return BL_ERR_INVALID_ARG;
  const bl_adamw_args_t& r = *args;
  if (!(r.beta1 >= 0.0 && r.beta1 < 1.0 && r.beta2 >= 0.0 && r.beta2 < 1.0)) return BL_ERR_INVALID_ARG;
  if (!(r.eps >= 0.0) || !std::isfinite(r.eps) || !(r.weight_decay >= 0.0) || !std::isfinite(r.weight_decay))
    return BL_ERR_INVALID_ARG;
  if (!r.live && (r.step < 1 || !(r.lr >= 0.0) || !std::isfinite(r.lr))) return BL_ERR_INVALID_ARG;
  if (!p->first.back()) return BL_OK;
  if (!params || !grads || !state) return BL_ERR_INVALID_ARG;
  for (size_t i = 0; i < p->sizes.size(); ++i)
    if (p->sizes[i] && (!params[i] || !grads[i])) return BL_ERR_INVALID_ARG;
  StepArgs a = state_of(p, state);
  a.b1 = (float)r.beta1;
  a.r1 = (float)(1.0 - r.beta1);
  a.b2 = (float)r.beta2;
  a.r2 = (float)(1.0 - r.beta2);
  a.eps = (float)r.eps;
  a.seed = r.seed;
  a.beta1 = r.beta1;
  a.beta2 = r.beta2;
  a.wd = r.weight_decay;
  a.grad_scale = r.grad_scale;
  a.live = r.live;
  if (!r.live) step_scalars(a, r.lr, (double)r.step);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return p->param_dtype == BL_F32 ? step_grad<float>(p, params, grads, a, s)
                                  : step_grad<bf16_t>(p, params, grads, a, s);
}

extern "C" bl_status_t bl_adamw_get_moments(bl_adamw_plan_t p, const void* state, void* m, void* v, void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  const unsigned blocks = (unsigned)p->first.back();
  if (!blocks) return BL_OK;
  if (!state || !m || !v) return BL_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const StepArgs a = state_of(p, state);
  return timed_launch("adamw_get", (double)blocks * kChunk * (p->bits == 8 ? 6 : 16), 0.0, s,
                      [&](hipEvent_t e0, hipEvent_t e1) {
                        if (p->bits == 8)
                          hipExtLaunchKernelGGL(k_get8, dim3(blocks), dim3(kT), 0, s, e0, e1, 0, a,
                                                static_cast<bf16_t*>(m), static_cast<bf16_t*>(v));
                        else
                          hipExtLaunchKernelGGL(k_copy2, dim3(blocks), dim3(kT), 0, s, e0, e1, 0, a.m, a.v,
                                                static_cast<float*>(m), static_cast<float*>(v));
                      });
}

extern "C" bl_status_t bl_adamw_set_moments(bl_adamw_plan_t p, void* state, const float* m, const float* v,
                                            void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  const unsigned blocks = (unsigned)p->first.back();
  if (!blocks) return BL_OK;
  if (!state || !m || !v) return BL_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const StepArgs a = state_of(p, state);
  return timed_launch("adamw_set", (double)blocks * kChunk * (p->bits == 8 ? 10 : 16), 0.0, s,
                      [&](hipEvent_t e0, hipEvent_t e1) {
                        if (p->bits == 8)
                          hipExtLaunchKernelGGL(k_set8, dim3(blocks), dim3(kT), 0, s, e0, e1, 0, a, m, v);
                        else
                          hipExtLaunchKernelGGL(k_copy2, dim3(blocks), dim3(kT), 0, s, e0, e1, 0, m, v, a.m, a.v);
                      });
}
