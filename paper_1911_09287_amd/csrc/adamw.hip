// AdamW over many tensors at once, moments in 32 bits or in 8.
#include <algorithm>
#include <cmath>
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
constexpr int kWaves = kT / kWave;
constexpr int kChunk = 1024;    // tensors start at multiples of this many elements of the layout
constexpr int kBlock = 128;     // elements that share a power of two: four on each of 32 lanes
constexpr int kTensors = 128;   // of one launch: their list is part of the kernel's arguments (4 KB at most)
constexpr int kFewTensors = 16; // 3 KB of arguments cost 1.7 us a launch: few tensors go in a short list

constexpr long long kMostChunks = (1LL << 26) - 1;  // of one launch, which has fewer than 2^32 threads
constexpr long long kMostBlocks = (1LL << 24) - 1;  // likewise, in blocks of kT threads

// The tensors of a launch; tensor i has chunks first[i] ... first[i + 1] - 1 of
// the layout (all ones past the last), |tail| elements in the last one, weight
// decay where tail < 0.
template <int N>
struct TensorList {
  void* p[N];
  const void* g[N];
  unsigned first[N + 1];
  short tail[N];
  unsigned chunks;
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
// exponent and fraction of the code in the bits from 20 on (m: 2^-113, v: 2^-97),
// where the dither is added.
constexpr unsigned kInf = 0x7F800000u, kLeast = 0x0F800000u;  // bits of infinity and of 2^-96
constexpr float kDownM = 0x1p-113f, kUpM = 0x1p113f, kDownV = 0x1p-97f, kUpV = 0x1p97f;
__device__ __forceinline__ unsigned bits_of(float x) { return __float_as_uint(x); }
__device__ __forceinline__ float from_bits(unsigned u) { return __uint_as_float(u); }
// S of a block from its largest magnitude's bits, and 1 / S.
__device__ __forceinline__ unsigned power_bits(unsigned largest) { return max(largest & kInf, kLeast); }
// (2^(e - 127) for e <= 253; 1 / 2^127 is subnormal)
__device__ __forceinline__ float inverse_power(unsigned s) { return s < 0x7F000000u ? from_bits(0x7F000000u - s) : 0x1p-127f; }
// For moments set from values: half of it where the largest is itself a power of
// two (which the code above all fractions then holds), so that values which
// codes stood for are held again as they are, however their block's S was.
__device__ __forceinline__ unsigned power_bits_below(unsigned largest) { return power_bits(largest ? largest - 1 : 0); }

__device__ __forceinline__ unsigned encode(float a, float inverse, float down, unsigned d16) {
  return (bits_of(a * inverse * down) + (d16 << 4)) >> 20;
}
__device__ __forceinline__ unsigned encode_m(float m, float inverse, unsigned d16) {
  const unsigned a = bits_of(m) & 0x7FFFFFFFu;
  const unsigned c = encode(from_bits(a), inverse, kDownM, d16) | (bits_of(m) >> 31 << 7);
  return a >= kInf ? 0x7Fu : c;
}
__device__ __forceinline__ unsigned encode_v(float v, float inverse, unsigned d16) {
  const unsigned c = max(encode(v, inverse, kDownV, d16), v > 0.f ? 1u : 0u);
  return bits_of(v) >= kInf ? 0xFFu : c;
}
// The code of all ones (exponent and fraction) is NaN.
__device__ __forceinline__ float decode_m(unsigned c, float scale) {
  const unsigned e = c & 0x7Fu;
  const float x = from_bits(e << 20) * kUpM * scale;
  return e == 0x7Fu ? NAN : from_bits(bits_of(x) | (c & 0x80u) << 24);
}
__device__ __forceinline__ float decode_v(unsigned c, float scale) {
  return c == 0xFFu ? NAN : from_bits(c << 20) * kUpV * scale;
}

// Largest over the 32 lanes that hold a block: rotations within rows of 16 lanes, then the other row.
__device__ __forceinline__ unsigned max32(unsigned x) {
#define BL_ROT(n) x = max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + n, 0xF, 0xF, false))
  BL_ROT(8);
  BL_ROT(4);
  BL_ROT(2);
  BL_ROT(1);
#undef BL_ROT
  return max(x, (unsigned)__builtin_amdgcn_ds_swizzle((int)x, 0x401F));  // lane xor 16
}
// Bits of the largest finite magnitude of a block, four values on each of 32 lanes.
__device__ __forceinline__ unsigned block_largest(const float (&x)[4]) {
  unsigned u[4], l = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) l = max(l, u[j] = bits_of(x[j]) & 0x7FFFFFFFu);
  if (__ballot(l >= kInf)) {  // rare: leave out what is not finite
    l = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) l = max(l, u[j] < kInf ? u[j] : 0u);
  }
  return max32(l);
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
__device__ __forceinline__ float round_param<float>(float x, unsigned) {
  return x;
}
template <>
__device__ __forceinline__ bf16_t round_param<bf16_t>(float x, unsigned h) {
  if (x != x) return (bf16_t)x;
  return (bf16_t)from_bits((bits_of(x) + (h * 0x6A09E667u >> 16)) & 0xFFFF0000u);
}

// One step.  A wave takes 256 V elements of one chunk: V vectors of four on each
// lane, 256 elements apart, so that its loads and stores are whole lines and a
// block of 128 lies on half a wave.
// sqrt and reciprocal are the vector unit's, off by an ulp each.  Bound by HBM:
// 126 million values with moments of 8 bits, gradients in bfloat16: 327 us,
// 5.4 TB/s (a large copy reaches 5.0).
template <typename P, typename G, int BITS, int V, bool LIVE, int N>
__global__ __launch_bounds__(kT) void k_adamw(const TensorList<N> list, StepArgs a) {
  constexpr int kParts = kChunk / (256 * V);
  const unsigned lane = threadIdx.x & 63;
  const unsigned wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
  if (wave / kParts >= list.chunks) return;
  const unsigned chunk = list.first[0] + wave / kParts;
  const unsigned from = wave % kParts * (256 * V) + lane * 4;  // of this lane's first vector, in the chunk
  const size_t at = (size_t)chunk * kChunk + from;             // in the layout
  // the moments lie at the chunk's place: their loads go out before the tensor is known
  Pack<float, 4> m0[V], v0[V];
  unsigned mc[V], vc[V];
  float ms[V], vs[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    if (BITS == 32) {
      m0[k] = load_pack<float, 4>(a.m + at + 256 * k);
      v0[k] = load_pack<float, 4>(a.v + at + 256 * k);
    } else {
      mc[k] = *reinterpret_cast<const unsigned*>(a.mc + at + 256 * k);
      vc[k] = *reinterpret_cast<const unsigned*>(a.vc + at + 256 * k);
      ms[k] = a.ms[at / kBlock + 2 * k];
      vs[k] = a.vs[at / kBlock + 2 * k];
    }
  }
  // the tensor: how many start at or before this chunk, less one
  int before = __popcll(__ballot((int)lane < N && list.first[1 + (lane < N ? lane : 0)] <= chunk));
  if (N > kWave) before += __popcll(__ballot(list.first[1 + (N > kWave ? kWave : 0) + lane] <= chunk));
  const unsigned t = __builtin_amdgcn_readfirstlane(before);
  const int tail = list.tail[t];
  const int n = (chunk + 1 == list.first[t + 1] ? abs(tail) : kChunk) - (int)from;  // from this lane's first on
  const size_t off = (size_t)(chunk - list.first[t]) * kChunk + from;               // in the tensor
  P* const pp = static_cast<P*>(list.p[t]) + off;
  const G* const gp = static_cast<const G*>(list.g[t]) + off;
  Pack<P, 4> p[V];
  Pack<G, 4> g[V];
#pragma unroll
  for (int k = 0; k < V; ++k) {
    p[k] = load_part<P, 4>(pp + 256 * k, n - 256 * k, (P)0.f);
    g[k] = load_part<G, 4>(gp + 256 * k, n - 256 * k, (G)0.f);
  }
  if (LIVE) step_scalars(a, a.live[0], a.live[1]);
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const float keep = tail < 0 ? a.keep : 1.f;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    float m[4], v[4];
    unsigned h[4] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (BITS == 8 || sizeof(P) == 2) h[j] = dither(at + 256 * k + j, a.key);
      m[j] = BITS == 32 ? m0[k].v[j] : decode_m(mc[k] >> (8 * j) & 0xFFu, ms[k]);
      v[j] = BITS == 32 ? v0[k].v[j] : decode_v(vc[k] >> (8 * j) & 0xFFu, vs[k]);
      const float gj = to_f32(g[k].v[j]) * gs;
      m[j] = decayed(m[j], a.b1, gj, a.r1);
      v[j] = decayed(v[j], a.b2, gj * gj, a.r2);
      if (BITS == 8 && j >= n - 256 * k) m[j] = v[j] = 0.f;  // past the tensor: no part of its block
      const float down = fmaf(__builtin_amdgcn_sqrtf(v[j]), a.root, a.eps);
      const float x = fmaf(to_f32(p[k].v[j]), keep, -(m[j] * a.rate) * __builtin_amdgcn_rcpf(down));
      p[k].v[j] = round_param<P>(x, h[j]);
    }
    store_part<P, 4>(pp + 256 * k, n - 256 * k, p[k]);
    if (BITS == 32) {
      store_part<float, 4>(a.m + at + 256 * k, n - 256 * k, Pack<float, 4>{{m[0], m[1], m[2], m[3]}});
      store_part<float, 4>(a.v + at + 256 * k, n - 256 * k, Pack<float, 4>{{v[0], v[1], v[2], v[3]}});
    } else {
      const unsigned sm = power_bits(block_largest(m)), sv = power_bits(block_largest(v));
      const float im = inverse_power(sm), iv = inverse_power(sv);
      unsigned cm = 0, cv = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        cm |= encode_m(m[j], im, h[j] & 0xFFFF) << (8 * j);
        cv |= encode_v(v[j], iv, h[j] >> 16) << (8 * j);
      }
      *reinterpret_cast<unsigned*>(a.mc + at + 256 * k) = cm;
      *reinterpret_cast<unsigned*>(a.vc + at + 256 * k) = cv;
      if (lane % 32 == 0) {
        a.ms[at / kBlock + 2 * k] = from_bits(sm);
        a.vs[at / kBlock + 2 * k] = from_bits(sv);
      }
    }
  }
}

// 8-bit moments as bfloat16 values, eight a thread.
__global__ __launch_bounds__(kT) void k_get8(const StepArgs a, bf16_t* m, bf16_t* v, size_t from, size_t total) {
  const size_t at = from + ((size_t)blockIdx.x * kT + threadIdx.x) * 8;
  if (at >= total) return;
  const uint2 mc = *reinterpret_cast<const uint2*>(a.mc + at), vc = *reinterpret_cast<const uint2*>(a.vc + at);
  const float ms = a.ms[at / kBlock], vs = a.vs[at / kBlock];
  Pack<bf16_t, 8> mo, vo;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    mo.v[j] = (bf16_t)decode_m((j < 4 ? mc.x : mc.y) >> (8 * (j & 3)) & 0xFFu, ms);
    vo.v[j] = (bf16_t)decode_v((j < 4 ? vc.x : vc.y) >> (8 * (j & 3)) & 0xFFu, vs);
  }
  store_pack<bf16_t, 8>(m + at, mo);
  store_pack<bf16_t, 8>(v + at, vo);
}

__global__ __launch_bounds__(kT) void k_set8(StepArgs a, const float* m, const float* v, size_t from) {
  const size_t at = from + ((size_t)blockIdx.x * kT + threadIdx.x) * 4;
  const Pack<float, 4> mi = load_pack<float, 4>(m + at), vi = load_pack<float, 4>(v + at);
  const unsigned sm = power_bits_below(block_largest(mi.v)), sv = power_bits_below(block_largest(vi.v));
  const float im = inverse_power(sm), iv = inverse_power(sv);
  unsigned cm = 0, cv = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    cm |= encode_m(mi.v[j], im, 1u << 15) << (8 * j);
    cv |= encode_v(vi.v[j], iv, 1u << 15) << (8 * j);
  }
  *reinterpret_cast<unsigned*>(a.mc + at) = cm;
  *reinterpret_cast<unsigned*>(a.vc + at) = cv;
  if (threadIdx.x % 32 == 0) {
    a.ms[at / kBlock] = from_bits(sm);
    a.vs[at / kBlock] = from_bits(sv);
  }
}

__global__ __launch_bounds__(kT) void k_copy2(const float* m, const float* v, float* mo, float* vo, size_t from) {
  const size_t at = from + ((size_t)blockIdx.x * kT + threadIdx.x) * 4;
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

TensorList<kFewTensors> few_of(const TensorList<kTensors>& l) {
  TensorList<kFewTensors> f;
  std::copy_n(l.p, kFewTensors, f.p);
  std::copy_n(l.g, kFewTensors, f.g);
  std::copy_n(l.first, kFewTensors + 1, f.first);
  std::copy_n(l.tail, kFewTensors, f.tail);
  f.chunks = l.chunks;
  return f;
}

// Chunks from which on a wave takes a whole chunk: fewer are spread thinner.
constexpr unsigned kWholeChunks = 4096;

template <typename P, typename G, int BITS>
bl_status_t step(const bl_adamw_plan_s* p, void* const* params, const void* const* grads, const StepArgs& a,
                 hipStream_t s) {
  const int count = (int)p->sizes.size();
  for (int at = 0; at < count;) {
    TensorList<kTensors> list{};
    int n = 0;
    double values = 0;
    for (; at < count && n < kTensors; ++at) {
      if (!p->sizes[at]) continue;
      const long long first = p->first[at];
      if (n && p->first[at + 1] - list.first[0] > kMostChunks) break;
      list.p[n] = params[at];
      list.g[n] = grads[at];
      list.first[n] = (unsigned)first;
      const int tail = (int)((p->sizes[at] - 1) % kChunk + 1);
      list.tail[n] = (short)(p->decay[at] ? -tail : tail);
      list.first[++n] = (unsigned)p->first[at + 1];
      values += (double)p->sizes[at];
    }
    if (!n) break;
    list.chunks = list.first[n] - list.first[0];
    for (int i = n + 1; i <= kTensors; ++i) list.first[i] = ~0u;
    const double bytes = values * (2 * sizeof(P) + sizeof(G) + (BITS == 32 ? 16 : 4 + 16.0 / kBlock));
    const bool whole = list.chunks >= kWholeChunks;
    const unsigned blocks = (unsigned)(((size_t)list.chunks * (whole ? 1 : 4) + kWaves - 1) / kWaves);
    const bl_status_t st = timed_launch("adamw", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      auto go = [&](auto kernel, const auto& l) {
        hipExtLaunchKernelGGL(kernel, dim3(blocks), dim3(kT), 0, s, e0, e1, 0, l, a);
      };
      if (a.live) whole ? go(k_adamw<P, G, BITS, 4, true, kTensors>, list) : go(k_adamw<P, G, BITS, 1, true, kTensors>, list);
      else if (whole) go(k_adamw<P, G, BITS, 4, false, kTensors>, list);
      else if (n > kFewTensors) go(k_adamw<P, G, BITS, 1, false, kTensors>, list);
      else go(k_adamw<P, G, BITS, 1, false, kFewTensors>, few_of(list));
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
    if (d->sizes[i] >= 1LL << 35) return BL_ERR_UNSUPPORTED;
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
  if (!params || !grads || !state || !aligned(state)) return BL_ERR_INVALID_ARG;
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

namespace {
// All of the moments' layout, `each` elements a block, in launches of at most kMostBlocks blocks.
template <typename Launch>
bl_status_t over_layout(const bl_adamw_plan_s* p, const char* name, double wide, int each, hipStream_t s,
                        Launch&& launch) {
  const size_t total = (size_t)p->first.back() * kChunk;
  for (size_t from = 0; from < total; from += (size_t)kMostBlocks * each) {
    const unsigned blocks = (unsigned)std::min<size_t>(kMostBlocks, (total - from + each - 1) / each);
    const bl_status_t st = timed_launch(name, wide * each * blocks, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      launch(dim3(blocks), from, e0, e1);
    });
    if (st != BL_OK) return st;
  }
  return BL_OK;
}
}  // namespace

extern "C" bl_status_t bl_adamw_get_moments(bl_adamw_plan_t p, const void* state, void* m, void* v, void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (!p->first.back()) return BL_OK;
  if (!state || !m || !v || !aligned(state)) return BL_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const StepArgs a = state_of(p, state);
  if (p->bits == 8)
    return over_layout(p, "adamw_get", 6.0, 8 * kT, s, [&](dim3 g, size_t from, hipEvent_t e0, hipEvent_t e1) {
      hipExtLaunchKernelGGL(k_get8, g, dim3(kT), 0, s, e0, e1, 0, a, static_cast<bf16_t*>(m), static_cast<bf16_t*>(v),
                            from, (size_t)p->first.back() * kChunk);
    });
  return over_layout(p, "adamw_get", 16.0, kChunk, s, [&](dim3 g, size_t from, hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL(k_copy2, g, dim3(kT), 0, s, e0, e1, 0, a.m, a.v, static_cast<float*>(m),
                          static_cast<float*>(v), from);
  });
}

extern "C" bl_status_t bl_adamw_set_moments(bl_adamw_plan_t p, void* state, const float* m, const float* v,
                                            void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (!p->first.back()) return BL_OK;
  if (!state || !m || !v || !aligned(state)) return BL_ERR_INVALID_ARG;
  hipStream_t s = static_cast<hipStream_t>(stream);
  const StepArgs a = state_of(p, state);
  return over_layout(p, "adamw_set", p->bits == 8 ? 10.0 : 16.0, kChunk, s,
                     [&](dim3 g, size_t from, hipEvent_t e0, hipEvent_t e1) {
                       if (p->bits == 8)
                         hipExtLaunchKernelGGL(k_set8, g, dim3(kT), 0, s, e0, e1, 0, a, m, v, from);
                       else
                         hipExtLaunchKernelGGL(k_copy2, g, dim3(kT), 0, s, e0, e1, 0, m, v, a.m, a.v, from);
                     });
}
