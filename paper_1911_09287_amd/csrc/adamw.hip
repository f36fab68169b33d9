// AdamW over many tensors at once, moments in 32 bits or in 8: elementwise, every
// parameter, gradient and moment read once and written once.  The tensors of a launch
// are part of its arguments, so that nothing is copied to the device beforehand and a
// captured step replays.
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
static_assert(kWaves == 4, "a block's waves take a chunk");
constexpr int kChunk = 1024;    // tensors start at multiples of this many elements of the layout
constexpr int kBlock = 128;     // elements that share a power of two: four on each of 32 lanes
constexpr int kTensors = 128;   // of one launch: their list is part of the kernel's arguments (4 KB at most)
constexpr int kFewTensors = 16; // 3 KB of arguments cost 1.7 us a launch: few tensors go in a short list

constexpr long long kMostBlocks = (1LL << 24) - 1;  // of a launch, which has fewer than 2^32 threads

// The tensors of a launch; tensor i has chunks first[i] ... first[i + 1] - 1 of
// the layout (all ones past the last), |tail| elements in the last one, weight
// decay where tail < 0.
template <int N>
struct TensorList {
  void* p[N];
  const void* g[N];
  unsigned first[N + 1];
  short tail[N];
};

struct StepArgs {
  float b1, r1, b2, r2;    // beta, 1 - beta
  float eps, keep;         // keep: 1 - lr weight_decay
  float rate, root;        // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  int careful;             // eps so small that a subnormal v counts beside it
  unsigned key;            // of the dither
  unsigned seed;
  double beta1, beta2, wd;
  const float* grad_scale;
  const double* live;
  float *m, *v;            // 32-bit moments
  unsigned char *mc, *vc;  // 8-bit codes
  float *ms, *vs;          // powers of two of their blocks
};

// What follows from lr and the step (on the device for a live step), eps being set.  The
// vector unit's square root and reciprocal take subnormal values for 0; sqrt(v) root of
// such a v is 2^-63 root at most, and 2^-25 of an eps from 2^-38 root on (of 1e-8 for all
// beta2 up to 1 - 2^-22).
__host__ __device__ void step_scalars(StepArgs& a, double lr, double t) {
  a.rate = (float)(lr / (1.0 - pow(a.beta1, t)));
  a.root = (float)(1.0 / sqrt(1.0 - pow(a.beta2, t)));
  a.careful = a.eps < a.root * 0x1p-38f;
  a.keep = (float)(1.0 - lr * a.wd);
  a.key = a.seed * 0x6A09E667u + (unsigned)(long long)t * 0xBB67AE85u;
}

// 32 bits for each of four elements from `place` on.
__device__ __forceinline__ void dither4(unsigned long long place, unsigned key, unsigned (&h)[4]) {
  unsigned x = (unsigned)place * 0x9E3779B9u + key;
#pragma unroll
  for (int j = 0; j < 4; ++j, x += 0x9E3779B9u) {
    const unsigned y = (x ^ (x >> 15)) * 0xBB67AE85u;
    h[j] = y ^ (y >> 16);
  }
}

// 8-bit values: S and a power of two that turns the code's lowest exponents into
// fp32's subnormals are divided out at once, which leaves exponent and fraction of the
// code in the bits from 20 on (of |m| 2^(-113 - log2 S), of v 2^(-97 - log2 S)), where
// the dither is added.
constexpr unsigned kInf = 0x7F800000u, kLeast = 0x0F800000u;  // bits of infinity and of 2^-96
constexpr int kDownM = 113, kDownV = 97;
__device__ __forceinline__ unsigned bits_of(float x) { return __float_as_uint(x); }
__device__ __forceinline__ float from_bits(unsigned u) { return __uint_as_float(u); }
// S of a block from its largest magnitude's bits, and log2 S.
__device__ __forceinline__ unsigned power_bits(unsigned largest) { return max(largest & kInf, kLeast); }
__device__ __forceinline__ int log2_of(unsigned s) { return (int)(s >> 23) - 127; }
// For moments set from values: half of it where the largest is itself a power of
// two (which the code above all fractions then holds), so that values which
// codes stood for are held again as they are, however their block's S was.
__device__ __forceinline__ unsigned power_bits_below(unsigned largest) { return power_bits(largest ? largest - 1 : 0); }

__device__ __forceinline__ unsigned encode(float a, int down, unsigned d16) {
  return (bits_of(__builtin_amdgcn_ldexpf(a, -down)) + (d16 << 4)) >> 20;
}
// (finite values; `down`: kDown + log2 S)
__device__ __forceinline__ unsigned encode_m(float m, int down, unsigned d16) {
  return encode(fabsf(m), down, d16) | (bits_of(m) >> 24 & 0x80u);
}
__device__ __forceinline__ unsigned encode_v(float v, int down, unsigned d16) {
  return max(encode(v, down, d16), min(bits_of(v), 1u));  // (what is positive is not held as 0)
}
__device__ __forceinline__ float decode_m(unsigned c, int down) {
  const float x = __builtin_amdgcn_ldexpf(from_bits((c & 0x7Fu) << 20), down);
  return from_bits(bits_of(x) | (c & 0x80u) << 24);
}
__device__ __forceinline__ float decode_v(unsigned c, int down) {
  return __builtin_amdgcn_ldexpf(from_bits(c << 20), down);
}
// The codes of all ones (exponent and fraction) are NaN: four values from their codes.
__device__ __forceinline__ void decode4(unsigned mc, unsigned vc, float ms, float vs, float (&m)[4], float (&v)[4]) {
  // (a state of zero bytes has S = 0, and codes of 0)
  const int dm = kDownM + log2_of(bits_of(ms)), dv = kDownV + log2_of(bits_of(vs));
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    m[j] = decode_m(mc >> (8 * j) & 0xFFu, dm);
    v[j] = decode_v(vc >> (8 * j) & 0xFFu, dv);
  }
  const unsigned ones = (((mc & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) | ((~vc - 0x01010101u) & vc & 0x80808080u);
  if (__ballot(ones != 0))  // rare (and at times with no such code: a borrow)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if ((mc >> (8 * j) & 0x7Fu) == 0x7Fu) m[j] = NAN;
      if ((vc >> (8 * j) & 0xFFu) == 0xFFu) v[j] = NAN;
    }
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
// Bits of the largest finite magnitude of a block, four values on each of 32 lanes,
// and whether the wave has any value that is not finite.
__device__ __forceinline__ unsigned block_largest(const float (&x)[4], bool& wild) {
  unsigned u[4], l = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) l = max(l, u[j] = bits_of(x[j]) & 0x7FFFFFFFu);
  wild = __ballot(l >= kInf) != 0;
  if (wild) {  // rare: leave them out
    l = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) l = max(l, u[j] < kInf ? u[j] : 0u);
  }
  return max32(l);
}
// Codes of four values, and their blocks' powers of two.  h: 32 bits of dither each.
template <bool BELOW>
__device__ __forceinline__ void encode4(const float (&m)[4], const float (&v)[4], const unsigned (&h)[4], unsigned& mc,
                                        unsigned& vc, unsigned& sm, unsigned& sv) {
  bool wild_m, wild_v;
  const unsigned lm = block_largest(m, wild_m), lv = block_largest(v, wild_v);
  sm = BELOW ? power_bits_below(lm) : power_bits(lm);
  sv = BELOW ? power_bits_below(lv) : power_bits(lv);
  const int dm = kDownM + log2_of(sm), dv = kDownV + log2_of(sv);
  mc = vc = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    mc |= encode_m(m[j], dm, h[j] & 0xFFFFu) << (8 * j);
    vc |= encode_v(v[j], dv, h[j] >> 16) << (8 * j);
  }
  if (wild_m || wild_v) {
    mc = vc = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool fine_m = (bits_of(m[j]) & 0x7FFFFFFFu) < kInf, fine_v = (bits_of(v[j]) & 0x7FFFFFFFu) < kInf;
      mc |= (fine_m ? encode_m(m[j], dm, h[j] & 0xFFFFu) : 0x7Fu) << (8 * j);
      vc |= (fine_v ? encode_v(v[j], dv, h[j] >> 16) : 0xFFu) << (8 * j);
    }
  }
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

// One step.  A wave takes 256 elements, a quarter of a chunk, four on each lane, so
// that a block of 128 lies on half a wave.  (A whole chunk a wave, 16 elements on each
// lane, is slower at every size: 11 million values with fp32 moments 62 us against 55.)
// sqrt and reciprocal are the vector unit's, off by an ulp each (see `careful`).  Bound
// by HBM: 126 million values, moments of 8 bits, gradients in bfloat16 313 us, 5.7 TB/s
// (a large copy reaches 5.0); 11 million, fp32 moments 56 us, 5.2 TB/s.  With bfloat16
// parameters too (10 bytes a value) the arithmetic of the codes comes near: 294 us, 4.3
// TB/s.  A live step takes its scalars' powers in 64 bits on every lane: 579 us instead
// of the 313, but 60 instead of the 56 (and 1 more of the smallest).
template <typename P, typename G, int BITS, bool LIVE, int N>
__global__ __launch_bounds__(kT) void k_adamw(const TensorList<N> list, StepArgs a) {
  const unsigned lane = threadIdx.x & 63;
  const unsigned wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + (threadIdx.x >> 6));
  const unsigned chunk = list.first[0] + wave / 4;              // (a block's waves make one chunk)
  const unsigned quarter = wave % 4 * 256, from = quarter + lane * 4;  // of this lane's first, in the chunk
  const size_t at = (size_t)chunk * kChunk + from;              // in the layout
  // the moments lie at the chunk's place: their loads go out before the tensor is known
  Pack<float, 4> m0, v0;
  unsigned mc, vc;
  float ms, vs;
  if (BITS == 32) {
    m0 = load_pack<float, 4>(a.m + at);
    v0 = load_pack<float, 4>(a.v + at);
  } else {
    mc = *reinterpret_cast<const unsigned*>(a.mc + at);
    vc = *reinterpret_cast<const unsigned*>(a.vc + at);
    ms = a.ms[at / kBlock];
    vs = a.vs[at / kBlock];
  }
  // the tensor: how many start at or before this chunk, less one
  int before = __popcll(__ballot((int)lane < N && list.first[1 + (lane < N ? lane : 0)] <= chunk));
  if (N > kWave) before += __popcll(__ballot(list.first[1 + (N > kWave ? kWave : 0) + lane] <= chunk));
  const unsigned t = __builtin_amdgcn_readfirstlane(before);
  const int tail = list.tail[t];
  const int here = chunk + 1 == list.first[t + 1] ? abs(tail) : kChunk;  // the tensor's elements in this chunk
  const int n = here - (int)from;                                         // from this lane's first on
  const size_t off = (size_t)(chunk - list.first[t]) * kChunk + from;     // in the tensor
  P* const pp = static_cast<P*>(list.p[t]) + off;
  Pack<P, 4> p = load_part<P, 4>(pp, n, (P)0.f);
  const Pack<G, 4> g = load_part<G, 4>(static_cast<const G*>(list.g[t]) + off, n, (G)0.f);
  if (LIVE) step_scalars(a, a.live[0], a.live[1]);
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const float keep = tail < 0 ? a.keep : 1.f;
  float m[4], v[4];
  unsigned h[4] = {};
  if (BITS == 8 || sizeof(P) == 2) dither4(at, a.key, h);
  if (BITS == 8) decode4(mc, vc, ms, vs, m, v);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if (BITS == 32) m[j] = m0.v[j], v[j] = v0.v[j];
    const float gj = to_f32(g.v[j]) * gs;
    m[j] = decayed(m[j], a.b1, gj, a.r1);
    v[j] = decayed(v[j], a.b2, gj * gj, a.r2);
  }
  float go[4];  // the step
  if (a.careful) {
#pragma unroll
    for (int j = 0; j < 4; ++j) go[j] = m[j] * a.rate / fmaf(sqrtf(v[j]), a.root, a.eps);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      go[j] = m[j] * a.rate * __builtin_amdgcn_rcpf(fmaf(__builtin_amdgcn_sqrtf(v[j]), a.root, a.eps));
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) p.v[j] = round_param<P>(fmaf(to_f32(p.v[j]), keep, -go[j]), h[j]);
  store_part<P, 4>(pp, n, p);
  if (BITS == 32) {
    store_part<float, 4>(a.m + at, n, Pack<float, 4>{{m[0], m[1], m[2], m[3]}});
    store_part<float, 4>(a.v + at, n, Pack<float, 4>{{v[0], v[1], v[2], v[3]}});
  } else {
    if (here < (int)quarter + 256)  // what lies past the tensor has no part in its block
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (j >= n) m[j] = v[j] = 0.f;
    unsigned sm, sv;
    encode4<false>(m, v, h, mc, vc, sm, sv);
    *reinterpret_cast<unsigned*>(a.mc + at) = mc;
    *reinterpret_cast<unsigned*>(a.vc + at) = vc;
    if (lane % 32 == 0) {
      a.ms[at / kBlock] = from_bits(sm);
      a.vs[at / kBlock] = from_bits(sv);
    }
  }
}

// 8-bit moments as bfloat16 values, eight a thread.  Bound by HBM: 126 million in 127
// us, 5.9 TB/s.
__global__ __launch_bounds__(kT) void k_get8(const StepArgs a, bf16_t* m, bf16_t* v, size_t from, size_t total) {
  const size_t at = from + ((size_t)blockIdx.x * kT + threadIdx.x) * 8;
  if (at >= total) return;
  const uint2 mc = *reinterpret_cast<const uint2*>(a.mc + at), vc = *reinterpret_cast<const uint2*>(a.vc + at);
  const float ms = a.ms[at / kBlock], vs = a.vs[at / kBlock];
  Pack<bf16_t, 8> mo, vo;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    float x[4], y[4];
    decode4(half ? mc.y : mc.x, half ? vc.y : vc.x, ms, vs, x, y);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      mo.v[4 * half + j] = (bf16_t)x[j];
      vo.v[4 * half + j] = (bf16_t)y[j];
    }
  }
  store_pack<bf16_t, 8>(m + at, mo);
  store_pack<bf16_t, 8>(v + at, vo);
}

__global__ __launch_bounds__(kT) void k_set8(StepArgs a, const float* m, const float* v, size_t from) {
  const size_t at = from + ((size_t)blockIdx.x * kT + threadIdx.x) * 4;
  const Pack<float, 4> mi = load_pack<float, 4>(m + at);
  Pack<float, 4> vi = load_pack<float, 4>(v + at);
#pragma unroll
  for (int j = 0; j < 4; ++j) vi.v[j] = vi.v[j] < 0.f ? NAN : fabsf(vi.v[j]);  // (-0 is 0)
  const unsigned half = 1u << 15 | 1u << 31, h[4] = {half, half, half, half};  // to nearest
  unsigned mc, vc, sm, sv;
  encode4<true>(mi.v, vi.v, h, mc, vc, sm, sv);
  *reinterpret_cast<unsigned*>(a.mc + at) = mc;
  *reinterpret_cast<unsigned*>(a.vc + at) = vc;
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
  return f;
}

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
      if (n && p->first[at + 1] - list.first[0] > kMostBlocks) break;
      list.p[n] = params[at];
      list.g[n] = grads[at];
      list.first[n] = (unsigned)first;
      const int tail = (int)((p->sizes[at] - 1) % kChunk + 1);
      list.tail[n] = (short)(p->decay[at] ? -tail : tail);
      list.first[++n] = (unsigned)p->first[at + 1];
      values += (double)p->sizes[at];
    }
    if (!n) break;
    const unsigned chunks = list.first[n] - list.first[0];
    for (int i = n + 1; i <= kTensors; ++i) list.first[i] = ~0u;
    const double bytes = values * (2 * sizeof(P) + sizeof(G) + (BITS == 32 ? 16 : 4 + 16.0 / kBlock));
    const bl_status_t st = timed_launch("adamw", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      auto go = [&](auto kernel, const auto& l) {
        hipExtLaunchKernelGGL(kernel, dim3(chunks), dim3(kT), 0, s, e0, e1, 0, l, a);
      };
      if (a.live) go(k_adamw<P, G, BITS, true, kTensors>, list);
      else if (n > kFewTensors) go(k_adamw<P, G, BITS, false, kTensors>, list);
      else go(k_adamw<P, G, BITS, false, kFewTensors>, few_of(list));
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
    if (d->sizes[i] > kMostBlocks * kChunk) return BL_ERR_UNSUPPORTED;  // (a launch takes whole tensors)
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
  a.eps = r.eps > 0.0 ? std::max((float)r.eps, 0x1p-149f) : 0.f;  // (a v and m of 0 leave the parameter where it is)
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
