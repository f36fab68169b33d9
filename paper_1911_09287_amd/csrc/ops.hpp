// Device helpers of the operators around the convolution (norm.hip, logprob.hip, adamw.hip,
// gnorm*.hip, recur*.hip, muon*.hip): element types, vector loads of any alignment, wave reductions.
#pragma once

#include <cstdint>
#include <type_traits>

#include "bltrain.h"
#include "common.hpp"

namespace blc {

constexpr int kWave = 64;

// Element types as the device sees them.
using bf16_t = __bf16;
using f16_t = _Float16;

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(bf16_t x) { return (float)x; }
__device__ __forceinline__ float to_f32(f16_t x) { return (float)x; }

// N elements moved as one access.  Global memory takes accesses of 4 to 16
// bytes at any element's alignment, so rows of odd length need no path of their own.
template <typename T, int N>
struct Pack {
  T v[N];
};
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
  Pack<T, N> r;
  __builtin_memcpy(&r, p, sizeof(r));
  return r;
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T* p, const Pack<T, N>& r) {
  __builtin_memcpy(p, &r, sizeof(r));
}
// The first n of them (n <= 0: none; the others are given as `fill`).
template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_part(const T* p, long n, T fill) {
  if (n >= N) return load_pack<T, N>(p);
  Pack<T, N> r;
#pragma unroll
  for (int j = 0; j < N; ++j) r.v[j] = j < n ? p[j] : fill;
  return r;
}
template <typename T, int N>
__device__ __forceinline__ void store_part(T* p, long n, const Pack<T, N>& r) {
  if (n >= N) {
    store_pack<T, N>(p, r);
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (j < n) p[j] = r.v[j];
}

// p, which a whole wave shares, and a lane's bytes from there: one address register.
template <typename T>
__device__ __forceinline__ T* at_bytes(T* p, unsigned bytes) {
  return reinterpret_cast<T*>(reinterpret_cast<std::conditional_t<std::is_const_v<T>, const char, char>*>(p) +
                              (size_t)bytes);
}

// N elements as they were loaded, in 32-bit words, for kernels that hold many.
// refresh() after the loads keeps conversions (and the wait for a load) out of
// the branch that loads, so that all loads of a lane are in flight together;
// later it makes the compiler convert again instead of keeping fp32 copies.
template <typename T, int N>
struct Held {
  static constexpr int kWords = (N * (int)sizeof(T) + 3) / 4;
  unsigned w[kWords];

  // The first n elements at p (n <= 0: none; the others are `fill`, a word's bits).
  __device__ __forceinline__ void load(const T* p, long n, unsigned fill = 0) {
    if (n >= N) {
      if (N * sizeof(T) % 4) w[kWords - 1] = 0;
      __builtin_memcpy(w, p, N * sizeof(T));
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = fill;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < n) {
          if constexpr (sizeof(T) == 4) w[j] = __builtin_bit_cast(unsigned, p[j]);
          else w[j / 2] = (w[j / 2] & (j & 1 ? 0xFFFFu : 0xFFFF0000u)) |
                          (unsigned)__builtin_bit_cast(unsigned short, p[j]) << (16 * (j & 1));
        }
    }
  }
  // All of them at `bytes` from p, or zeros.
  __device__ __forceinline__ void load_at(const T* p, unsigned bytes, bool there) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0;
    if (there) __builtin_memcpy(w, at_bytes(p, bytes), N * sizeof(T));
  }
  __device__ __forceinline__ float operator[](int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[j]);
    else if constexpr (std::is_same_v<T, bf16_t>) return __uint_as_float(j & 1 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    else return (float)__builtin_bit_cast(f16_t, (unsigned short)(j & 1 ? w[j / 2] >> 16 : w[j / 2]));
  }
  __device__ __forceinline__ void refresh() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(w[i]));
  }
};

// ---- exponentials ----------------------------------------------------------------
// exp(g) by the hardware's power of two, and what g log2(e) and log2(e) itself round, which
// would be |g| units: within two units of the last place, results below 2^-126 as 0.  (The
// library's expf takes three times the instructions, and they bound 16-bit passes.)  GROWS:
// g may be so large that the result is infinite, which has no part that could be corrected;
// at minus infinity, where r is NaN, it is 0 whatever the correction.
template <bool GROWS>
__device__ __forceinline__ float exp_of(float g) {
  constexpr float kLog2e = 0x1.715476p+0f, kRest = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;
  const float t = g * kLog2e, r = fmaf(g, kLog2e, -t), e = __builtin_amdgcn_exp2f(t);
  const float x = fmaf(e, __builtin_amdgcn_fmed3f(fmaf(r, kLn2, g * (kRest * kLn2)), -0x1p-10f, 0x1p-10f), e);
  return GROWS && e == INFINITY ? e : x;
}

// q = 1 / (1 + exp(-z)), 1 - q and q (1 - q).  exp of -|z| does not overflow, and the smaller of the
// first two keeps its relative precision, six units.
__device__ __forceinline__ void logistic_of(float z, float& q, float& rest, float& slope) {
  const float e = exp_of<false>(-fabsf(z)), big = __builtin_amdgcn_rcpf(1.f + e), small = e * big;
  q = z >= 0.f ? big : small;  // (a NaN: both are)
  rest = z >= 0.f ? small : big;
  slope = small * big;
}

// ---- sums over lanes ------------------------------------------------------------
// x of the lane that DPP control CTRL names.
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xF, 0xF, false));
}
// x + x of the lane 16 (32) further or back: two copies that exchange their odd
// and even rows of 16 (upper and lower halves of 32).
__device__ __forceinline__ float add16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float max16(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max32(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float wave_max(float x) {
  x = fmaxf(x, dpp<0xB1>(x));
  x = fmaxf(x, dpp<0x4E>(x));
  x = fmaxf(x, dpp<0x141>(x));
  x = fmaxf(x, dpp<0x140>(x));
  return max32(max16(x));
}
// Sum over groups of `lanes` neighbouring lanes (a power of two, the same for the
// whole wave; every lane of a group active), for each of them.
__device__ __forceinline__ float wave_sum(float x, int lanes = kWave) {
  if (lanes > 1) x += dpp<0xB1>(x);   // quad_perm 1 0 3 2
  if (lanes > 2) x += dpp<0x4E>(x);   // quad_perm 2 3 0 1
  if (lanes > 4) x += dpp<0x141>(x);  // row_half_mirror: the other four of eight
  if (lanes > 8) x += dpp<0x140>(x);  // row_mirror: the other eight of sixteen
  if (lanes > 16) x = add16(x);
  if (lanes > 32) x = add32(x);
  return x;
}

inline bool known_dtype(int d) { return d == BL_F32 || d == BL_BF16 || d == BL_F16; }
inline int dtype_bytes(int d) { return d == BL_F32 ? 4 : 2; }
// Whether a workspace or state starts where its widest accesses may.
inline bool aligned(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
inline size_t round_up(size_t n, size_t a) { return (n + a - 1) / a * a; }

}  // namespace blc
