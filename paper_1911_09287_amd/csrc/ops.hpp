// Device helpers of the operators around the convolution (norm.hip, logprob.hip,
// adamw.hip): element types, vector loads of any alignment, wave reductions.
#pragma once

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

// N elements as they were loaded, in 32-bit words, for kernels that keep many:
// refresh() makes the compiler convert them again at the next use instead of
// keeping fp32 copies in registers.
template <typename T, int N>
struct Held {
  static constexpr int kWords = (N * (int)sizeof(T) + 3) / 4;
  unsigned w[kWords];

  __device__ __forceinline__ void load(const T* p, long n) {
    const Pack<T, N> r = load_part<T, N>(p, n, (T)0.f);
    if (N * sizeof(T) % 4) w[kWords - 1] = 0;
    __builtin_memcpy(w, &r, sizeof(r));
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

__device__ __forceinline__ float wave_sum(float x, int width = kWave) {
  for (int o = width / 2; o > 0; o >>= 1) x += __shfl_xor(x, o);
  return x;
}
__device__ __forceinline__ float wave_max(float x, int width = kWave) {
  for (int o = width / 2; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
  return x;
}

inline bool known_dtype(int d) { return d == BL_F32 || d == BL_BF16 || d == BL_F16; }
inline int dtype_bytes(int d) { return d == BL_F32 ? 4 : 2; }
inline size_t round_up(size_t n, size_t a) { return (n + a - 1) / a * a; }

}  // namespace blc
