// Device helpers of the operators around the convolution (norm.hip, logprob.hip,
// adamw.hip): element types, vector loads of any alignment, wave reductions.
#pragma once

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
