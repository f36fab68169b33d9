// The products of a Newton-Schulz step, A = X X^T, B = a I + b A + c A A and X = B X, of many
// matrices in one launch each.
//
// Both operands of each lie with the summed index side by side: A and B are symmetric, and X
// is held together with its transpose.  Values are two fp16 parts, v = high + low to 22 bits;
// a product takes high high + high low + low high on the matrix cores (the last, low low, is
// below 2^-22) and sums in fp32.  One fp16 part alone leaves errors of 1 % in the result where a
// gradient has a few strong directions: rounding is noise in all directions, and the steps
// raise the weak ones by up to 3.44 each.  Symmetric products are taken for tiles on and
// below the diagonal only and stored twice.
#include "muon.hpp"

namespace blc {
namespace {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kRowBytes = 128;               // 32 values of a row, high and low parts
constexpr int kStage = 2 * kMuonTile * kRowBytes;  // of both operands' tiles

// 32 values of each of the tile's rows from both operands into LDS, 16 bytes a lane and
// eight rows an access.  A row's eight pieces are exchanged by the row's number, so that
// the lanes of a fragment, which lie on rows, read different banks.
__device__ __forceinline__ void stage(const char* from, size_t stride, char* to) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const char* p = from + (size_t)(lane / 8) * stride + ((lane % 8) ^ (lane / 8)) * 16;
#pragma unroll
  for (int k = 0; k < 8; ++k)
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(p + (size_t)k * 8 * stride),
                                     (__attribute__((address_space(3))) void*)(to + (wave * 8 + k) * 8 * kRowBytes), 16,
                                     0, 0);
}
__device__ __forceinline__ f16x8 fragment(const char* rows, int row, int piece) {
  return *reinterpret_cast<const f16x8*>(rows + row * kRowBytes + ((piece ^ (row & 7)) * 16));
}

// acc[tp][tq] += the 64 x 64 part of a wave over `steps` times 32 of the summed index: P and Q
// are the rows of the tile's operands.
__device__ __forceinline__ void product(const char* P, const char* Q, size_t stride, int steps, char* lds,
                                        f32x16 (&acc)[2][2]) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  // waves 0 and 1 fetch P, 2 and 3 Q: 64 rows each
  const char* from = (wave < 2 ? P : Q) + (size_t)(wave & 1) * 64 * stride;
  const int pr = wave / 2 * 64 + lane % 32, qr = kMuonTile + wave % 2 * 64 + lane % 32, half = lane / 32;
  stage(from, stride, lds);
  for (int k = 0; k < steps; ++k) {
    // what this wave fetched has arrived; then all waves' has, and all have read the other half
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (k + 1 < steps) stage(from + (size_t)(k + 1) * kRowBytes, stride, lds + (k + 1) % 2 * kStage);
    const char* now = lds + k % 2 * kStage;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      f16x8 p[2][2], q[2][2];  // [tile][high, low]
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int l = 0; l < 2; ++l) {
          p[t][l] = fragment(now, pr + t * 32, l * 4 + s * 2 + half);
          q[t][l] = fragment(now, qr + t * 32, l * 4 + s * 2 + half);
        }
#pragma unroll
      for (int tp = 0; tp < 2; ++tp)
#pragma unroll
        for (int tq = 0; tq < 2; ++tq) {
          acc[tp][tq] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[tp][0], q[tq][1], acc[tp][tq], 0, 0, 0);
          acc[tp][tq] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[tp][1], q[tq][0], acc[tp][tq], 0, 0, 0);
          acc[tp][tq] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[tp][0], q[tq][0], acc[tp][tq], 0, 0, 0);
        }
    }
  }
  __syncthreads();  // (LDS may be used again)
}

// Place of 4 values (8 bytes of high parts; their low parts 64 bytes on) of a row from
// column c on.
__device__ __forceinline__ size_t held_at(size_t row, size_t stride, unsigned c) {
  return row * stride + c / 32 * 128 + c % 32 * 2;
}
template <int N>
__device__ __forceinline__ void hold(char* at, const float (&v)[N]) {
  Pack<f16_t, N> hi, lo;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    hi.v[j] = (f16_t)v[j];
    lo.v[j] = (f16_t)(v[j] - (float)hi.v[j]);
  }
  store_pack(reinterpret_cast<f16_t*>(at), hi);
  store_pack(reinterpret_cast<f16_t*>(at + 64), lo);
}

// go(row, column, v) for every four rows of a column that this lane holds of the tile, rows
// P's and columns Q's: row ... row + 3.
template <typename Go>
__device__ __forceinline__ void each_four(const f32x16 (&acc)[2][2], Go&& go) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
#pragma unroll
  for (int tp = 0; tp < 2; ++tp)
#pragma unroll
    for (int tq = 0; tq < 2; ++tq)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = acc[tp][tq][4 * r + k];
        go(wave / 2 * 64 + tp * 32 + r * 8 + lane / 32 * 4, wave % 2 * 64 + tq * 32 + lane % 32, v);
      }
}

// The tile, which all lanes have written to LDS as [row][column], to rows of `to`.
__device__ __forceinline__ void hold_rows(const float* tile, char* to, size_t stride) {
  for (int i = threadIdx.x; i < kMuonTile * kMuonTile / 8; i += kThreads) {
    const int row = i / (kMuonTile / 8), c = i % (kMuonTile / 8) * 8;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = tile[row * kMuonTile + c + j];
    hold<8>(to + held_at(row, stride, c), v);
  }
}

template <int MODE>
__global__ __launch_bounds__(kThreads, 2) void k_muon_product(MuonShapes list, MuonProduct q) {
  __shared__ __align__(16) char lds[2 * kStage];
  static_assert(2 * kStage == kMuonTile * kMuonTile * 4, "a tile of fp32");
  const unsigned at = muon_find(list.first, list.count, blockIdx.x);
  unsigned tile = blockIdx.x - list.first[at];
  const unsigned m = list.m[at], n = list.n[at];
  const MuonPlaces w = muon_places(m, n);
  char* part = q.ws + (size_t)list.off[at] * 256;
  unsigned ti, tj;  // of the result, in tiles
  if (MODE == kApply) {
    ti = tile % m;
    tj = tile / m;
  } else {  // on and below the diagonal
    ti = (unsigned)((sqrtf(8.f * tile + 1.f) - 1.f) * 0.5f);
    while ((ti + 1) * (ti + 2) / 2 <= tile) ++ti;
    while (ti * (ti + 1) / 2 > tile) --ti;
    tj = tile - ti * (ti + 1) / 2;
  }
  const unsigned sum = MODE == kGram ? n : m;                       // tiles of the summed index
  const size_t stride = (size_t)sum * kMuonTile * 4, mm = (size_t)m * kMuonTile * 4, nn = (size_t)n * kMuonTile * 4;
  const char* P = part + (MODE == kGram ? w.x : MODE == kPoly ? w.a : w.b);
  const char* Q = MODE == kApply ? part + w.t(q.turn) : P;
  f32x16 acc[2][2] = {};
  product(P + (size_t)ti * kMuonTile * stride, Q + (size_t)tj * kMuonTile * stride, stride, (int)sum * (kMuonTile / 32),
          lds, acc);
  float* tiled = reinterpret_cast<float*>(lds);
  // columns of the tile are rows of the transpose: four of a lane's values lie side by side
  char* across = part + (MODE == kGram ? w.a : MODE == kPoly ? w.b : w.t(q.turn ^ 1));
  const bool both = MODE == kApply || ti != tj;
  each_four(acc, [&](int row, int col, float (&v)[4]) {
    const size_t place = held_at((size_t)tj * kMuonTile + col, mm, ti * kMuonTile + row);
    if (MODE == kPoly) {
      const char* from = part + w.a + place;
      const Pack<f16_t, 4> hi = load_pack<f16_t, 4>(reinterpret_cast<const f16_t*>(from)),
                           lo = load_pack<f16_t, 4>(reinterpret_cast<const f16_t*>(from + 64));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[k] = fmaf(q.c, v[k], q.b * ((float)hi.v[k] + (float)lo.v[k]));
        if (ti == tj && row + k == col) v[k] += q.a;
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] *= q.scale;
    }
    hold<4>(across + place, v);
    if (both)
#pragma unroll
      for (int k = 0; k < 4; ++k) tiled[(row + k) * kMuonTile + col] = v[k];
  });
  if (!both) return;
  __syncthreads();
  const size_t other = MODE == kApply ? nn : mm;
  hold_rows(tiled, part + (MODE == kGram ? w.a : MODE == kPoly ? w.b : w.x) + held_at((size_t)ti * kMuonTile, other, tj * kMuonTile),
            other);
}

// The last step: X goes into the parameters.
template <typename P>
__global__ __launch_bounds__(kThreads, 2) void k_muon_update(MuonList list, MuonProduct q, MuonArgs a) {
  __shared__ __align__(16) char lds[2 * kStage];
  const unsigned at = muon_find(list.first, list.count, blockIdx.x);
  const unsigned tile = blockIdx.x - list.first[at];
  const MuonItem& it = list.item[at];
  const unsigned m = it.m, ti = tile % m, tj = tile / m;
  const MuonPlaces w = muon_places(m, it.n);
  const char* part = q.ws + (size_t)it.off * 256;
  const size_t stride = (size_t)m * kMuonTile * 4;
  f32x16 acc[2][2] = {};
  product(part + w.b + (size_t)ti * kMuonTile * stride, part + w.t(q.turn) + (size_t)tj * kMuonTile * stride, stride,
          (int)m * (kMuonTile / 32), lds, acc);
  float keep = 1.f, rate = 1.f;
  unsigned key = a.key;
  if (!a.set) {
    double lr = a.lr;
    if (a.live) {
      lr = a.live[0];
      key = a.seed * 0x6A09E667u + (unsigned)(long long)a.live[1] * 0xBB67AE85u;
    }
    if (it.decay) keep = (float)(1.0 - lr * a.wd);
    rate = (float)(lr * (double)it.scale);
  }
  P* p = static_cast<P*>(it.p);
  each_four(acc, [&](int row, int col, float (&v)[4]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = (int)ti * kMuonTile + row + k, j = (int)tj * kMuonTile + col;
      const int r = it.tall ? j : i, c = it.tall ? i : j;
      if (r >= it.rows || c >= it.cols) continue;
      const size_t e = (size_t)r * it.cols + c;
      const float x = v[k] * q.scale;
      if (a.set) {
        p[e] = (P)x;
        continue;
      }
      const float next = fmaf(-rate, x, to_f32(p[e]) * keep);
      if constexpr (sizeof(P) == 4) {
        p[e] = next;
      } else {
        const unsigned bits = __float_as_uint(next);
        const bool finite = (bits & 0x7F800000u) != 0x7F800000u;
        const unsigned up = finite ? bits + muon_dither((unsigned long long)it.start + e, key) : bits | (next != next ? 0x400000u : 0u);
        p[e] = __builtin_bit_cast(bf16_t, (unsigned short)(up >> 16));
      }
    }
  });
}

}  // namespace

bl_status_t muon_product(int mode, const MuonShapes& shapes, unsigned blocks, double flops, const MuonProduct& q,
                         hipStream_t s) {
  const char* names[] = {"muon_gram", "muon_poly", "muon_apply"};
  return timed_launch(names[mode], 0.0, flops, s, [&](hipEvent_t e0, hipEvent_t e1) {
    auto go = [&](auto kernel) { hipExtLaunchKernelGGL(kernel, dim3(blocks), dim3(kThreads), 0, s, e0, e1, 0, shapes, q); };
    if (mode == kGram) go(k_muon_product<kGram>);
    else if (mode == kPoly) go(k_muon_product<kPoly>);
    else go(k_muon_product<kApply>);
  });
}

bl_status_t muon_update(int param_dtype, const MuonList& list, unsigned blocks, double flops, const MuonProduct& q,
                        const MuonArgs& a, hipStream_t s) {
  return timed_launch("muon_update", 0.0, flops, s, [&](hipEvent_t e0, hipEvent_t e1) {
    if (param_dtype == BL_F32)
      hipExtLaunchKernelGGL(k_muon_update<float>, dim3(blocks), dim3(kThreads), 0, s, e0, e1, 0, list, q, a);
    else
      hipExtLaunchKernelGGL(k_muon_update<bf16_t>, dim3(blocks), dim3(kThreads), 0, s, e0, e1, 0, list, q, a);
  });
}

}  // namespace blc
