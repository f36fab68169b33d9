// Orthogonalised update of small matrices: a block takes one matrix through all of the step.
//
// With a shorter side of at most 64 the square matrices of the products lie in LDS, 16 KB each,
// a wave has 16 x 16 of them, and a product ends after six matrix instructions; X and its
// transpose (up to 1024 long) are written to the workspace and come back from the caches.  Bound
// by the chain of some 20 products with a barrier each, not by their work: launches of
// many blocks, one for each product, take 80 us here.
#include "muon.hpp"

namespace blc {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kT = 1024;          // threads: 16 waves, 4 x 4 tiles of 16
constexpr int kSide = 64;
constexpr int kSlotBytes = kSide * kSide * 4;

__device__ __forceinline__ int lane_row() { return threadIdx.x % 16; }
__device__ __forceinline__ int lane_quad() { return threadIdx.x % kWave / 16; }

// acc += P Q^T over 32 of the summed index, from their fragments [high, low].
__device__ __forceinline__ void multiply(const f16x8 (&p)[2], const f16x8 (&q)[2], f32x4& acc) {
  acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[0], q[1], acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[1], q[0], acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(p[0], q[0], acc, 0, 0, 0);
}
// A slot's pieces of 16 bytes (32 values of a row: four of high parts, four of low ones) are
// exchanged by the row's number, so that rows read different banks.
__device__ __forceinline__ char* piece(char* slot, int row, int k) { return slot + row * 256 + ((k ^ (row & 15)) * 16); }
__device__ __forceinline__ void fragments(char* slot, int row, int step, f16x8 (&f)[2]) {
#pragma unroll
  for (int l = 0; l < 2; ++l) f[l] = *reinterpret_cast<const f16x8*>(piece(slot, row, step * 8 + l * 4 + lane_quad()));
}
__device__ __forceinline__ void fragments_at(const char* row, int step, f16x8 (&f)[2]) {
#pragma unroll
  for (int l = 0; l < 2; ++l) f[l] = *reinterpret_cast<const f16x8*>(row + step * 128 + l * 64 + lane_quad() * 16);
}
// Four values of a row from column c on.
__device__ __forceinline__ void split4(const f32x4& v, Pack<f16_t, 4>& hi, Pack<f16_t, 4>& lo) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    hi.v[k] = (f16_t)v[k];
    lo.v[k] = (f16_t)(v[k] - (float)hi.v[k]);
  }
}
__device__ __forceinline__ void hold(char* slot, int row, int c, const f32x4& v) {
  Pack<f16_t, 4> hi, lo;
  split4(v, hi, lo);
  const int k = c / 32 * 8 + c % 32 / 8, at = c % 8 * 2;
  store_pack(reinterpret_cast<f16_t*>(piece(slot, row, k) + at), hi);
  store_pack(reinterpret_cast<f16_t*>(piece(slot, row, k + 4) + at), lo);
}
__device__ __forceinline__ f32x4 held(char* slot, int row, int c) {
  const int k = c / 32 * 8 + c % 32 / 8, at = c % 8 * 2;
  const Pack<f16_t, 4> hi = load_pack<f16_t, 4>(reinterpret_cast<const f16_t*>(piece(slot, row, k) + at)),
                       lo = load_pack<f16_t, 4>(reinterpret_cast<const f16_t*>(piece(slot, row, k + 4) + at));
  f32x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = (float)hi.v[j] + (float)lo.v[j];
  return v;
}
// A symmetric result: a lane's four values are rows r ... r + 3 of column c, and go to its columns r ...
// r + 3 of row c, and those below the diagonal to their own place (after the wave's others, which a tile on
// the diagonal has stored there), so that what is held is symmetric to the last bit: an antisymmetric part would
// grow tenfold with every joined step (50 x 128 after five steps: off by 3e-5 of the norm with both halves as
// computed, 3e-6 so).
__device__ __forceinline__ void hold_both(char* slot, int r, int c, const f32x4& v) {
  hold(slot, c, r, v);
  Pack<f16_t, 4> hi, lo;
  split4(v, hi, lo);
  const int k = c / 32 * 8 + c % 32 / 8, at = c % 8 * 2;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (r + j > c) {
      *reinterpret_cast<f16_t*>(piece(slot, r + j, k) + at) = hi.v[j];
      *reinterpret_cast<f16_t*>(piece(slot, r + j, k + 4) + at) = lo.v[j];
    }
}
// This wave's tile of a product of square matrices, over `sum` times 32.
__device__ __forceinline__ f32x4 square(char* p, char* q, int sum) {
  const int wave = threadIdx.x / kWave;
  f32x4 acc = {};
  for (int s = 0; s < sum; ++s) {
    f16x8 a[2], b[2];
    fragments(p, wave / 4 * 16 + lane_row(), s, a);
    fragments(q, wave % 4 * 16 + lane_row(), s, b);
    multiply(a, b, acc);
  }
  return acc;
}

template <typename G, typename P>
__global__ __launch_bounds__(kT) void k_muon_small(MuonList list, MuonSmallSteps steps, MuonArgs a) {
  extern __shared__ __align__(16) char lds[];  // kSlots square matrices
  __shared__ double red[kT / kWave];
  const MuonItem& it = list.item[blockIdx.x];
  const int rows = it.rows, cols = it.cols, size = rows * cols;
  const bool tall = it.tall;
  const G* g = static_cast<const G*>(it.g);
  float* m = a.momentum ? a.momentum + it.start : nullptr;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  // momentum, and the squares of u in double precision
  double sum = 0.0;
  constexpr int kAhead = 4;
  for (int e0 = threadIdx.x; e0 < size; e0 += kAhead * kT) {
    float gv[kAhead], mv[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int e = min(e0 + k * kT, size - 1);  // (the last one again, and not counted)
      gv[k] = to_f32(g[e]);
      mv[k] = m ? m[e] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (e0 + k * kT >= size) break;
      const float next = fmaf(a.beta, mv[k], gs * gv[k]);
      if (m) m[e0 + k * kT] = next;
      const double u = muon_update_of(gv[k], next, gs, a);
      sum = fma(u, u, sum);
    }
  }
  for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < kT / kWave; ++w) sum += red[w];
  const double inv = muon_inverse(sum, a.eps);
  // X [short][n] and its transpose [n][short], padded with zeros to 32 or 64 and 64s.  A thread
  // takes eight rows of the matrix at a column, which lie side by side in one of the two.
  const MuonPlaces w = muon_places(1, it.n);
  char* part = a.ws + (size_t)it.off * 256;
  char *X = part + w.x, *T = part + w.t0;
  const size_t x_row = muon_row(it.n), t_row = muon_row(1);
  const int n = it.n * kMuonPad, short_side = tall ? cols : rows, long_side = tall ? rows : cols;
  const int half = short_side <= 32 ? 1 : 2, side = half * 32;  // of the square matrices, in 32s and whole
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  {
    char *together = tall ? X : T, *apart = tall ? T : X;
    const size_t together_row = tall ? x_row : t_row, apart_row = tall ? t_row : x_row;
    const int across = tall ? side : n, down = tall ? n : side, groups = (across + kWave - 1) / kWave;
    for (int task = wave; task < down / 8 * groups; task += kT / kWave) {
      const int r0 = task / groups * 8, c = task % groups * kWave + lane;
      float gv[8], mv[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const bool there = r0 + k < rows && c < cols;
        const int e = there ? (r0 + k) * cols + c : 0;  // (a value that is not used)
        gv[k] = to_f32(g[e]);
        mv[k] = m ? m[e] : 0.f;
      }
      if (c >= across) continue;
      Pack<f16_t, 8> hi, lo;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const bool there = r0 + k < rows && c < cols;
        const float v = there ? (float)((double)muon_update_of(gv[k], mv[k], gs, a) * inv) : 0.f;
        hi.v[k] = (f16_t)v;
        lo.v[k] = (f16_t)(v - (float)hi.v[k]);
        f16_t* to = reinterpret_cast<f16_t*>(apart + (r0 + k) * apart_row + c / 32 * 128 + c % 32 * 2);
        to[0] = hi.v[k];
        to[32] = lo.v[k];
      }
      f16_t* to = reinterpret_cast<f16_t*>(together + c * together_row + r0 / 32 * 128 + r0 % 32 * 2);
      store_pack(to, hi);
      store_pack(to + 32, lo);
    }
  }
  auto slot = [&](int s) { return lds + s * kSlotBytes; };
  const int tr = wave / 4 * 16, tc = wave % 4 * 16;
  const int col = tc + lane_row(), row = tr + lane_quad() * 4;  // of a lane's four values: rows row ... row + 3
  const bool mine = tr < side && tc <= tr;  // (tiles on and below the diagonal)
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
  int product = kSlotB;
  float hold_q = 1.f;
  for (int k = 0; k < steps.count; ++k) {
    const MuonSmallSteps::Step& step = steps.step[k];
    const float back = 1.f / step.hold_b;  // (powers of two)
    __syncthreads();
    if (step.first) {
      if (mine) {
        f32x4 acc = {};
        const char *p = X + (tr + lane_row()) * x_row, *q = X + (tc + lane_row()) * x_row;
#pragma unroll 4
        for (int s = 0; s < n / 32; ++s) {
          f16x8 fp[2], fq[2];
          fragments_at(p, s, fp);
          fragments_at(q, s, fq);
          multiply(fp, fq, acc);
        }
        hold_both(slot(kSlotA), row, col, acc * (kHoldA / (kHoldX * kHoldX)));
      }
      __syncthreads();
    }
    const int b = step.first && !step.last ? kSlotQ0 : kSlotB;
    if (mine) {
      f32x4 v = square(slot(kSlotA), slot(kSlotA), half) * step.c + held(slot(kSlotA), col, row) * step.b;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (row + j == col) v[j] += step.a;
      hold_both(slot(b), row, col, v);
    }
    __syncthreads();
    // the product so far times B, and A B, then B (A B)
    const int next = step.first ? b : product == kSlotQ0 ? kSlotQ1 : kSlotQ0;
    if (mine && !step.first)
      hold_both(slot(next), row, col, square(slot(b), slot(product), half) * (step.hold_q / (step.hold_b * hold_q)));
    if (!step.last) {
      if (mine) hold_both(slot(kSlotAB), row, col, square(slot(b), slot(kSlotA), half) * back);
      __syncthreads();
      if (mine) hold_both(slot(kSlotA), row, col, square(slot(b), slot(kSlotAB), half) * back);
    }
    product = next;
    hold_q = step.hold_q;
    if (!step.last) continue;
    __syncthreads();
    // X = Q X: a wave takes 16 columns of X at a time
    const bool end = k + 1 == steps.count;
    const float scale = end ? 1.f / (step.hold_q * kHoldX) : 1.f / step.hold_q;
    for (int j0 = wave * 16; j0 < n; j0 += kT / kWave * 16) {
      const int j = j0 + lane_row();
      char* t_at = T + j * t_row;
      f16x8 fx[2][2];
#pragma unroll
      for (int s = 0; s < 2; ++s) fragments_at(t_at, min(s, half - 1), fx[s]);
#pragma unroll 1
      for (int t = 0; t < 2 * half; ++t) {
        f32x4 acc = {};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          if (s == half) break;
          f16x8 fq[2];
          fragments(slot(product), t * 16 + lane_row(), s, fq);
          multiply(fq, fx[s], acc);
        }
        acc *= scale;
        const int i = t * 16 + lane_quad() * 4;  // rows i ... i + 3 of column j
        if (end) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (i + r < short_side && j < long_side) {
              const size_t e = tall ? (size_t)j * cols + i + r : (size_t)(i + r) * cols + j;
              muon_put(static_cast<P*>(it.p), e, acc[r], (unsigned long long)it.start, keep, rate, key, a.set);
            }
        } else {
          Pack<f16_t, 4> hi, lo;
          split4(acc, hi, lo);
          // (all lanes of the wave have read their columns)
          store_pack(reinterpret_cast<f16_t*>(t_at + i / 32 * 128 + i % 32 * 2), hi);
          store_pack(reinterpret_cast<f16_t*>(t_at + i / 32 * 128 + i % 32 * 2 + 64), lo);
          f16_t* x = reinterpret_cast<f16_t*>(X + i * x_row + j / 32 * 128 + j % 32 * 2);
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            x[r * x_row / 2] = hi.v[r];
            x[r * x_row / 2 + 32] = lo.v[r];
          }
        }
      }
    }
  }
}

}  // namespace

bl_status_t muon_small(int param_dtype, int grad_dtype, const MuonList& list, const MuonSmallSteps& steps,
                       const MuonArgs& a, double flops, hipStream_t s) {
  auto go = [&](auto g, auto p) {
    auto kernel = k_muon_small<decltype(g), decltype(p)>;
    const int bytes = kSlots * kSlotBytes;
    const bl_status_t st = lds_opt_in(reinterpret_cast<const void*>(kernel), bytes);
    if (st != BL_OK) return st;
    return timed_launch("muon_small", 0.0, flops, s, [&](hipEvent_t e0, hipEvent_t e1) {
      hipExtLaunchKernelGGL(kernel, dim3((unsigned)list.count), dim3(kT), bytes, s, e0, e1, 0, list, steps, a);
    });
  };
  auto with = [&](auto g) { return param_dtype == BL_F32 ? go(g, float()) : go(g, bf16_t()); };
  return grad_dtype == BL_F32 ? with(float()) : grad_dtype == BL_BF16 ? with(bf16_t()) : with(f16_t());
}

}  // namespace blc
