// The products of Newton-Schulz steps of many matrices, in one launch each: A = X X^T, B =
// a I + b A + c A A, products of the square matrices (which commute, being polynomials of
// one, so that they are symmetric) and X = B X.
//
// Both operands of each lie with the summed index side by side: square matrices are
// symmetric, and X is held together with its transpose.  Values are two fp16 parts, v = high +
// low to 22 bits; a product takes high high + high low + low high on the matrix cores (the
// last, low low, is below 2^-22) and sums in fp32.  One fp16 part alone leaves errors of 1 %
// in the result where a gradient has a few strong directions: rounding is noise in all
// directions, and the steps raise the weak ones by up to 3.44 each.  Symmetric products
// are taken on and below the diagonal only and stored twice, in the tiles on it too: what they
// held of an antisymmetric part would grow tenfold with every joined step (64 x 1100 after five steps:
// off by 3e-5 of the norm with both halves of those tiles as computed).
//
// Bound by the matrix cores where there are many tiles: 1024 x 4096 and squares of 1024, 126 M
// values, 5.0e12 operations in 7.0 ms (0.62 of what a library's fp16 product of 8192 reaches, 1.15e15
// a second); with the 200 tiles of a residual network's grams by their fetch, 64 KB a compute
// unit in 1.25 us.
#include "muon.hpp"

namespace blc {
namespace {

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kRowBytes = 128;  // 32 values of a row, high and low parts

// A product's tile: SIDE rows of P and of Q, on kGrid x kGrid waves that hold kSub x kSub tiles
// of 32 each.  64: for launches of few blocks, with four groups of waves that take 32 of the
// summed index each in turn; 256: each value that is fetched meets the most others.  A buffer is
// fetched ahead while one is multiplied; with 128 the compute unit's other blocks cover the
// wait instead.
template <int SIDE>
struct MuonShape {
  static constexpr int kSub = SIDE == 64 ? 1 : 2;
  static constexpr int kGrid = SIDE / 32 / kSub;
  static constexpr int kGroups = SIDE == 64 ? 4 : 1;
  static constexpr int kWaves = kGrid * kGrid;           // of a group
  static constexpr int kThreads = kGroups * kWaves * kWave;
  static constexpr int kBuffers = SIDE == 128 ? 1 : 2;
  static constexpr int kRows = 2 * SIDE / kWaves;        // that a wave fetches
  static constexpr int kFetches = kRows / 8;             // of a thread for a buffer, 16 bytes each
  static constexpr int kStage = 2 * SIDE * kRowBytes;    // bytes of a group's buffer
  static constexpr int kLds = kBuffers * kGroups * kStage;
  static constexpr int kBlocks = SIDE == 128 ? 4 : 1;    // of a compute unit
};

// 32 values of kRows rows into LDS, 16 bytes a lane and eight rows an access.  A row's eight
// pieces are exchanged by half the row's number: rows of two share the 64 banks, and the lanes
// of a fragment, which lie on rows, then read all of them.
template <int SIDE>
__device__ __forceinline__ void stage(const char* from, size_t stride, char* to) {
  const int wave = threadIdx.x / kWave % MuonShape<SIDE>::kWaves, lane = threadIdx.x % kWave, row = lane / 8;
#pragma unroll
  for (int k = 0; k < MuonShape<SIDE>::kFetches; ++k) {
    const char* p = from + (size_t)(k * 8 + row) * stride + (lane % 8 ^ (k % 2 * 4 + row / 2)) * 16;
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                     (__attribute__((address_space(3))) void*)(to + (wave * MuonShape<SIDE>::kRows + k * 8) * kRowBytes),
                                     16, 0, 0);
  }
}
__device__ __forceinline__ f16x8 fragment(const char* rows, int row, int piece) {
  return *reinterpret_cast<const f16x8*>(rows + row * kRowBytes + ((piece ^ (row / 2 & 7)) * 16));
}

// What a wave holds of the product of the tile's rows: the sums over `steps` times 32 of the
// summed index, of which its group has taken every fourth 32 where there are four.  `from`: the
// rows that this wave fetches.
template <int SIDE>
struct MuonSums {
  static constexpr int N = MuonShape<SIDE>::kSub;
  f32x16 acc[N][N];

  __device__ __forceinline__ void product(const char* from, size_t stride, int steps, char* lds) {
    using S = MuonShape<SIDE>;
    constexpr int B = S::kBuffers, G = S::kGroups;
    const int wave = threadIdx.x / kWave % S::kWaves, lane = threadIdx.x % kWave;
    const int group = G == 1 ? 0 : threadIdx.x / kWave / S::kWaves;
    const int pr = wave / S::kGrid * (N * 32) + lane % 32, qr = SIDE + wave % S::kGrid * (N * 32) + lane % 32,
              half = lane / 32;
#pragma unroll
    for (int tp = 0; tp < N; ++tp)
#pragma unroll
      for (int tq = 0; tq < N; ++tq) acc[tp][tq] = f32x16{};
    if (B > 1 && group < steps) stage<SIDE>(from + (size_t)group * kRowBytes, stride, lds + group * S::kStage);
    for (int k = 0, turn = 0; k < steps; k += G, turn = (turn + 1) % B) {
      const int mine = k + group;
      if constexpr (B == 1) {
        __syncthreads();  // (the buffer has been read)
        stage<SIDE>(from + (size_t)mine * kRowBytes, stride, lds);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
      } else {
        // this wave's fetches have arrived, and its reads of the other buffer are done; behind the
        // barrier so are all waves'
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (mine + G < steps)
          stage<SIDE>(from + (size_t)(mine + G) * kRowBytes, stride, lds + ((turn ^ 1) * G + group) * S::kStage);
        if (mine >= steps) continue;
      }
      const char* now = lds + (turn * G + group) * S::kStage;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        f16x8 p[N][2], q[N][2];  // [tile][high, low]
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
          for (int l = 0; l < 2; ++l) {
            p[t][l] = fragment(now, pr + t * 32, l * 4 + s * 2 + half);
            q[t][l] = fragment(now, qr + t * 32, l * 4 + s * 2 + half);
          }
#pragma unroll
        for (int l = 0; l < 3; ++l)  // high low, low high, high high
#pragma unroll
          for (int tp = 0; tp < N; ++tp)
#pragma unroll
            for (int tq = 0; tq < N; ++tq)
              acc[tp][tq] = __builtin_amdgcn_mfma_f32_32x32x16_f16(p[tp][l == 1], q[tq][l == 0], acc[tp][tq], 0, 0, 0);
      }
    }
    __syncthreads();  // (LDS may be used again)
    if constexpr (G > 1) {
      // the groups' sums, in order; each group keeps a quarter of the rows, in acc's first four
      static_assert(G == 4 && N == 1 && G * S::kWaves * kWave * 64 <= S::kLds / 2, "room in half of LDS");
      f32x4* all = reinterpret_cast<f32x4*>(lds);
      const int at = wave * kWave + lane;
#pragma unroll
      for (int r = 0; r < 4; ++r)
        all[(group * 4 + r) * (S::kWaves * kWave) + at] = f32x4{acc[0][0][4 * r], acc[0][0][4 * r + 1], acc[0][0][4 * r + 2], acc[0][0][4 * r + 3]};
      __syncthreads();
      f32x4 sum = {};
#pragma unroll
      for (int g = 0; g < G; ++g) sum += all[(g * 4 + group) * (S::kWaves * kWave) + at];
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[0][0][k] = sum[k];
    }
  }

  // go(row, column, v) for every four rows of a column that this lane has of the tile, rows P's
  // and columns Q's: row ... row + 3; those of the wave's tiles tp.
  template <typename Go>
  __device__ __forceinline__ void each_four(int tp, Go&& go) const {
    using S = MuonShape<SIDE>;
    const int wave = threadIdx.x / kWave % S::kWaves, lane = threadIdx.x % kWave, group = threadIdx.x / kWave / S::kWaves;
#pragma unroll
    for (int tq = 0; tq < N; ++tq)
#pragma unroll
      for (int r = 0; r < 4 / S::kGroups; ++r) {
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = acc[tp][tq][4 * r + k];
        go((wave / S::kGrid * N + tp) * 32 + (S::kGroups > 1 ? group : r) * 8 + lane / 32 * 4,
           (wave % S::kGrid * N + tq) * 32 + lane % 32, v);
      }
  }
};

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

// Blocks go to the GPU's eight dies in turn, each with a cache of its own: a die takes `each`
// neighbouring tiles, which share rows, then as many further on, so that all dies work at
// the long sums, which lie at the front, for as long; the last ones go evenly over the dies
// (products of squares up to 512: 10.4 and 10.7 us, in the order of the blocks 12.1 and 13.0).
template <int SIDE>
__device__ __forceinline__ unsigned near_tile(unsigned block, unsigned blocks) {
  constexpr unsigned each = SIDE == 256 ? 16 : 32, turn = 8 * each;
  const unsigned first = block / turn * turn;
  const unsigned rest = min(blocks - first, turn), die = block % 8;
  return first + die * (rest / 8) + min(die, rest % 8) + block % turn / 8;
}

// What a block's tile is: matrix, place and the rows that this thread's wave fetches.
struct MuonTilePlace {
  unsigned at, m, n, ti, tj, p_rows, q_rows;  // m, n and the rows that there are of P and Q: in 64s
  template <int SIDE, bool TRIANGLE>
  __device__ __forceinline__ static MuonTilePlace make(const unsigned* first, int count, const unsigned short* ms,
                                                       const unsigned short* ns, unsigned block) {
    MuonTilePlace p;
    p.at = muon_find(first, count, block);
    const unsigned tile = block - first[p.at];
    p.m = ms[p.at];
    p.n = ns[p.at];
    if (TRIANGLE) {  // on and below the diagonal
      p.ti = (unsigned)((sqrtf(8.f * tile + 1.f) - 1.f) * 0.5f);
      while ((p.ti + 1) * (p.ti + 2) / 2 <= tile) ++p.ti;
      while (p.ti * (p.ti + 1) / 2 > tile) --p.ti;
      p.tj = tile - p.ti * (p.ti + 1) / 2;
    } else {
      const unsigned across = (p.m + SIDE / 64 - 1) / (SIDE / 64);
      p.ti = tile % across;
      p.tj = tile / across;
    }
    p.p_rows = min(p.m - p.ti * (SIDE / 64), (unsigned)SIDE / 64);
    p.q_rows = min((TRIANGLE ? p.m : p.n) - p.tj * (SIDE / 64), (unsigned)SIDE / 64);
    return p;
  }
};
// The rows that this wave fetches; in the place of a 64 of them that there is not, the last one
// (whose products are not stored).
template <int SIDE>
__device__ __forceinline__ const char* fetched(const char* P, const char* Q, size_t stride, const MuonTilePlace& p) {
  using S = MuonShape<SIDE>;
  const unsigned wave = threadIdx.x / kWave % S::kWaves, row = wave * S::kRows % SIDE;
  const bool first = wave < S::kWaves / 2;
  const unsigned part = min(row / 64, (first ? p.p_rows : p.q_rows) - 1);
  return (first ? P + (size_t)p.ti * SIDE * stride : Q + (size_t)p.tj * SIDE * stride) + (part * 64 + row % 64) * stride;
}
// Whether there is this wave's part of the tile.
template <int SIDE>
__device__ __forceinline__ bool wave_there(const MuonTilePlace& p) {
  using S = MuonShape<SIDE>;
  const unsigned wave = threadIdx.x / kWave;
  return SIDE == 64 || (wave / S::kGrid < p.p_rows && wave % S::kGrid < p.q_rows);
}

template <int MODE, int SIDE>
__global__ __launch_bounds__(MuonShape<SIDE>::kThreads, MuonShape<SIDE>::kBlocks) void k_muon_product(MuonShapes list, MuonProduct q) {
  using S = MuonShape<SIDE>;
  // 32 rows of each wave at a time are turned by way of LDS
  static_assert(S::kLds >= S::kGrid * 32 * SIDE * 4 * (S::kGroups > 1 ? 2 : 1), "room for them");
  extern __shared__ __align__(16) char lds[];
  const unsigned blocks = MODE == kSquare ? list.first[kMuonList] : gridDim.x;
  const bool second = MODE == kSquare && blockIdx.x >= blocks;
  const MuonTilePlace p = MuonTilePlace::make<SIDE, MODE != kApply>(
      list.first, list.count, list.m, list.n, near_tile<SIDE>(second ? blockIdx.x - blocks : blockIdx.x, blocks));
  const MuonPlaces w = muon_places(p.m, p.n);
  char* part = q.ws + (size_t)list.off[p.at] * 256;
  const unsigned sum = MODE == kGram ? p.n : p.m;  // of the summed index
  const size_t stride = muon_row(sum), mm = muon_row(p.m), nn = muon_row(p.n);
  const char* P = part + (MODE == kGram ? w.x : w.slot(q.p));
  const char* Q = MODE == kApply ? part + w.t(q.turn) : MODE == kSquare ? part + w.slot(second ? q.q2 : q.q) : P;
  MuonSums<SIDE> sums;
  sums.product(fetched<SIDE>(P, Q, stride, p), stride, (int)sum * 2, lds);
  float* tiled = reinterpret_cast<float*>(lds + (S::kGroups > 1 ? S::kLds / 2 : 0));
  // columns of the tile are rows of the transpose: four of a lane's values lie side by side
  char* across = part + (MODE == kApply ? w.t(q.turn ^ 1) : w.slot(second ? q.out2 : q.out));
  char* along = MODE == kApply ? part + w.x : across;
  const size_t along_row = MODE == kApply ? nn : mm;
  const float scale = second ? q.scale2 : q.scale;
  // (on the diagonal the values below it, with what of their blocks of 8 x 8 lies on it read from both sides)
  const bool diagonal = MODE != kApply && p.ti == p.tj, there = wave_there<SIDE>(p);
#pragma unroll
  for (int tp = 0; tp < S::kSub; ++tp) {
    if (there)
      sums.each_four(tp, [&](int row, int col, float (&v)[4]) {
        const size_t place = held_at((size_t)p.tj * SIDE + col, mm, p.ti * SIDE + row);
        if (MODE == kPoly) {
          const char* from = P + place;
          const Pack<f16_t, 4> hi = load_pack<f16_t, 4>(reinterpret_cast<const f16_t*>(from)),
                               lo = load_pack<f16_t, 4>(reinterpret_cast<const f16_t*>(from + 64));
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            v[k] = fmaf(q.c, v[k], q.b * ((float)hi.v[k] + (float)lo.v[k]));
            if (p.ti == p.tj && row + k == col) v[k] += q.a;
          }
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] *= scale;
        }
        if (!diagonal || row / 8 > col / 8) hold<4>(across + place, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) tiled[(row / (S::kSub * 32) * 32 + row % 32 + k) * SIDE + col] = v[k];
      });
    __syncthreads();
    for (int i = threadIdx.x; i < S::kGrid * 32 * SIDE / 8; i += S::kThreads) {
      const int r = i / (SIDE / 8), c = i % (SIDE / 8) * 8, row = (r / 32 * S::kSub + tp) * 32 + r % 32;
      if (SIDE > 64 && ((unsigned)row / 64 >= p.p_rows || (unsigned)c / 64 >= p.q_rows)) continue;
      if (diagonal && row / 8 < c / 8) continue;
      const bool turned = diagonal && row / 8 == c / 8;
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int up = turned ? max(c + j - row, 0) : 0;  // from above the diagonal to below it
        v[j] = tiled[(r + up) * SIDE + c + j - up];
      }
      hold<8>(along + held_at((size_t)p.ti * SIDE + row, along_row, p.tj * SIDE + c), v);
    }
    if (tp + 1 < S::kSub) __syncthreads();
  }
}

// The last step: X goes into the parameters.
template <int SIDE, typename P>
__global__ __launch_bounds__(MuonShape<SIDE>::kThreads, MuonShape<SIDE>::kBlocks) void k_muon_update(MuonList list, MuonProduct q, MuonArgs a) {
  using S = MuonShape<SIDE>;
  extern __shared__ __align__(16) char lds[];
  const unsigned block = near_tile<SIDE>(blockIdx.x, gridDim.x), at = muon_find(list.first, list.count, block), none = 0;
  const MuonItem& it = list.item[at];
  const MuonTilePlace p = MuonTilePlace::make<SIDE, false>(&none, 1, &it.m, &it.n, block - list.first[at]);
  const MuonPlaces w = muon_places(p.m, p.n);
  const char* part = q.ws + (size_t)it.off * 256;
  const size_t stride = muon_row(p.m);
  MuonSums<SIDE> sums;
  sums.product(fetched<SIDE>(part + w.slot(q.p), part + w.t(q.turn), stride, p), stride, (int)p.m * 2, lds);
  if (!wave_there<SIDE>(p)) return;
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
  P* param = static_cast<P*>(it.p);
  const int rows = it.rows, cols = it.cols;
  const bool tall = it.tall;
  const unsigned long long start = (unsigned long long)it.start;
#pragma unroll
  for (int tp = 0; tp < S::kSub; ++tp) {
    P old[S::kSub * 16 / S::kGroups] = {};
    auto each = [&](auto&& go) {  // go(old value, element, v) for all that there are
      int n = 0;
      sums.each_four(tp, [&](int row, int col, const float (&v)[4]) {
#pragma unroll
        for (int k = 0; k < 4; ++k, ++n) {
          const int i = (int)p.ti * SIDE + row + k, j = (int)p.tj * SIDE + col, r = tall ? j : i, c = tall ? i : j;
          if (r < rows && c < cols) go(old[n], (size_t)r * cols + c, v[k]);
        }
      });
    };
    // all old values are in flight before the first is used
    if (!a.set) each([&](P& o, size_t e, float) { o = param[e]; });
    each([&](P& o, size_t e, float v) {
      param[e] = muon_next<P>(to_f32(o), v * q.scale, start + e, keep, rate, key, a.set);
    });
  }
}

}  // namespace

// go(side) as a constant.
template <typename Go>
bl_status_t with_side(int side, Go&& go) {
  if (side == 64) return go(std::integral_constant<int, 64>());
  if (side == 128) return go(std::integral_constant<int, 128>());
  return go(std::integral_constant<int, 256>());
}

bl_status_t muon_product(int mode, int side, const MuonShapes& shapes, unsigned blocks, double flops,
                         const MuonProduct& q, hipStream_t s) {
  const char* names[] = {"muon_gram", "muon_poly", "muon_square", "muon_apply"};
  if (mode == kSquare && q.q2 >= 0) blocks *= 2;
  return with_side(side, [&](auto n) {
    using S = MuonShape<decltype(n)::value>;
    constexpr int N = decltype(n)::value;
    auto kernel = mode == kGram ? k_muon_product<kGram, N> : mode == kPoly ? k_muon_product<kPoly, N>
                  : mode == kSquare ? k_muon_product<kSquare, N> : k_muon_product<kApply, N>;
    const bl_status_t st = lds_opt_in(reinterpret_cast<const void*>(kernel), S::kLds);
    if (st != BL_OK) return st;
    return timed_launch(names[mode], 0.0, flops, s, [&](hipEvent_t e0, hipEvent_t e1) {
      hipExtLaunchKernelGGL(kernel, dim3(blocks), dim3(S::kThreads), S::kLds, s, e0, e1, 0, shapes, q);
    });
  });
}

bl_status_t muon_update(int param_dtype, int side, const MuonList& list, unsigned blocks, double flops,
                        const MuonProduct& q, const MuonArgs& a, hipStream_t s) {
  return with_side(side, [&](auto n) {
    using S = MuonShape<decltype(n)::value>;
    auto kernel = param_dtype == BL_F32 ? k_muon_update<decltype(n)::value, float> : k_muon_update<decltype(n)::value, bf16_t>;
    const bl_status_t st = lds_opt_in(reinterpret_cast<const void*>(kernel), S::kLds);
    if (st != BL_OK) return st;
    return timed_launch("muon_update", 0.0, flops, s, [&](hipEvent_t e0, hipEvent_t e1) {
      hipExtLaunchKernelGGL(kernel, dim3(blocks), dim3(S::kThreads), S::kLds, s, e0, e1, 0, list, q, a);
    });
  });
}

}  // namespace blc
