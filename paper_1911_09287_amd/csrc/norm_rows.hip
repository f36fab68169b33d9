// Layer norm of rows (inner = 1).
//
// A row stays in the registers of the lanes that hold it: it is read once, its
// mean and then the squares of what differs from the mean are summed over the
// lanes, and it is written once (backward: x and dy are read once, the two sums
// of u and u h taken together).  Bound by HBM.  Short rows lie on 1 to 64 lanes
// of a wave, long ones on a block; rows that a block's registers do not hold are cut
// over many blocks, in two launches: partial statistics, then the result.  The sums
// over rows that dw and db are come from sums that a thread keeps for its columns
// over its block's rows, in registers, and a last small launch.
//
// Measured (kernel, bytes read and written once): 16384 rows of 1024 fp32 values
// forward 27 us, 4.9 TB/s, backward 38 us, 5.2 TB/s; of 2048 bfloat16 values 33 us,
// 4.1 TB/s, and 43 us, 4.7 TB/s (twice the values to convert for the same bytes);
// 4096 of 8192 fp32 values 52 us, 5.2 TB/s, and 82 us, 4.9 TB/s (of over 8192
// backward 4.3 TB/s: a lane's 128 registers are short by five); 32 of 200704 fp32
// values, two launches, 6.3 + 11 us forward, 10 + 19 us backward while the tensors lie
// in the 256 MB cache, 8.3 + 11 and 14 + 19 from memory.
#include <algorithm>

#include "norm.hpp"

namespace blc {
namespace {

constexpr int kT = kNormThreads;
constexpr int kMostThreads = 1024;
constexpr int kTargetBlocks = 512;  // two a compute unit
// Seven a compute unit (half of them / these / twice: 32 rows of 200704 fp32 values
// 12.0 / 11.4 / 12.6 us, 200 of 50000 14.9 / 13.4 / 13.9, 2000 of 60000 bfloat16 127 / 114 / 109).
constexpr int kSplitBlocks = 1792;

// ---- sums over the lanes of a row ---------------------------------------------
// BLOCK: over the block, by way of LDS; `red` alternates between two arrays from
// one sum to the next, so that one barrier a sum is enough.
template <bool BLOCK, int N>
__device__ __forceinline__ void row_sum(float (&x)[N], int lanes, float (*red)[kMostThreads / kWave]) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = wave_sum(x[i], BLOCK ? kWave : lanes);
  if (!BLOCK) return;
  const int wave = threadIdx.x / kWave, waves = blockDim.x / kWave;  // a multiple of 4
  if (threadIdx.x % kWave == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) red[i][wave] = x[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    x[i] = 0.f;
    for (int k = 0; k < waves; k += 4) {
      const float4 r = *reinterpret_cast<const float4*>(&red[i][k]);
      x[i] += (r.x + r.y) + (r.z + r.w);
    }
  }
}

// A thread's first row; where it is the whole wave's the compiler is told so.
template <bool BLOCK, int E>
__device__ __forceinline__ long first_row(int lanes) {
  if (BLOCK) return blockIdx.x;
  const int in_block = threadIdx.x / lanes;
  return (long)blockIdx.x * (kT / lanes) + (E > 1 ? __builtin_amdgcn_readfirstlane(in_block) : in_block);
}

// E vectors of 16 bytes a lane; their weights are kept over a block's rows.
template <typename T, int E, bool BLOCK>
__global__ __launch_bounds__(BLOCK ? kMostThreads : kT) void k_rows_fwd(NormPtrs a, bl_norm_desc_t d, int lanes) {
  constexpr int V = 16 / sizeof(T);
  __shared__ __align__(16) float red[2][1][kMostThreads / kWave];
  if (!BLOCK && E > 1) lanes = kWave;  // (rows of more than 64 vectors)
  const int in = BLOCK ? threadIdx.x : threadIdx.x % lanes, step = BLOCK ? blockDim.x : lanes;
  const long rows = d.outer, M = d.size;
  const long each = BLOCK ? 1 : kT / lanes;
  const bool wide = d.wdtype == BL_F32;
  float w[E][V], b[E][V];
  load_weights<T, V, E>(a.w, wide, (long)in * V, (long)step * V, M, 1.f, w);
  load_weights<T, V, E>(a.b, wide, (long)in * V, (long)step * V, M, 0.f, b);
  for (long row = first_row<BLOCK, E>(lanes); row < rows; row += gridDim.x * each) {
    const T* x = static_cast<const T*>(a.x) + row * d.x_stride;
    T* y = static_cast<T*>(a.y) + row * d.y_stride;
    Held<T, V> v[E];
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const unsigned i = (in + k * step) * V;
      v[k].load(at_bytes(x, i * sizeof(T)), M - (long)i);
    }
#pragma unroll
    for (int k = 0; k < E; ++k) {
      v[k].refresh();
#pragma unroll
      for (int j = 0; j < V; ++j) s[0] += v[k][j];
    }
    row_sum<BLOCK>(s, lanes, red[0]);
    const float mean = s[0] / (float)M;
    s[0] = 0.f;
#pragma unroll
    for (int k = 0; k < E; ++k) {
      v[k].refresh();
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float c = v[k][j] - mean;
        s[0] += (long)(in + k * step) * V + j < M ? c * c : 0.f;
      }
      v[k].refresh();
    }
    row_sum<BLOCK>(s, lanes, red[1]);
    const float rstd = 1.f / sqrtf(s[0] / (float)M + (float)d.eps);
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const unsigned i = (in + k * step) * V;
      Pack<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) o.v[j] = (T)fmaf((v[k][j] - mean) * rstd, w[k][j], b[k][j]);
      store_part<T, V>(at_bytes(y, i * sizeof(T)), M - (long)i, o);
    }
    if (a.stats && in == 0) {
      a.stats[row] = mean;
      a.stats[rows + row] = rstd;
    }
  }
}

// Element i of a row: of a row that one wave holds by a shared address and a lane's
// offset.  (In a block of 1024 with four vectors a lane that costs the registers that
// are left: 2000 rows of 16384 fp32 values backward take 111 us with it, 95 without.)
template <bool BLOCK, typename T>
__device__ __forceinline__ T* place(T* row, long i) {
  return BLOCK ? row + i : at_bytes(row, (unsigned)i * (unsigned)sizeof(T));
}

// dx; and where part is given this block's sums of dy h and dy by column, [block][2][M].
template <typename T, int E, bool BLOCK>
__global__ __launch_bounds__(BLOCK ? kMostThreads : kT) void k_rows_bwd(NormPtrs a, bl_norm_desc_t d, int lanes,
                                                                        bool sums) {
  constexpr int V = 16 / sizeof(T);
  __shared__ __align__(16) float red[2][2][kMostThreads / kWave];
  __shared__ float comb[BLOCK ? 1 : 2 * kWave * E * V];
  if (!BLOCK && E > 1) lanes = kWave;  // (rows of more than 64 vectors)
  const int in = BLOCK ? threadIdx.x : threadIdx.x % lanes, step = BLOCK ? blockDim.x : lanes;
  const long rows = d.outer, M = d.size;
  const long each = BLOCK ? 1 : kT / lanes;
  const float inv = 1.f / (float)M;
  float w[E][V], aw[E][V] = {}, ab[E][V] = {};
  load_weights<T, V, E>(a.w, d.wdtype == BL_F32, (long)in * V, (long)step * V, M, 1.f, w);
  int turn = 0;
  for (long row = first_row<BLOCK, E>(lanes); row < rows; row += gridDim.x * each) {
    const T* x = static_cast<const T*>(a.x) + row * d.x_stride;
    const T* dy = static_cast<const T*>(a.dy) + row * d.y_stride;
    T* dx = static_cast<T*>(a.dx) + row * d.x_stride;
    Held<T, V> v[E], g[E];
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const long i = (long)(in + k * step) * V;
      v[k].load(place<BLOCK>(x, i), M - i);
      g[k].load(place<BLOCK>(dy, i), M - i);
    }
    const float mean = a.stats[row], rstd = a.stats[rows + row];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < E; ++k) {
      v[k].refresh();
      g[k].refresh();
#pragma unroll
      for (int j = 0; j < V; ++j) {  // (past the row dy is 0)
        const float h = (v[k][j] - mean) * rstd, dyj = g[k][j], u = dyj * w[k][j];
        if (E == 1) {
          add_sums(u, h, s[0], s[1]);
        } else {  // rows of hundreds of values: no sum is exact, and registers count (105 us for the 95 above)
          s[0] += u;
          s[1] = fmaf(u, h, s[1]);
        }
        aw[k][j] = fmaf(dyj, h, aw[k][j]);
        ab[k][j] += dyj;
      }
      v[k].refresh();
      g[k].refresh();
    }
    row_sum<BLOCK>(s, lanes, red[turn]);
    turn ^= 1;
    const float c1 = s[0] * inv, c2 = s[1] * inv;
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const long i = (long)(in + k * step) * V;
      Pack<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float h = (v[k][j] - mean) * rstd;
        o.v[j] = (T)grad_of(g[k][j] * w[k][j], c1, h, c2, rstd);
      }
      store_part<T, V>(place<BLOCK>(dx, i), M - i, o);
    }
  }
  if (!sums) return;
  float* part = a.part + (size_t)blockIdx.x * 2 * M;
  if (BLOCK) {
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const long i = (long)(in + k * step) * V;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (i + j < M) {
          part[i + j] = aw[k][j];
          part[M + i + j] = ab[k][j];
        }
    }
    return;
  }
  // the rows of a wave, then the waves in order
#pragma unroll
  for (int k = 0; k < E; ++k)
#pragma unroll
    for (int j = 0; j < V; ++j)
      for (int o = lanes; o < kWave; o <<= 1) {
        aw[k][j] += __shfl_xor(aw[k][j], o);
        ab[k][j] += __shfl_xor(ab[k][j], o);
      }
  const int width = lanes * E * V;  // >= M
  for (int wave = 0; wave < kT / kWave; ++wave) {
    if ((int)threadIdx.x / kWave == wave && (int)(threadIdx.x % kWave) < lanes)
#pragma unroll
      for (int k = 0; k < E; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
          float* c = comb + (in + k * step) * V + j;
          c[0] = aw[k][j] + (wave ? c[0] : 0.f);
          c[width] = ab[k][j] + (wave ? c[width] : 0.f);
        }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < M; i += kT) {
    part[i] = comb[i];
    part[M + i] = comb[width + i];
  }
}

// ---- rows over several blocks ---------------------------------------------------
// A block takes a chunk of a row, each of its waves a piece of that, in tiles of
// four vectors a lane that are in flight together.  The first launch leaves two sums
// for each piece; no wave waits for another.
constexpr int kTileVecs = 4;
constexpr int kBlockWaves = kT / kWave;
constexpr int kMostChunks = kT / kBlockWaves;  // so that a block joins a row's pieces, one a thread

struct Split {
  long piece;   // elements of a wave, a multiple of its tile
  int pieces;   // of a row, kBlockWaves a block
};
template <typename T>
__device__ __forceinline__ long wave_tile() {
  return (long)kWave * (16 / (int)sizeof(T)) * kTileVecs;
}

// Forward: mean and sum of squared differences from it of one piece of one row.  A
// tile's are exact to fp32 (the mean first), tiles are joined by the update for two
// sets: n, mean and M2 of both give n, mean and M2 of the union.
template <typename T>
__global__ __launch_bounds__(kT) void k_split_stats(NormPtrs a, bl_norm_desc_t d, Split c) {
  constexpr int V = 16 / sizeof(T);
  const int chunks = c.pieces / kBlockWaves, lane = threadIdx.x % kWave;
  const long row = blockIdx.x / (unsigned)chunks;
  const int piece = blockIdx.x % (unsigned)chunks * kBlockWaves + threadIdx.x / kWave;
  const long from = piece * c.piece, to = min((long)d.size, from + c.piece);
  const T* x = static_cast<const T*>(a.x) + row * d.x_stride;
  float n = 0.f, mean = 0.f, m2 = 0.f;
  for (long at = from; at < to; at += wave_tile<T>()) {
    Held<T, V> v[kTileVecs];
    float s = 0.f, q = 0.f;
#pragma unroll
    for (int k = 0; k < kTileVecs; ++k) {
      const long i = at + (long)(lane + k * kWave) * V;
      v[k].load(x + i, to - i);
    }
#pragma unroll
    for (int k = 0; k < kTileVecs; ++k) {
      v[k].refresh();
#pragma unroll
      for (int j = 0; j < V; ++j) s += v[k][j];
    }
    const float nt = (float)min(wave_tile<T>(), to - at), mt = wave_sum(s) / nt;
#pragma unroll
    for (int k = 0; k < kTileVecs; ++k)
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float c0 = v[k][j] - mt;
        q += at + (long)(lane + k * kWave) * V + j < to ? c0 * c0 : 0.f;
      }
    const float all = n + nt, diff = mt - mean;
    mean += diff * (nt / all);
    m2 += wave_sum(q) + diff * diff * (n * nt / all);
    n = all;
  }
  if (lane < 2) a.sums[((size_t)row * c.pieces + piece) * 2 + lane] = lane ? m2 : mean;
}

// y of one tile of two vectors a thread of every groups-th row.  The tile's weights
// stay in registers over the rows (in 16 bits they are four times the values).
constexpr int kFwdVecs = 2;
constexpr int kRowsKnown = 128;  // rows whose statistics are in LDS at a time
template <typename T>
__global__ __launch_bounds__(kT) void k_split_fwd(NormPtrs a, bl_norm_desc_t d, Split c, unsigned tiles, int groups) {
  constexpr int V = 16 / sizeof(T), kJoin = kMostChunks * kBlockWaves / kWave;
  __shared__ float2 known[kRowsKnown];  // mean and rstd
  const int lane = threadIdx.x % kWave;
  const long first = blockIdx.x / tiles, M = d.size;
  const long i = ((long)(blockIdx.x % tiles) * kFwdVecs * kT + threadIdx.x) * V;  // and kT V further
  const long rows = (d.outer - first + groups - 1) / groups;                      // of this block
  const T* x = static_cast<const T*>(a.x) + first * d.x_stride + i;
  T* y = static_cast<T*>(a.y) + first * d.y_stride + i;
  Held<T, V> v[kFwdVecs];
#pragma unroll
  for (int k = 0; k < kFwdVecs; ++k) v[k].load(x + k * kT * V, M - i - k * kT * V);
  float w[kFwdVecs][V], b[kFwdVecs][V];
  load_weights<T, V, kFwdVecs>(a.w, d.wdtype == BL_F32, i, kT * V, M, 1.f, w);
  load_weights<T, V, kFwdVecs>(a.b, d.wdtype == BL_F32, i, kT * V, M, 0.f, b);
  for (long r0 = 0; r0 < rows; r0 += kRowsKnown) {
    const int n = (int)min((long)kRowsKnown, rows - r0);
    if (r0) __syncthreads();
    for (int r = threadIdx.x / kWave; r < n; r += kBlockWaves) {
      const long row = first + (r0 + r) * groups;
      const float* all = a.sums + (size_t)row * c.pieces * 2;
      float mc[kJoin], nc[kJoin], s = 0.f, q = 0.f;
#pragma unroll
      for (int u = 0; u < kJoin; ++u) {
        const int p = lane + u * kWave;
        const long left = M - p * c.piece;
        nc[u] = p < c.pieces && left > 0 ? (float)min(c.piece, left) : 0.f;
        mc[u] = nc[u] > 0.f ? all[2 * p] : 0.f;
        q += nc[u] > 0.f ? all[2 * p + 1] : 0.f;
        s = fmaf(nc[u], mc[u], s);
      }
      const float mean = wave_sum(s) / (float)M;
#pragma unroll
      for (int u = 0; u < kJoin; ++u) q = fmaf(nc[u] * (mc[u] - mean), mc[u] - mean, q);
      const float rstd = 1.f / sqrtf(wave_sum(q) / (float)M + (float)d.eps);
      if (lane == 0) known[r] = make_float2(mean, rstd);
      if (a.stats && blockIdx.x % tiles == 0 && lane == 0) {
        a.stats[row] = mean;
        a.stats[d.outer + row] = rstd;
      }
    }
    __syncthreads();
    for (int r = 0; r < n; ++r) {
      const float2 t = known[r];
      Pack<T, V> o[kFwdVecs];
#pragma unroll
      for (int k = 0; k < kFwdVecs; ++k) {
        v[k].refresh();
#pragma unroll
        for (int j = 0; j < V; ++j) o[k].v[j] = (T)fmaf((v[k][j] - t.x) * t.y, w[k][j], b[k][j]);
      }
      if (r0 + r + 1 < rows) {  // the next row is on its way while this one is stored
        x += (long)groups * d.x_stride;
#pragma unroll
        for (int k = 0; k < kFwdVecs; ++k) v[k].load(x + k * kT * V, M - i - k * kT * V);
      }
#pragma unroll
      for (int k = 0; k < kFwdVecs; ++k) store_part<T, V>(y + k * kT * V, M - i - k * kT * V, o[k]);
      y += (long)groups * d.y_stride;
    }
  }
}

// Backward: sums of u and u h of one piece of one row.
template <typename T>
__global__ __launch_bounds__(kT) void k_split_sums(NormPtrs a, bl_norm_desc_t d, Split c) {
  constexpr int V = 16 / sizeof(T);
  const int chunks = c.pieces / kBlockWaves, lane = threadIdx.x % kWave;
  const long row = blockIdx.x / (unsigned)chunks;
  const int piece = blockIdx.x % (unsigned)chunks * kBlockWaves + threadIdx.x / kWave;
  const long from = piece * c.piece, to = min((long)d.size, from + c.piece);
  const T* x = static_cast<const T*>(a.x) + row * d.x_stride;
  const T* dy = static_cast<const T*>(a.dy) + row * d.y_stride;
  const float mean = a.stats[row], rstd = a.stats[d.outer + row];
  float s0 = 0.f, s1 = 0.f;
  for (long at = from; at < to; at += wave_tile<T>()) {
    Held<T, V> v[kTileVecs], g[kTileVecs];
#pragma unroll
    for (int k = 0; k < kTileVecs; ++k) {
      const long i = at + (long)(lane + k * kWave) * V;
      v[k].load(x + i, to - i);
      g[k].load(dy + i, to - i);
    }
    float w[kTileVecs][V];
    load_weights<T, V, kTileVecs>(a.w, d.wdtype == BL_F32, at + (long)lane * V, kWave * V, to, 1.f, w);
#pragma unroll
    for (int k = 0; k < kTileVecs; ++k) {
      v[k].refresh();
      g[k].refresh();
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float h = (v[k][j] - mean) * rstd, u = g[k][j] * w[k][j];
        add_sums(u, h, s0, s1);
      }
    }
  }
  s0 = wave_sum(s0);
  s1 = wave_sum(s1);
  if (lane < 2) a.sums[((size_t)row * c.pieces + piece) * 2 + lane] = lane ? s1 : s0;
}

// dx of one chunk of every groups-th row, and this block's sums by column,
// [group][2][M].  One vector a thread, so that the sums stay in registers, and four
// rows in flight together.
constexpr int kRowsFlying = 4;
template <typename T>
__global__ __launch_bounds__(kT) void k_split_bwd(NormPtrs a, bl_norm_desc_t d, Split c, int groups, bool sums) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float4 known[kRowsKnown];  // mean, rstd and the means of u and u h
  const int chunks = c.pieces / kBlockWaves, lane = threadIdx.x % kWave;
  const long chunk = c.piece * kBlockWaves, M = d.size;
  const long first = blockIdx.x / (unsigned)chunks, from = blockIdx.x % (unsigned)chunks * chunk;
  const long to = min(M, from + chunk), rows = (d.outer - first + groups - 1) / groups;  // of this block
  for (long at = from; at < to; at += (long)kT * V) {
    const long i = at + (long)threadIdx.x * V;
    float w[1][V], aw[V] = {}, ab[V] = {};
    load_weights<T, V, 1>(a.w, d.wdtype == BL_F32, i, 0, to, 1.f, w);
    for (long r0 = 0; r0 < rows; r0 += kRowsKnown) {
      const int n = (int)min((long)kRowsKnown, rows - r0);
      if (at == from || rows > kRowsKnown) {
        __syncthreads();
        for (int r = threadIdx.x / kWave; r < n; r += kBlockWaves) {
          const long row = first + (r0 + r) * groups;
          const float* all = a.sums + (size_t)row * c.pieces * 2;
          float s0 = 0.f, s1 = 0.f;
          for (int p = lane; p < c.pieces; p += kWave) s0 += all[2 * p], s1 += all[2 * p + 1];
          s0 = wave_sum(s0);
          s1 = wave_sum(s1);
          if (lane == 0) known[r] = make_float4(a.stats[row], a.stats[d.outer + row], s0 / (float)M, s1 / (float)M);
        }
        __syncthreads();
      }
      for (int r = 0; r < n; r += kRowsFlying) {
        Held<T, V> v[kRowsFlying], g[kRowsFlying];
#pragma unroll
        for (int k = 0; k < kRowsFlying; ++k) {
          const long row = first + (r0 + r + k) * groups, left = r + k < n ? to - i : 0;
          v[k].load(static_cast<const T*>(a.x) + row * d.x_stride + i, left);
          g[k].load(static_cast<const T*>(a.dy) + row * d.y_stride + i, left);
        }
#pragma unroll
        for (int k = 0; k < kRowsFlying; ++k) {
          if (r + k >= n) break;
          const long row = first + (r0 + r + k) * groups;
          const float4 t = known[r + k];
          v[k].refresh();
          g[k].refresh();
          Pack<T, V> o;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float h = (v[k][j] - t.x) * t.y, dyj = g[k][j];
            aw[j] = fmaf(dyj, h, aw[j]);
            ab[j] += dyj;
            o.v[j] = (T)grad_of(dyj * w[0][j], t.z, h, t.w, t.y);
          }
          store_part<T, V>(static_cast<T*>(a.dx) + row * d.x_stride + i, to - i, o);
        }
      }
    }
    if (!sums) continue;
    float* part = a.part + (size_t)first * 2 * M;
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (i + j < to) {
        part[i + j] = aw[j];
        part[M + i + j] = ab[j];
      }
  }
}

// How a row of nv vectors lies on lanes, `most` vectors on one at most: on a wave up to
// four a lane, else on a block.  16384 rows, wave / block of 256, forward and backward:
// 600 fp32 values 14.9 / 22.2 and 27 / 41 us, 1024 27.1 / 29.7 and 38 / 43, 2048
// bfloat16 33 / 35 and 43 / 52.  Of 2048 fp32 values, eight on a wave / block: 53.5 / 51
// and 77 / 71; of 4096 bfloat16 63 / 61 and 108 / 83.
bl_norm_rows rows_shape(long nv, int most, bool backward) {
  bl_norm_rows r{};
  if (nv <= 4L * kWave) {
    r.each = nv <= kWave ? 1 : nv <= 2 * kWave ? 2 : 4;
    r.threads = 1;
    while ((long)r.threads * r.each < nv) r.threads *= 2;
    return r;
  }
  r.block = true;
  r.each = 2;
  r.threads = 256;
  while ((long)r.threads * r.each < nv) {
    if (r.each < (backward ? 2 : 4)) r.each *= 2;
    else if (r.threads < kMostThreads) r.threads *= 2;
    else if (r.each < most) r.each *= 2;
    else return bl_norm_rows{true, 0, 0};  // does not fit
  }
  return r;
}

template <typename T, bool BLOCK>
bl_status_t launch_fwd(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  const bl_norm_rows& r = p->fwd;
  const long each = BLOCK ? 1 : kT / r.threads;
  // A block reads the weights once, so no more blocks than run at a time, 1024 threads a
  // compute unit (2000 rows of 32768 fp32 values 108 us, with four times as many 117;
  // 16384 of 2048 bfloat16 values 34, with twice as many 35), but twice as many where a
  // wave holds its row in two vectors a lane (65536 of 256 fp32 values 27, with half 30).
  const long cap = BLOCK ? 2 * kTargetBlocks * kT / r.threads : r.each > 2 ? 2 * kTargetBlocks : 4 * kTargetBlocks;
  const unsigned blocks = (unsigned)std::min<long>((p->d.outer + each - 1) / each, cap);
  const double bytes = 2.0 * p->d.outer * p->d.size * sizeof(T);
  return timed_launch("norm_fwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    auto go = [&](auto kernel) {
      hipExtLaunchKernelGGL(kernel, dim3(blocks), dim3(BLOCK ? r.threads : kT), 0, s, e0, e1, 0, a, p->d, r.threads);
    };
    if (r.each == 1) go(k_rows_fwd<T, 1, false>);
    else if (r.each == 2) go(k_rows_fwd<T, 2, BLOCK>);
    else if (r.each == 4) go(k_rows_fwd<T, 4, BLOCK>);
    else go(k_rows_fwd<float, 8, true>);
  });
}

template <typename T, bool BLOCK>
bl_status_t launch_bwd(const bl_norm_plan_s* p, const NormPtrs& a, bool sums, hipStream_t s) {
  const bl_norm_rows& r = p->bwd;
  const double bytes = 3.0 * p->d.outer * p->d.size * sizeof(T);
  return timed_launch("norm_bwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    auto go = [&](auto kernel) {
      hipExtLaunchKernelGGL(kernel, dim3(p->parts), dim3(BLOCK ? r.threads : kT), 0, s, e0, e1, 0, a, p->d, r.threads,
                            sums);
    };
    if (r.each == 1) go(k_rows_bwd<T, 1, false>);
    else if (r.each == 2) go(k_rows_bwd<T, 2, BLOCK>);
    else if (BLOCK) go(k_rows_bwd<float, 4, true>);
    else go(k_rows_bwd<T, 4, false>);
  });
}

template <typename T>
bl_status_t forward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  if (!p->fwd_split) return p->fwd.block ? launch_fwd<T, true>(p, a, s) : launch_fwd<T, false>(p, a, s);
  const dim3 grid((unsigned)(p->pieces / kBlockWaves * p->d.outer));
  const Split c{p->piece, p->pieces};
  const double bytes = (double)p->d.outer * p->d.size * sizeof(T);
  const bl_status_t st = timed_launch("norm_stats", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL(k_split_stats<T>, grid, dim3(kT), 0, s, e0, e1, 0, a, p->d, c);
  });
  if (st != BL_OK) return st;
  const long tile = (long)kT * (16 / (long)sizeof(T)) * kFwdVecs, tiles = (p->d.size + tile - 1) / tile;
  // about the blocks that are on the GPU together, with as many rows each as the others
  const long most = std::min<long>(p->d.outer, std::max<long>(1, kSplitBlocks / tiles));
  const long each = (p->d.outer + most - 1) / most;
  const int groups = (int)((p->d.outer + each - 1) / each);
  return timed_launch("norm_fwd", 2 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL(k_split_fwd<T>, dim3((unsigned)(tiles * groups)), dim3(kT), 0, s, e0, e1, 0, a, p->d, c,
                          (unsigned)tiles, groups);
  });
}

template <typename T>
bl_status_t backward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  const bool sums = a.dw || a.db;
  bl_status_t st;
  if (!p->bwd_split) {
    st = p->bwd.block ? launch_bwd<T, true>(p, a, sums, s) : launch_bwd<T, false>(p, a, sums, s);
  } else {
    const unsigned chunks = p->pieces / kBlockWaves;
    const Split c{p->piece, p->pieces};
    const double bytes = (double)p->d.outer * p->d.size * sizeof(T);
    st = timed_launch("norm_sums", 2 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      hipExtLaunchKernelGGL(k_split_sums<T>, dim3((unsigned)(chunks * p->d.outer)), dim3(kT), 0, s, e0, e1, 0, a, p->d,
                            c);
    });
    if (st != BL_OK) return st;
    st = timed_launch("norm_bwd", 3 * bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      hipExtLaunchKernelGGL(k_split_bwd<T>, dim3(chunks * p->row_groups), dim3(kT), 0, s, e0, e1, 0, a, p->d, c,
                            p->row_groups, sums);
    });
  }
  return st == BL_OK && sums ? norm_sum_parts(p, a, p->parts, s) : st;
}

}  // namespace

bl_status_t norm_rows_plan(bl_norm_plan_s* p) {
  const long rows = p->d.outer, M = p->d.size, V = 16 / dtype_bytes(p->d.dtype), nv = (M + V - 1) / V;
  // more would not fit the registers of a block of 1024 (with x, in fp32: w and b, or
  // backward dy, w and two sums)
  p->fwd = rows_shape(nv, p->d.dtype == BL_F32 ? 8 : 4, false);
  p->bwd = rows_shape(nv, p->d.dtype == BL_F32 ? 4 : 2, true);
  p->fwd_split = !p->fwd.threads;
  p->bwd_split = !p->bwd.threads;
  if (p->fwd_split || p->bwd_split) {
    const long tile = (long)kT * V * kTileVecs;
    long chunks = std::min<long>(kMostChunks, (M + tile - 1) / tile);
    const long chunk = ((M + chunks - 1) / chunks + tile - 1) / tile * tile;
    chunks = (M + chunk - 1) / chunk;
    if (rows * chunks >= kMostBlocks) return BL_ERR_UNSUPPORTED;
    p->piece = chunk / kBlockWaves;
    p->pieces = (int)chunks * kBlockWaves;
    p->off_sums = 0;
    p->bytes = round_up((size_t)rows * p->pieces * 2 * sizeof(float), 256);
  }
  p->off_part = p->bytes;
  if (p->bwd_split) {
    p->row_groups = (int)std::min<long>(rows, std::max<long>(1, kTargetBlocks / (p->pieces / kBlockWaves)));
    p->parts = p->row_groups;
  } else {
    // as many blocks as run at a time, each with a row of partial sums (half of them /
    // these / twice, with the last sum: 16384 rows of 2048 bfloat16 values 49 + 4 / 43 +
    // 4 / 47 + 6.5 us, of 1024 fp32 43 + 4 / 38 + 4 / 42 + 6.6; on blocks of 1024 2000
    // of 16384 113 + 4 / 92 + 6 / 103 + 11)
    const long each = p->bwd.block ? 1 : kT / p->bwd.threads;
    p->parts = (int)std::min<long>((rows + each - 1) / each, p->bwd.block && p->bwd.threads > 512 ? kTargetBlocks / 2 : kTargetBlocks);
  }
  p->bytes += (size_t)p->parts * 2 * M * sizeof(float);
  return BL_OK;
}

bl_status_t norm_rows_forward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  if (p->d.dtype == BL_F32) return forward<float>(p, a, s);
  if (p->d.dtype == BL_BF16) return forward<bf16_t>(p, a, s);
  return forward<f16_t>(p, a, s);
}

bl_status_t norm_rows_backward(const bl_norm_plan_s* p, const NormPtrs& a, hipStream_t s) {
  if (p->d.dtype == BL_F32) return backward<float>(p, a, s);
  if (p->d.dtype == BL_BF16) return backward<bf16_t>(p, a, s);
  return backward<f16_t>(p, a, s);
}

}  // namespace blc
