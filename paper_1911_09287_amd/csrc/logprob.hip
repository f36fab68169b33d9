// Log probabilities of given classes, entropies and likeliest classes of rows of
// logits, and the gradient of the logits.
//
// Forward: a row of up to 2048 classes lies in the registers of a wave, a longer one
// is cut in pieces of up to 8 vectors a lane (8192 fp32, 16384 16-bit logits), each in
// the registers of a block; the logits are read once.  A lane takes its own largest
// logit m and sums a = sum e^(z - m) and b = sum e^(z - m) (z - m); two such triples
// over sets of classes join to one (m' = max, a' = a e^(m - m'), b' = e^(m - m') (b +
// (m - m') a), added), over lanes, waves and pieces, in an order that sizes alone
// decide.  log q_t = z_t - m - log a and the entropy log a - b / a come from the row's.
// Bound by HBM, in 16 bits nearly by the vector instructions (11 a logit).
//
// The `top` likeliest: a value and its class make one key of 64 bits whose order is
// the wanted one.  Of the largest values on each lane, every wave of a block takes the
// ceil(top / waves)-th; at least `top` values are no less than the least of these, so
// that it bounds the answer from below and few values are left.  (The top-th over all
// of a block's lanes is nearer by 1 to 3 % of the time at 20 and costs twice the time
// at 64, where most lanes hold one.)  What is left goes to LDS and one wave sorts it,
// 64 keys on its lanes, by a bitonic network.  Where more are left than there is room for
// (many equal values), or the row holds NaN, the waves take 64 keys after another and
// join them to a sorted list.  Pieces leave their `top` keys for a second launch that
// joins them.
//
// Measured: 4096 rows of 32000 logits without likeliest classes fp32 88 us, 6.0 TB/s,
// bfloat16 50 us, 5.2 TB/s, with 8 of them 68 us; 513 rows of 50021 fp32 logits with
// 20 of them 26 us, 4.0 TB/s, and 5.7 us for the join; one row of 131071 bfloat16
// logits with 8 of them 5.6 + 5.6 us, hardly more than two launches take anyhow.  Rows
// with hardly any class left (the others at minus infinity) leave lanes without one, the
// bound falls to minus infinity and 64 keys after another are taken: 513 rows of 50021 with
// 300 left 46 us, with 16 56; 4096 of 32000 bfloat16 with 16 left 221.  Rows of 1025 to 2048
// fp32 logits with likeliest classes are short of five registers a lane (3.8 TB/s).
#include <algorithm>
#include <new>

#include "ops.hpp"

struct bl_logprob_plan_s {
  bl_logprob_desc_t d;
  int each;          // vectors of 16 bytes of a lane: 1, 2, 4 or 8
  bool block;        // a piece by a block (else a row by a wave)
  int pieces;        // of a row
  long piece;        // classes of one
  size_t off_sums, bytes;  // workspace: keys of the pieces, then their (m, a, b)
};

namespace blc {
namespace {

constexpr int kT = 256;
constexpr int kWaves = kT / kWave;
constexpr int kRoom = 512;  // keys that are left after the bound, for which LDS has room
constexpr float kLog2e = 1.44269504f, kLn2 = 0.69314718f;
// Lanes whose largest logit is no further from zero take the exponent by one fused
// multiply-add: what the rounding of 1.5 * 2^20 leaves is 2^-4 at most.  Further out it
// grows with the logit (128 at 4e9, where 2^r overflows): there z - base comes first.
constexpr float kMostFused = 1048576.f;
using u64 = unsigned long long;

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// ---- keys -----------------------------------------------------------------------
// A value as a number of the same order: -0 as 0, NaN above all others.
__device__ __forceinline__ unsigned order_of(float z) {
  const unsigned u = __float_as_uint(z + 0.f);
  return z != z ? 0xFFFFFFFFu : u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(unsigned o) {
  return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xFFFFFFFFu));  // (all ones is a NaN)
}
// Larger values first, then lower classes.  No key is 0.
__device__ __forceinline__ u64 key_of(float z, unsigned j) { return (u64)order_of(z) << 32 | (0xFFFFFFFFu - j); }

// x of the lane whose number differs in bit J.
template <int J>
__device__ __forceinline__ unsigned lane_xor(unsigned x) {
  if constexpr (J == 1) return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, false);
  if constexpr (J == 2) return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, false);
  if constexpr (J == 4) {  // reversed within eights, then within fours
    const int r = __builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, false);
    return (unsigned)__builtin_amdgcn_update_dpp(0, r, 0x1B, 0xF, 0xF, false);
  }
  if constexpr (J == 8) return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, false);
  if constexpr (J == 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    return threadIdx.x & 16 ? r[0] : r[1];
  }
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return threadIdx.x & 32 ? r[0] : r[1];
}
template <int J>
__device__ __forceinline__ u64 lane_xor(u64 x) {
  return (u64)lane_xor<J>((unsigned)(x >> 32)) << 32 | lane_xor<J>((unsigned)x);
}
// One step of a bitonic network: lanes that differ in bit J exchange.  Stretches of
// K lanes fall and rise in turn (K = 64: all fall); where they fall the larger goes
// to the lower lane.  The lanes that keep the larger are known beforehand.
constexpr u64 larger_lanes(int J, int K) {
  u64 m = 0;
  for (int l = 0; l < kWave; ++l)
    if (((l & J) == 0) == (K == kWave || (l & K) == 0)) m |= 1ull << l;
  return m;
}
template <int J, int K>
__device__ __forceinline__ unsigned exchange(unsigned x) {
  const unsigned y = lane_xor<J>(x);
  return __builtin_amdgcn_inverse_ballot_w64(larger_lanes(J, K)) ? max(x, y) : min(x, y);
}
template <int J, int K>
__device__ __forceinline__ u64 exchange(u64 x) {
  const u64 y = lane_xor<J>(x);
  return __builtin_amdgcn_inverse_ballot_w64(larger_lanes(J, K) ^ __ballot(y < x)) ? y : x;
}
// Steps J, J / 2, ... 1.
template <int J, int K, typename X>
__device__ __forceinline__ X merge_stretches(X x) {
  x = exchange<J, K>(x);
  if constexpr (J > 1) x = merge_stretches<J / 2, K>(x);
  return x;
}
// Falling order over the wave of values that rise and then fall (or the reverse).
template <typename X>
__device__ __forceinline__ X merge64(X x) {
  return merge_stretches<32, 64>(x);
}
// Falling order over the wave.
template <typename X>
__device__ __forceinline__ X sort64(X x) {
  x = merge_stretches<1, 2>(x);
  x = merge_stretches<2, 4>(x);
  x = merge_stretches<4, 8>(x);
  x = merge_stretches<8, 16>(x);
  x = merge_stretches<16, 32>(x);
  return merge64(x);
}
// The 64 largest of two lists in falling order, in falling order.
__device__ __forceinline__ u64 join64(u64 a, u64 b) {
  b = lane_xor<1>(lane_xor<2>(lane_xor<4>(lane_xor<8>(lane_xor<16>(lane_xor<32>(b))))));  // reversed
  return merge64(a > b ? a : b);
}
__device__ __forceinline__ u64 lane_value(u64 x, int lane) {
  return (u64)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 |
         (unsigned)__builtin_amdgcn_readlane((int)(unsigned)x, lane);
}
// Joins 64 keys in any order (0: none) to a list whose top-th is `last`.
__device__ __forceinline__ void take64(u64 x, int top, u64& list, u64& last) {
  if (!__ballot(x > last)) return;
  x = sort64(x);
  list = lane_value(list, 0) ? join64(list, x) : x;
  last = lane_value(list, top - 1);
}

// ---- softmax statistics -----------------------------------------------------------
// Largest value m, a = sum 2^t and b = sum 2^t t with t = (z - m) log2 e.
struct Sums {
  float m, a, b;
};
// The same sums relative to m2 >= m.
__device__ __forceinline__ Sums rebased(Sums s, float m2) {
  if (s.m == m2) return s;
  // (bounded: of values that far below 2^t is 0, and 0 times infinity is not)
  const float t = fmaxf((s.m - m2) * kLog2e, -1000.f), f = exp2_(t);
  return Sums{m2, s.a * f, f * fmaf(t, s.a, s.b)};
}
__device__ __forceinline__ Sums over_wave(Sums s) {
  s = rebased(s, wave_max(s.m));
  return Sums{s.m, wave_sum(s.a), wave_sum(s.b)};
}
__device__ __forceinline__ Sums joined(Sums p, Sums q) {
  const float m = fmaxf(p.m, q.m);
  p = rebased(p, m);
  q = rebased(q, m);
  return Sums{m, p.a + q.a, p.b + q.b};
}

// What a row's results follow from.
struct Row {
  float base, log_sum;  // log q_j = z_j - base - log_sum
  bool none;            // every class is ruled out
  __device__ Row(const Sums& s) {
    none = s.m == -INFINITY && s.a == 0.f;  // (a is NaN where there is a NaN)
    base = s.m == -INFINITY ? 0.f : s.m;
    log_sum = logf(s.a);
  }
};

struct Ptrs {
  const void* logits;
  const long long* targets;
  float *logp, *stats, *top_logp;
  long long* top_index;
  u64* keys;    // [row][piece][top]
  float* sums;  // [row][piece][3]
};

// One lane writes a row's logp and stats.
template <typename T>
__device__ __forceinline__ void write_row(const Ptrs& a, const bl_logprob_desc_t& d, long row, const Sums& s,
                                          const Row& r) {
  const long long t = a.targets ? a.targets[row] : -1;
  if (a.logp) {
    float x = 0.f;
    if (t >= 0 && t < d.classes)
      x = r.none ? -INFINITY : to_f32(static_cast<const T*>(a.logits)[row * d.stride + t]) - r.base - r.log_sum;
    a.logp[row] = x;
  }
  if (a.stats) {
    a.stats[row] = s.m;
    a.stats[d.rows + row] = r.log_sum;
    a.stats[2 * d.rows + row] = r.none ? 0.f : r.log_sum - s.b * kLn2 / s.a;
  }
}
// A wave writes a row's likeliest classes from its list.
__device__ __forceinline__ void write_top(const Ptrs& a, const bl_logprob_desc_t& d, long row, const Row& r, u64 list) {
  const int i = threadIdx.x % kWave;
  if (i >= d.top) return;
  const long at = row * d.top + i;
  a.top_index[at] = list ? (long long)(0xFFFFFFFFu - (unsigned)list) : -1;
  a.top_logp[at] = !list || r.none ? -INFINITY : value_of((unsigned)(list >> 32)) - r.base - r.log_sum;
}

template <typename T>
constexpr unsigned kMinusInf = sizeof(T) == 4 ? 0xFF800000u : std::is_same_v<T, bf16_t> ? 0xFF80FF80u : 0xFC00FC00u;

template <int WAVES>
__device__ __forceinline__ void part_sync() {  // over the waves that work on one piece
  if (WAVES == 1) wave_sync();
  else __syncthreads();
}

// Adds 2^t and 2^t t of all values to a lane's sums.
template <typename T, int V, int E, typename Exponent>
__device__ __forceinline__ void add_terms(Held<T, V> (&v)[E], Sums& s, Exponent&& exponent) {
#pragma unroll
  for (int k = 0; k < E; ++k) {
    v[k].refresh();
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float t = exponent(v[k][j]), e = exp2_(t);
      s.a += e;
      s.b = fmaf(e, fmaxf(t, -1000.f), s.b);  // (t = -infinity: e is 0)
    }
  }
}

// Pieces of rows (WAVES = 1: whole rows), E vectors a lane.  With `pieces` > 1 each
// leaves its sums and keys, else it gives the row's results.
template <typename T, int E, int WAVES, bool TOP>
__global__ __launch_bounds__(kT, TOP ? 6 : 8) void k_logprob_fwd(Ptrs a, bl_logprob_desc_t d, int pieces, long piece) {
  constexpr int V = 16 / sizeof(T), kParts = kWaves / WAVES;  // pieces of a block at a time
  __shared__ u64 room[kParts][TOP ? kRoom : 1];
  __shared__ unsigned bounds[WAVES];
  __shared__ int left[kParts];
  __shared__ Sums wave_sums[WAVES];
  const int part = WAVES == 1 ? threadIdx.x / kWave : 0, in = WAVES == 1 ? threadIdx.x % kWave : threadIdx.x;
  const int lane = threadIdx.x % kWave, wave = in / kWave;
  const unsigned long long count = (unsigned long long)d.rows * pieces;
  const unsigned long long stride = (unsigned long long)gridDim.x * kParts;
  for (unsigned long long q = (unsigned long long)blockIdx.x * kParts + part; q < count; q += stride) {
    const long row = pieces == 1 ? (long)q : (long)(q / (unsigned)pieces);
    const long from = pieces == 1 ? 0 : (long)(q % (unsigned)pieces) * piece;
    const int len = (int)min(piece, (long)d.classes - from);
    const T* z = static_cast<const T*>(a.logits) + row * d.stride + from;
    Held<T, V> v[E];
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const int i = (in + k * WAVES * kWave) * V;
      v[k].load(z + i, len - i, kMinusInf<T>);
    }
    Sums s{-INFINITY, 0.f, 0.f};
    float most[E];  // of each vector
#pragma unroll
    for (int k = 0; k < E; ++k) {
      v[k].refresh();
      most[k] = v[k][0];
#pragma unroll
      for (int j = 1; j < V; ++j) most[k] = fmaxf(most[k], v[k][j]);
      s.m = fmaxf(s.m, most[k]);
    }
    unsigned bound = 0;
    if (TOP) {
      bound = (unsigned)__builtin_amdgcn_readlane((int)sort64(order_of(s.m)), (d.top + WAVES - 1) / WAVES - 1);
      if (WAVES > 1 && lane == 0) bounds[wave] = bound;
      if (in == 0) left[part] = 0;
    }
    const float base = s.m == -INFINITY ? 0.f : s.m;
    if (!__ballot(fabsf(base) > kMostFused)) {
      // t = z log2 e + c with c rounded once: all terms are 2^r too large, r what the
      // rounding left, which is taken out of the sums
      const float c = -(base * kLog2e), left_over = fmaf(base, kLog2e, c), f = exp2_(-left_over);
      add_terms<T, V, E>(v, s, [&](float z) { return fmaf(z, kLog2e, c); });
      s.b = fmaf(-left_over, s.a, s.b) * f;
      s.a *= f;
    } else {
      add_terms<T, V, E>(v, s, [&](float z) { return (z - base) * kLog2e; });
    }
    if (!(s.a < INFINITY)) s.a = NAN;  // (infinite only beside an infinite logit)
    s = over_wave(s);
    if (WAVES > 1 && lane == 0) wave_sums[wave] = s;
    part_sync<WAVES>();
    if (WAVES > 1) {
      s = wave_sums[0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) s = joined(s, wave_sums[w]);
    }
    const Row r(s);
    u64 list = 0, last = 0;
    if (TOP) {
#pragma unroll
      for (int w = 0; w < (WAVES > 1 ? WAVES : 0); ++w) bound = min(bound, bounds[w]);
      const float least = value_of(bound);
      bool whole = s.a == s.a;  // no NaN
      if (whole) {
        // each lane's vectors that hold such a value (mostly none, seldom two), read again
        unsigned hits = 0;
#pragma unroll
        for (int k = 0; k < E; ++k) hits |= most[k] >= least ? 1u << k : 0u;
        while (__ballot(hits != 0)) {
          const int i = hits ? (in + __builtin_ctz(hits) * WAVES * kWave) * V : len;
          hits &= hits - 1;
          Held<T, V> u;
          u.load(z + i, len - i, kMinusInf<T>);
          u.refresh();
          u64 pass[V];
          int n = 0;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            pass[j] = __ballot(u[j] >= least && i + j < len);
            n += __popcll(pass[j]);
          }
          int at = 0;
          if (lane == 0) at = atomicAdd(&left[part], n);
          at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const int to = at + __builtin_amdgcn_mbcnt_hi((unsigned)(pass[j] >> 32),
                                                          __builtin_amdgcn_mbcnt_lo((unsigned)pass[j], 0));
            if ((pass[j] >> lane & 1) && to < kRoom) room[part][to] = key_of(u[j], (unsigned)(from + i + j));
            at += __popcll(pass[j]);
          }
        }
      }
      part_sync<WAVES>();
      const int n = left[part];
      whole = whole && n <= kRoom;
      if (whole) {
        if (wave == 0)
          for (int i = lane; i - lane < n; i += kWave) take64(i < n ? room[part][i] : 0, d.top, list, last);
      } else {  // 64 by 64, the waves in turn; then their lists
        for (int i = in; i - lane < len; i += 4 * WAVES * kWave) {
          float zi[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) zi[u] = i + u * WAVES * kWave < len ? to_f32(z[i + u * WAVES * kWave]) : 0.f;
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int iu = i + u * WAVES * kWave;
            take64(iu < len ? key_of(zi[u], (unsigned)(from + iu)) : 0, d.top, list, last);
          }
        }
        if (WAVES > 1) {
          __syncthreads();  // `left` has been read
          room[0][in] = list;
          __syncthreads();
          if (wave == 0)
#pragma unroll
            for (int w = 1; w < WAVES; ++w) list = join64(list, room[0][w * kWave + lane]);
        }
      }
    }
    if (wave == 0) {
      if (pieces == 1) {
        if (lane == 0) write_row<T>(a, d, row, s, r);
        if (TOP) write_top(a, d, row, r, list);
      } else {
        if (lane < 3) a.sums[q * 3 + lane] = lane == 0 ? s.m : lane == 1 ? s.a : s.b;
        if (TOP && lane < d.top) a.keys[q * d.top + lane] = list;
      }
    }
    if (q + stride < count) part_sync<WAVES>();  // before LDS is written again
  }
}

// Rows of pieces: a block, or a wave where there are few keys, joins a row's sums
// and keys.
template <typename T, int WAVES, bool TOP>
__global__ __launch_bounds__(kT) void k_logprob_join(Ptrs a, bl_logprob_desc_t d, int pieces) {
  constexpr int kRows = kWaves / WAVES, threads = WAVES * kWave;
  __shared__ u64 lists[WAVES > 1 && TOP ? kT : 1];
  __shared__ Sums wave_sums[WAVES];
  const int lane = threadIdx.x % kWave, in = threadIdx.x % threads, wave = in / kWave;
  for (long row = (long)blockIdx.x * kRows + threadIdx.x / threads; row < d.rows; row += (long)gridDim.x * kRows) {
    const float* sums = a.sums + (size_t)row * pieces * 3;
    Sums s{-INFINITY, 0.f, 0.f};
    for (int p = in; p < pieces; p += threads) s = joined(s, Sums{sums[3 * p], sums[3 * p + 1], sums[3 * p + 2]});
    s = over_wave(s);
    u64 list = 0, last = 0;
    if (TOP) {
      const u64* keys = a.keys + (size_t)row * pieces * d.top;
      const long n = (long)pieces * d.top;
      for (long i = in; i - lane < n; i += threads) take64(i < n ? keys[i] : 0, d.top, list, last);
    }
    if (WAVES > 1) {
      if (lane == 0) wave_sums[wave] = s;
      if (TOP) lists[in] = list;
      __syncthreads();
      s = wave_sums[0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) s = joined(s, wave_sums[w]);
    }
    const Row r(s);
    if (in == 0) write_row<T>(a, d, row, s, r);
    if (TOP && wave == 0) {
#pragma unroll
      for (int w = 1; w < WAVES; ++w) list = join64(list, lists[w * kWave + lane]);
      write_top(a, d, row, r, list);
    }
    if (WAVES > 1) __syncthreads();
  }
}

// Gradient: E vectors of a piece a lane (WAVES = 1: a row by a wave), read and
// written once.  Bound by HBM: 4096 rows of 65536 bfloat16 logits 212 us, 5.1 TB/s, with
// the entropy's gradient 213.
struct GradPtrs {
  const void* logits;
  const long long* targets;
  const float *stats, *g_logp, *g_entropy;
  void* dlogits;
};
template <typename T, int E, int WAVES, bool ENTROPY>
__global__ __launch_bounds__(kT) void k_logprob_bwd(GradPtrs a, bl_logprob_desc_t d, int pieces, long piece) {
  constexpr int V = 16 / sizeof(T), kParts = kWaves / WAVES;
  const int part = WAVES == 1 ? threadIdx.x / kWave : 0, in = WAVES == 1 ? threadIdx.x % kWave : threadIdx.x;
  const unsigned long long count = (unsigned long long)d.rows * pieces;
  for (unsigned long long q = (unsigned long long)blockIdx.x * kParts + part; q < count;
       q += (unsigned long long)gridDim.x * kParts) {
    const long row = pieces == 1 ? (long)q : (long)(q / (unsigned)pieces);
    const long from = pieces == 1 ? 0 : (long)(q % (unsigned)pieces) * piece;
    const int len = (int)min(piece, (long)d.classes - from);
    const T* z = static_cast<const T*>(a.logits) + row * d.stride + from;
    T* dz = static_cast<T*>(a.dlogits) + row * d.grad_stride + from;
    Held<T, V> v[E];
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const int i = (in + k * WAVES * kWave) * V;
      v[k].load(z + i, len - i);
    }
    const float m = a.stats[row], log_sum = a.stats[d.rows + row];
    const float entropy = ENTROPY ? a.stats[2 * d.rows + row] : 0.f, ge = ENTROPY ? a.g_entropy[row] : 0.f;
    const long long t = a.targets ? a.targets[row] : -1;
    const float g = a.g_logp && t >= 0 && t < d.classes ? a.g_logp[row] : 0.f;
    const bool none = m == -INFINITY && log_sum == -INFINITY;
    const int at = t >= from && t < from + len ? (int)(t - from) : -1;  // the target in this piece
#pragma unroll
    for (int k = 0; k < E; ++k) {
      const int i = (in + k * WAVES * kWave) * V;
      v[k].refresh();
      Pack<T, V> o;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float lq = v[k][j] - m - log_sum, p = exp2_(lq * kLog2e);
        float x = i + j == at ? g - g * p : -(g * p);
        if (ENTROPY) x -= ge * p * fmaxf(lq + entropy, -1000.f);  // (a class ruled out: p is 0)
        o.v[j] = (T)(none ? 0.f : x);
      }
      store_part<T, V>(dz + i, len - i, o);
    }
  }
}

}  // namespace
}  // namespace blc

using namespace blc;

namespace {
// Rows up to so many classes lie on one wave.  8192 rows, wave / block, forward with 8
// likeliest classes and without, backward: 1100 fp32 16.5 / 31, 9.4 / 14.7, 15.5 / 14.0
// us; 2048 18.6 / 32, 12.5 / 14.8, 28 / 28; 2048 bfloat16 18.2 / 35, 9.0 / 14, 15.9 /
// 13.4; 4096 fp32 105 / 40 (registers), 105 / 24, 56 / 48.  4096 bfloat16 take 23 us on a
// wave and 40 on a block, but 64 rows of 2048 6.6 and 5.5.
constexpr long kWaveClasses = 2048;
constexpr long kPieceVectors = 8 * kT; // and pieces of longer ones on a block, 8 vectors a lane
constexpr unsigned kGrid = 1u << 20;  // blocks of a launch, which go on with what is left

// Vectors of a lane, of those that kernels are compiled for, for `n` classes on `threads` lanes.
int vectors_of(long n, int threads, int wide) {
  const long per = (long)threads * (16 / wide);
  int each = 1;
  while (each * per < n) each *= 2;
  return each;
}

// go(the vectors of a lane as a constant), of those that calls reach: powers of two from LEAST to MOST.
template <int LEAST, int MOST, typename Go>
void with_vectors(int each, Go&& go) {
  if constexpr (LEAST < MOST)
    if (each > LEAST) return with_vectors<2 * LEAST, MOST>(each, go);
  go(std::integral_constant<int, LEAST>());
}

template <typename T, int WAVES, bool TOP>
bl_status_t forward(const bl_logprob_plan_s* p, const Ptrs& a, hipStream_t s) {
  const bl_logprob_desc_t& d = p->d;
  const unsigned long long work = ((unsigned long long)d.rows * p->pieces + kWaves / WAVES - 1) / (kWaves / WAVES);
  const unsigned blocks = (unsigned)std::min<unsigned long long>(work, kGrid);
  const double bytes = (double)d.rows * d.classes * sizeof(T);
  bl_status_t st = timed_launch("logprob_fwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    auto go = [&](auto kernel) {
      hipExtLaunchKernelGGL(kernel, dim3(blocks), dim3(kT), 0, s, e0, e1, 0, a, d, p->pieces, p->piece);
    };
    // (a block's pieces have over 1024 classes; 2048 on a wave are four vectors of 16 bits)
    constexpr int kLeast = WAVES > 1 && sizeof(T) == 4 ? 2 : 1, kMost = WAVES == 1 && sizeof(T) == 2 ? 4 : 8;
    with_vectors<kLeast, kMost>(p->each, [&](auto e) { go(k_logprob_fwd<T, decltype(e)::value, WAVES, TOP>); });
  });
  if (st != BL_OK || p->pieces == 1) return st;
  const double left = (double)d.rows * p->pieces * (12 + 8 * d.top);
  // (wave / block: 513 rows of 7 pieces with 8 classes 4.1 / 5.4 us, 16 5.2 / 5.4, 20 5.2 / 5.7,
  // 32 7.6 / 5.6; 4096 of 2 with 8 5.4 / 14.6; one of 64 with 8 10 / 5.5)
  const bool by_waves = p->pieces <= kWave && (long)p->pieces * d.top <= 2 * kWave;
  const long long join = by_waves ? (d.rows + kWaves - 1) / kWaves : d.rows;
  return timed_launch("logprob_join", left, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    auto go = [&](auto kernel) {
      hipExtLaunchKernelGGL(kernel, dim3((unsigned)std::min<long long>(join, kGrid)), dim3(kT), 0, s, e0, e1, 0, a, d,
                            p->pieces);
    };
    by_waves ? go(k_logprob_join<T, 1, TOP>) : go(k_logprob_join<T, kWaves, TOP>);
  });
}

template <typename T>
bl_status_t forward(const bl_logprob_plan_s* p, const Ptrs& a, hipStream_t s) {
  if (p->block) return p->d.top ? forward<T, kWaves, true>(p, a, s) : forward<T, kWaves, false>(p, a, s);
  return p->d.top ? forward<T, 1, true>(p, a, s) : forward<T, 1, false>(p, a, s);
}

template <typename T, int WAVES, bool ENTROPY>
bl_status_t backward(const bl_logprob_plan_s* p, const GradPtrs& a, hipStream_t s) {
  const bl_logprob_desc_t& d = p->d;
  const long most = 4L * kT * (16 / (long)sizeof(T));  // of a piece: four vectors a lane
  const int pieces = WAVES == 1 ? 1 : (int)((d.classes + most - 1) / most);
  const long piece = ((d.classes + pieces - 1) / pieces + 15) / 16 * 16;
  const int each = vectors_of(piece < d.classes ? piece : (long)d.classes, WAVES * kWave, (int)sizeof(T));
  const unsigned long long work = ((unsigned long long)d.rows * pieces + kWaves / WAVES - 1) / (kWaves / WAVES);
  const unsigned blocks = (unsigned)std::min<unsigned long long>(work, kGrid);
  return timed_launch("logprob_bwd", 2.0 * d.rows * d.classes * sizeof(T), 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    auto go = [&](auto kernel) {
      hipExtLaunchKernelGGL(kernel, dim3(blocks), dim3(kT), 0, s, e0, e1, 0, a, d, pieces, piece);
    };
    // (a block's pieces have over 2048 classes)
    constexpr int kLeast = WAVES == 1 ? 1 : sizeof(T) == 2 ? 2 : 4, kMost = WAVES == 1 && sizeof(T) == 4 ? 8 : 4;
    with_vectors<kLeast, kMost>(each, [&](auto e) { go(k_logprob_bwd<T, decltype(e)::value, WAVES, ENTROPY>); });
  });
}

template <typename T>
bl_status_t backward(const bl_logprob_plan_s* p, const GradPtrs& a, hipStream_t s) {
  if (p->d.classes > kWaveClasses) return a.g_entropy ? backward<T, kWaves, true>(p, a, s) : backward<T, kWaves, false>(p, a, s);
  return a.g_entropy ? backward<T, 1, true>(p, a, s) : backward<T, 1, false>(p, a, s);
}
}  // namespace

extern "C" bl_status_t bl_logprob_plan_create(bl_logprob_plan_t* out, const bl_logprob_desc_t* desc) {
  if (!out || !desc) return BL_ERR_INVALID_ARG;
  *out = nullptr;
  bl_logprob_desc_t d = *desc;
  if (d.rows < 0 || d.classes < 1 || d.top < 0 || !known_dtype(d.dtype)) return BL_ERR_INVALID_ARG;
  if (d.stride < 0 || d.grad_stride < 0) return BL_ERR_INVALID_ARG;
  if (!d.stride) d.stride = d.classes;
  if (!d.grad_stride) d.grad_stride = d.classes;
  if (d.rows > 1 && (d.stride < d.classes || d.grad_stride < d.classes)) return BL_ERR_INVALID_ARG;
  const long long limit = (1LL << 31) - 1;
  if (d.top > 64 || d.classes > limit || d.rows > limit) return BL_ERR_UNSUPPORTED;
  bl_logprob_plan_s* p = new (std::nothrow) bl_logprob_plan_s{};
  if (!p) return BL_ERR_OOM;
  p->d = d;
  p->block = d.classes > kWaveClasses;
  long most = kPieceVectors * (16 / dtype_bytes(d.dtype));
  // few rows in pieces anyway: smaller ones, until there is one for each compute unit (until
  // 128 / 256 / 512, and the join: 32 rows of 50021 fp32 logits with 20 classes 7.1 + 4.7 / 6.9
  // + 4.9 / 7.9 + 6.0 us; 4 of 131071 bfloat16 with 8 6.4 + 4.4 / 5.8 + 5.7 / 6.0 + 5.7)
  while (d.classes > kPieceVectors * (16 / dtype_bytes(d.dtype)) && most > kWaveClasses && d.rows * ((d.classes + most - 1) / most) < 256) most /= 2;
  p->pieces = p->block ? (int)((d.classes + most - 1) / most) : 1;
  p->piece = p->pieces == 1 ? (long)d.classes : ((d.classes + p->pieces - 1) / p->pieces + 15) / 16 * 16;
  p->each = vectors_of(p->piece, p->block ? kT : kWave, dtype_bytes(d.dtype));
  if (p->pieces > 1) {
    p->off_sums = (size_t)d.rows * p->pieces * d.top * sizeof(u64);
    p->bytes = p->off_sums + (size_t)d.rows * p->pieces * 3 * sizeof(float);
  }
  *out = p;
  return BL_OK;
}

extern "C" bl_status_t bl_logprob_plan_destroy(bl_logprob_plan_t p) {
  if (!p) return BL_ERR_INVALID_ARG;
  delete p;
  return BL_OK;
}

extern "C" bl_status_t bl_logprob_workspace_size(bl_logprob_plan_t p, size_t* bytes) {
  if (!p || !bytes) return BL_ERR_INVALID_ARG;
  *bytes = p->bytes;
  return BL_OK;
}

extern "C" bl_status_t bl_logprob_forward(bl_logprob_plan_t p, const void* logits, const long long* targets,
                                          float* logp, float* stats, float* top_logp, long long* top_index, void* ws,
                                          void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (!p->d.rows) return BL_OK;
  if (!logits || (p->d.top && (!top_logp || !top_index)) || (p->bytes && (!ws || !aligned(ws)))) return BL_ERR_INVALID_ARG;
  const Ptrs a{logits, targets, logp, stats, top_logp, top_index, static_cast<u64*>(ws),
               reinterpret_cast<float*>(static_cast<char*>(ws) + p->off_sums)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p->d.dtype == BL_F32) return forward<float>(p, a, s);
  if (p->d.dtype == BL_BF16) return forward<bf16_t>(p, a, s);
  return forward<f16_t>(p, a, s);
}

extern "C" bl_status_t bl_logprob_backward(bl_logprob_plan_t p, const void* logits, const long long* targets,
                                           const float* stats, const float* g_logp, const float* g_entropy,
                                           void* dlogits, void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (!p->d.rows) return BL_OK;
  if (!logits || !stats || !dlogits) return BL_ERR_INVALID_ARG;
  const GradPtrs a{logits, targets, stats, g_logp, g_entropy, dlogits};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (p->d.dtype == BL_F32) return backward<float>(p, a, s);
  if (p->d.dtype == BL_BF16) return backward<bf16_t>(p, a, s);
  return backward<f16_t>(p, a, s);
}
