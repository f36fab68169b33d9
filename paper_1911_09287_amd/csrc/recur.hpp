// Gated linear recurrence: plan, launch arguments and the device code that both
// directions share (recur.hip: plan, dispatch and forward; recur_bwd.hip: backward).
#pragma once

#include "ops.hpp"

struct bl_recurrence_plan_s {
  bl_recurrence_desc_t d;
  int layout;       // RecurLayout
  int waves[2];     // of a block, forward and backward
  long every;       // steps between two saved states, a multiple of both directions' thread's steps
  long chunk[2];    // steps that a block takes, forward and backward (>= length: all)
  long chunks[2];   // of them
  size_t bytes;
};

namespace blc {

// How threads lie on [length][inner].  Wide: 16 lanes of channels, 8 bytes of them on
// each, so that a step's channels are read as lines of 128 bytes; the wave's four
// groups of lanes and the block's waves lie along steps.  Narrow: four lanes of one
// channel each.  Row (inner = 1, steps side by side): every lane along steps.
enum RecurLayout { kWide, kNarrow, kRow };

struct RecurArgs {
  const void *gate, *x, *dy;
  const unsigned char* resets;
  const float *h0, *dlast;
  void *y, *dgate, *dx;
  float *last, *states, *dh0;
  long outer, length, inner;
  long in_outer, in_step, out_outer, out_step;
  long every, chunk;
  float *part_a, *part_b;    // chunks: [1 + chunk][outer][inner] products and sums, entry 0 the state from outside
  unsigned char* part_drop;  // [1 + chunk][outer]: the state from outside does not reach the chunk's end
};

// What a stretch of steps does to the state: h -> drop ? b : a h + b.  (A dropped state
// is not multiplied by 0, so that NaN and infinity end there.)
template <int N>
struct Stretch {
  float a[N], b[N];
  bool drop;
};
template <int N>
__device__ __forceinline__ Stretch<N> stretch_none() {
  Stretch<N> s;
#pragma unroll
  for (int j = 0; j < N; ++j) s.a[j] = 1.f, s.b[j] = 0.f;
  s.drop = false;
  return s;
}
// first and then `second`, as one (in place of second).
template <int N, bool RESETS>
__device__ __forceinline__ void stretch_join(const Stretch<N>& first, Stretch<N>& second) {
  if (RESETS && second.drop) return;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    second.b[j] = fmaf(second.a[j], first.b[j], second.b[j]);
    second.a[j] *= first.a[j];
  }
  if (RESETS) second.drop = first.drop;
}
template <int N, bool RESETS>
__device__ __forceinline__ void stretch_apply(const Stretch<N>& s, float (&h)[N]) {
#pragma unroll
  for (int j = 0; j < N; ++j) h[j] = RESETS && s.drop ? s.b[j] : fmaf(s.a[j], h[j], s.b[j]);
}

// a and 1 - a (exp: 1) of a gate.  sigmoid: exp of -|gate| does not overflow, and the
// smaller of the two keeps its relative precision.
template <int GATE>
__device__ __forceinline__ void gate_of(float g, float& a, float& rest) {
  if (GATE == BL_GATE_EXP) {
    a = expf(g);
    rest = 1.f;
  } else {
    const float e = expf(-fabsf(g)), big = 1.f / (1.f + e), small = e * big;
    a = g >= 0.f ? big : small;  // (a NaN: both are)
    rest = g >= 0.f ? small : big;
  }
}

// Lanes of channels, channels of a lane and steps of a thread.
template <typename T, int LAYOUT>
struct RecurShape {
  static constexpr int kLanes = LAYOUT == kWide ? 16 : LAYOUT == kNarrow ? 4 : 1;
  static constexpr int kVec = LAYOUT == kWide ? 8 / (int)sizeof(T) : 1;
  static constexpr int kSlices = kWave / kLanes;  // of a wave, along steps
};

// Where a thread stands: its sequence, channels and slice of the tile's steps.
template <typename T, int LAYOUT, int WAVES>
struct RecurPlace {
  using S = RecurShape<T, LAYOUT>;
  long o, i, n;  // n: its channels that there are (<= 0: none)
  int wave, lane, slice;
  __device__ __forceinline__ explicit RecurPlace(const RecurArgs& r) {
    const long tiles = (r.inner + S::kLanes * S::kVec - 1) / (S::kLanes * S::kVec);
    o = (long)blockIdx.x / tiles;
    wave = WAVES == 1 ? 0 : threadIdx.x / kWave;
    lane = threadIdx.x % kWave;
    slice = wave * S::kSlices + lane / S::kLanes;
    i = ((long)blockIdx.x % tiles * S::kLanes + lane % S::kLanes) * S::kVec;
    n = r.inner - i;
  }
};

// EACH steps of a thread as they lie in memory: steps apart (Wide, Narrow), or side by
// side (Row).
template <typename T, int LAYOUT, int EACH>
struct RecurRaw {
  static constexpr int kVec = RecurShape<T, LAYOUT>::kVec;
  Held<T, LAYOUT == kRow ? EACH : kVec> w[LAYOUT == kRow ? 1 : EACH];
  // from p, the thread's first step of `there`
  __device__ __forceinline__ void load(const T* p, long step, long there, long n) {
    if constexpr (LAYOUT == kRow) {
      w[0].load(p, there);
    } else {
#pragma unroll
      for (int k = 0; k < EACH; ++k) w[k].load(p + k * step, k < there ? n : 0);
    }
  }
  __device__ __forceinline__ void refresh() {
#pragma unroll
    for (int k = 0; k < (LAYOUT == kRow ? 1 : EACH); ++k) w[k].refresh();
  }
  __device__ __forceinline__ float at(int k, int j) const {
    if constexpr (LAYOUT == kRow) return w[0][k];
    else return w[k][j];
  }
};
template <typename T, int LAYOUT, int EACH>
struct RecurOut {
  static constexpr int kVec = RecurShape<T, LAYOUT>::kVec;
  Pack<T, LAYOUT == kRow ? EACH : kVec> w[LAYOUT == kRow ? 1 : EACH];
  __device__ __forceinline__ void set(int k, int j, float v) {
    if constexpr (LAYOUT == kRow) w[0].v[k] = (T)v;
    else w[k].v[j] = (T)v;
  }
  __device__ __forceinline__ void store(T* p, long step, long there, long n) const {
    if constexpr (LAYOUT == kRow) {
      store_part(p, there, w[0]);
    } else {
#pragma unroll
      for (int k = 0; k < EACH; ++k) store_part(p + k * step, k < there ? n : 0, w[k]);
    }
  }
};
// The reset bytes of a thread's steps, as bits.
template <int EACH, bool RESETS>
__device__ __forceinline__ unsigned reset_bits(const unsigned char* p, long there) {
  unsigned bits = 0;
  if (RESETS) {
#pragma unroll
    for (int k = 0; k < EACH; ++k)
      if (k < there && p[k]) bits |= 1u << k;
  }
  return bits;
}

// The stretches of all slices of a wave before (FORWARD) or behind a thread's own,
// joined; `all`: those of the whole wave, in every lane.
template <int N, int LANES, bool RESETS, bool FORWARD>
__device__ __forceinline__ Stretch<N> wave_others(Stretch<N> own, Stretch<N>& all) {
  const int lane = threadIdx.x % kWave, slice = lane / LANES;
  auto from = [&](const Stretch<N>& s, int at) {
    Stretch<N> r;
#pragma unroll
    for (int j = 0; j < N; ++j) r.a[j] = __shfl(s.a[j], at), r.b[j] = __shfl(s.b[j], at);
    r.drop = RESETS ? (bool)__shfl((int)s.drop, at) : false;
    return r;
  };
#pragma unroll
  for (int d = 1; d < kWave / LANES; d *= 2) {
    const bool there = FORWARD ? slice >= d : slice + d < kWave / LANES;
    const Stretch<N> o = from(own, (lane + (FORWARD ? -d : d) * LANES) & (kWave - 1));
    if (there) stretch_join<N, RESETS>(o, own);
  }
  all = from(own, (FORWARD ? kWave - LANES : 0) + lane % LANES);
  const Stretch<N> o = from(own, (lane + (FORWARD ? -LANES : LANES)) & (kWave - 1));
  return (FORWARD ? slice > 0 : slice + 1 < kWave / LANES) ? o : stretch_none<N>();
}

// State before a chunk from the parts: that from outside and the chunks between.
// Forward: chunks 0 ... c - 1; backward: from the last down to c + 1.
template <int N, bool RESETS>
__device__ __forceinline__ void state_at(const RecurArgs& r, long o, long i, long n, long first, long step, long count,
                                         float (&h)[N]) {
  const long sites = r.outer * r.inner, at = o * r.inner + i;
#pragma unroll
  for (int j = 0; j < N; ++j) h[j] = j < n ? r.part_b[at + j] : 0.f;
  for (long c = 0; c < count; ++c) {
    const long k = 1 + first + c * step;
    Stretch<N> s = stretch_none<N>();
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < n) s.a[j] = r.part_a[k * sites + at + j], s.b[j] = r.part_b[k * sites + at + j];
    s.drop = RESETS && r.part_drop[k * r.outer + o];
    stretch_apply<N, RESETS>(s, h);
  }
}

// What a chunk does to the state, to its part: every thread walks its own stretch of
// the chunk, which are then joined over the block.  The first chunk (backward: the
// last) also leaves the state from outside, so that a call may give back a state in its place.
template <int N, int LANES, int WAVES, bool RESETS, bool FORWARD, typename Place>
__device__ __forceinline__ void chunk_part(const RecurArgs& r, const Place& p, Stretch<N> own, long chunk,
                                           const float* outside, bool first) {
  __shared__ float sa[WAVES][LANES][N], sb[WAVES][LANES][N];
  __shared__ int sd[WAVES];
  Stretch<N> all;
  wave_others<N, LANES, RESETS, FORWARD>(own, all);
  if (p.lane < LANES) {
#pragma unroll
    for (int j = 0; j < N; ++j) sa[p.wave][p.lane][j] = all.a[j], sb[p.wave][p.lane][j] = all.b[j];
    if (p.lane == 0) sd[p.wave] = all.drop;
  }
  __syncthreads();
  if (p.slice) return;
  Stretch<N> got = stretch_none<N>();
  for (int w = 0; w < WAVES; ++w) {
    const int k = FORWARD ? w : WAVES - 1 - w;
    Stretch<N> s;
#pragma unroll
    for (int j = 0; j < N; ++j) s.a[j] = sa[k][p.lane][j], s.b[j] = sb[k][p.lane][j];
    s.drop = sd[k];
    stretch_join<N, RESETS>(got, s);
    got = s;
  }
  const long sites = r.outer * r.inner, at = p.o * r.inner + p.i;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (j < p.n) {
      r.part_a[(1 + chunk) * sites + at + j] = got.a[j];
      r.part_b[(1 + chunk) * sites + at + j] = got.b[j];
      if (first) r.part_b[at + j] = outside ? outside[at + j] : 0.f;
    }
  // (every block of a sequence finds the same)
  if (RESETS && p.i == 0) r.part_drop[(1 + chunk) * r.outer + p.o] = got.drop;
}

// go(gate, layout, waves, resets) as constants.
template <typename Go>
void recur_dispatch(int gate, int layout, int waves, bool resets, Go&& go) {
  auto with = [&](auto g, auto l, auto w) {
    if (resets) go(g, l, w, std::true_type());
    else go(g, l, w, std::false_type());
  };
  auto in = [&](auto g) {
    using std::integral_constant;
    if (layout == kNarrow) with(g, integral_constant<int, kNarrow>(), integral_constant<int, 8>());
    else if (layout == kRow && waves == 1) with(g, integral_constant<int, kRow>(), integral_constant<int, 1>());
    else if (layout == kRow) with(g, integral_constant<int, kRow>(), integral_constant<int, 8>());
    else if (waves == 1) with(g, integral_constant<int, kWide>(), integral_constant<int, 1>());
    else with(g, integral_constant<int, kWide>(), integral_constant<int, 8>());
  };
  if (gate == BL_GATE_EXP) in(std::integral_constant<int, BL_GATE_EXP>());
  else in(std::integral_constant<int, BL_GATE_SIGMOID>());
}

// Steps of a thread in a tile: enough loads in flight, in the registers there are.
template <typename T, int LAYOUT, bool BACKWARD>
constexpr int recur_each() {
  if (LAYOUT == kRow) return 16 / (int)sizeof(T);
  return BACKWARD ? 4 : 8;
}

bl_status_t recur_backward(const bl_recurrence_plan_s* p, const RecurArgs& r, hipStream_t s);

}  // namespace blc
