// Gated linear recurrence: plan, launch arguments and the device code that both
// directions share (recur.hip: plan, dispatch and forward; recur_bwd.hip: backward).
#pragma once

#include "ops.hpp"

struct bl_recurrence_plan_s {
  bl_recurrence_desc_t d;
  int layout[2];    // RecurLayout, forward and backward, as all that follow
  int lanes[2];     // of channels that a block takes
  int waves[2];     // of a block
  long every;       // steps between two saved states, a multiple of both directions' thread's steps
  long chunk[2];    // steps that a block takes (>= length: all)
  long chunks[2];   // of them
  size_t bytes;
};

namespace blc {

// How threads lie on [length][inner].  Wide: 16 lanes of channels, 8 bytes of them on
// each, so that a step's channels are read as lines of 128 bytes; the wave's four
// groups of lanes and the block's waves lie along steps.  Half: the same with 4 bytes,
// for twice the blocks.  Narrow: four lanes of one channel each.  Row (inner = 1, steps
// side by side): every lane along steps.
enum RecurLayout { kWide, kHalf, kNarrow, kRow };

struct RecurArgs {
  const void *gate, *x, *dy;
  const unsigned char* resets;
  const float *h0, *dlast;
  void *y, *dgate, *dx;
  float *last, *states, *dh0;
  long outer, length, inner;
  long in_outer, in_step, out_outer, out_step;
  long every, chunk;  // every: a power of two
  int every_log2;
  bool near;          // a tile's bytes count in 32 bits
  int lanes;          // of channels that a block takes
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

// a and 1 - a (exp: 1) of a gate.
template <int GATE>
__device__ __forceinline__ void gate_of(float g, float& a, float& rest) {
  if (GATE == BL_GATE_EXP) {
    a = exp_of<true>(g);
    rest = 1.f;
  } else {
    float slope;
    logistic_of(g, a, rest, slope);
  }
}

// Channels of a lane.
constexpr int recur_vec(int layout, int wide) { return layout == kWide ? 8 / wide : layout == kHalf ? 4 / wide : 1; }
// Lanes of channels, channels of a lane and steps of a thread.
template <typename T, int LAYOUT>
struct RecurShape {
  static constexpr int kLanes = LAYOUT == kNarrow ? 4 : LAYOUT == kRow ? 1 : 16;
  static constexpr int kVec = recur_vec(LAYOUT, (int)sizeof(T));
  static constexpr int kSlices = kWave / kLanes;  // of a wave, along steps
};

// Where a thread stands: its sequence and chunk of it, first channel and slice of the tile's
// steps.  Lanes that would reach over the block's channels (which are a lane's at least, see
// recur_lanes) take its last ones, as another lane of their wave does too: both read the same
// before either writes, and write the same.
template <typename T, int LAYOUT, int WAVES>
struct RecurPlace {
  using S = RecurShape<T, LAYOUT>;
  long o, chunk, i;
  int wave, lane, slice;
  __device__ __forceinline__ explicit RecurPlace(const RecurArgs& r) {
    const long tiles = (r.inner + r.lanes * S::kVec - 1) / (r.lanes * S::kVec);
    // blocks go to the GPU's eight dies in turn, each with caches of its own: a die takes
    // neighbouring channels of a sequence's chunk
    const unsigned index = blockIdx.y * gridDim.x + blockIdx.x, all = gridDim.x * gridDim.y;
    const unsigned die = index % 8, at = die * (all / 8) + min(die, all % 8) + index / 8;
    const unsigned q = at / (unsigned)tiles;  // chunks of a sequence, then sequences
    o = q / gridDim.y;
    chunk = q - (unsigned)o * gridDim.y;
    const unsigned block = at - q * (unsigned)tiles;
    wave = WAVES == 1 ? 0 : threadIdx.x / kWave;
    lane = threadIdx.x % kWave;
    slice = wave * S::kSlices + lane / S::kLanes;
    i = min(((long)block * r.lanes + min(lane % S::kLanes, r.lanes - 1)) * S::kVec, r.inner - S::kVec);
  }
};

// EACH steps of a thread as they lie in memory: steps apart, or side by side (Row).  Those
// that are all there are read and written without a branch, so that loads that have been
// issued before can be told from those after and stay in flight, and at a thread's bytes
// `off` from the tile's and step's place, which the block shares: one address register.
template <typename T, int LAYOUT, int EACH>
struct RecurRaw {
  static constexpr int kVec = RecurShape<T, LAYOUT>::kVec;
  Held<T, LAYOUT == kRow ? EACH : kVec> w[LAYOUT == kRow ? 1 : EACH];
  __device__ __forceinline__ void load_all(const T* tile, long step, unsigned off) {
#pragma unroll
    for (int k = 0; k < (LAYOUT == kRow ? 1 : EACH); ++k) w[k].load_at(tile + k * step, off, true);
  }
  // from p, the thread's first step, the first `there`
  __device__ __forceinline__ void load(const T* p, long step, long there) {
    if constexpr (LAYOUT == kRow) {
      w[0].load(p, there);
    } else {
#pragma unroll
      for (int k = 0; k < EACH; ++k) w[k].load(p + k * step, k < there ? kVec : 0);
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
  __device__ __forceinline__ void store_all(T* tile, long step, unsigned off) const {
#pragma unroll
    for (int k = 0; k < (LAYOUT == kRow ? 1 : EACH); ++k) store_pack(at_bytes(tile + k * step, off), w[k]);
  }
  __device__ __forceinline__ void store(T* p, long step, long there) const {
    if constexpr (LAYOUT == kRow) {
      store_part(p, there, w[0]);
    } else {
#pragma unroll
      for (int k = 0; k < EACH; ++k)
        if (k < there) store_pack(p + k * step, w[k]);
    }
  }
};
// The reset bytes of a thread's steps, as they are loaded and as bits.
template <int EACH, bool RESETS>
struct RecurResets {
  unsigned w[RESETS ? (EACH + 3) / 4 : 1];
  template <bool FULL>
  __device__ __forceinline__ void load(const unsigned char* p, long there) {
    static_assert(EACH % 4 == 0 && EACH <= 32, "whole words, and a word of bits");
    if constexpr (RESETS) {
      if (FULL || there >= EACH) {
        __builtin_memcpy(w, p, EACH);
      } else {
#pragma unroll
        for (int k = 0; k < EACH / 4; ++k) w[k] = 0;
#pragma unroll
        for (int k = 0; k < EACH; ++k)
          if (k < there) w[k / 4] |= (unsigned)p[k] << (8 * (k % 4));
      }
    }
  }
  __device__ __forceinline__ unsigned bits() const {
    unsigned got = 0;
    if constexpr (RESETS) {
#pragma unroll
      for (int k = 0; k < EACH; ++k) got |= (w[k / 4] >> (8 * (k % 4)) & 0xFFu ? 1u : 0u) << k;
    }
    return got;
  }
};

// A barrier for what lies in LDS alone: loads from memory stay in flight (a __syncthreads()
// waits for them).
__device__ __forceinline__ void block_sync() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Lanes' stretches with those of other lanes, by a function of a 32-bit value.
template <int N, bool RESETS, typename Move>
__device__ __forceinline__ Stretch<N> stretch_moved(const Stretch<N>& s, Move&& move) {
  Stretch<N> r;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    r.a[j] = __uint_as_float(move(__float_as_uint(s.a[j]), __float_as_uint(1.f)));
    r.b[j] = __uint_as_float(move(__float_as_uint(s.b[j]), 0u));
  }
  r.drop = RESETS ? (bool)move((unsigned)s.drop, 0u) : false;
  return r;
}
// Of two lanes' stretches, the even (lower) one and the odd (upper) one, in both: of
// neighbouring rows of 16 lanes, or of the wave's halves.
template <int N, bool RESETS, bool HALVES>
__device__ __forceinline__ void stretch_pair(const Stretch<N>& s, Stretch<N>& even, Stretch<N>& odd) {
  auto swap = [](unsigned x) {
    return HALVES ? __builtin_amdgcn_permlane32_swap(x, x, false, false) : __builtin_amdgcn_permlane16_swap(x, x, false, false);
  };
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const auto a = swap(__float_as_uint(s.a[j])), b = swap(__float_as_uint(s.b[j]));
    even.a[j] = __uint_as_float(a[0]), odd.a[j] = __uint_as_float(a[1]);
    even.b[j] = __uint_as_float(b[0]), odd.b[j] = __uint_as_float(b[1]);
  }
  even.drop = odd.drop = false;
  if (RESETS) {
    const auto d = swap((unsigned)s.drop);
    even.drop = d[0], odd.drop = d[1];
  }
}

// The stretches of all slices of a wave before (FORWARD) or behind a thread's own,
// joined; `all`: those of the whole wave, in every lane.
template <int N, int LANES, bool RESETS, bool FORWARD>
__device__ __forceinline__ Stretch<N> wave_others(Stretch<N> own, Stretch<N>& all) {
  static_assert(LANES == 1 || LANES == 4 || LANES == 16, "rows of 16 lanes, and slices within them");
  const int lane = threadIdx.x % kWave;
  Stretch<N> others = stretch_none<N>();
  if constexpr (LANES < 16) {
    // within rows of 16 lanes: inclusive over 1, 2, ... lanes, then one slice on; lanes that
    // would come from outside the row give nothing
    auto over = [&](auto shift) {
      Stretch<N> o = stretch_moved<N, RESETS>(own, [](unsigned x, unsigned none) {
        constexpr int kControl = (FORWARD ? 0x110 : 0x100) + decltype(shift)::value;  // row_shr, row_shl
        return (unsigned)__builtin_amdgcn_update_dpp((int)none, (int)x, kControl, 0xF, 0xF, false);
      });
      return o;
    };
    using std::integral_constant;
    if constexpr (LANES == 1) {
      stretch_join<N, RESETS>(over(integral_constant<int, 1>()), own);
      stretch_join<N, RESETS>(over(integral_constant<int, 2>()), own);
    }
    stretch_join<N, RESETS>(over(integral_constant<int, 4>()), own);
    stretch_join<N, RESETS>(over(integral_constant<int, 8>()), own);
    others = over(integral_constant<int, LANES>());
    // the row's stretch: that of its last (first) slice
    own = stretch_moved<N, RESETS>(own, [&](unsigned x, unsigned) {
      return (unsigned)__shfl((int)x, (lane & 48) + (FORWARD ? 16 - LANES : 0) + lane % LANES);
    });
  }
  Stretch<N> even, odd;
  stretch_pair<N, RESETS, false>(own, even, odd);
  if constexpr (FORWARD) {
    if (lane & 16) stretch_join<N, RESETS>(even, others);
    stretch_join<N, RESETS>(even, odd);
    own = odd;
  } else {
    if (!(lane & 16)) stretch_join<N, RESETS>(odd, others);
    stretch_join<N, RESETS>(odd, even);
    own = even;
  }
  stretch_pair<N, RESETS, true>(own, even, odd);
  if constexpr (FORWARD) {
    if (lane & 32) stretch_join<N, RESETS>(even, others);
    stretch_join<N, RESETS>(even, odd);
    all = odd;
  } else {
    if (!(lane & 32)) stretch_join<N, RESETS>(odd, others);
    stretch_join<N, RESETS>(odd, even);
    all = even;
  }
  return others;
}

// The stretches of all of a block's threads, joined in the order of their slices (FORWARD) or
// against it, in every thread.
template <int N, int LANES, int WAVES, bool RESETS, bool FORWARD, typename Place>
__device__ __forceinline__ Stretch<N> block_stretch(const Place& p, const Stretch<N>& own) {
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
  Stretch<N> got = stretch_none<N>();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const int k = FORWARD ? w : WAVES - 1 - w, l = p.lane % LANES;
    Stretch<N> s;
#pragma unroll
    for (int j = 0; j < N; ++j) s.a[j] = sa[k][l][j], s.b[j] = sb[k][l][j];
    s.drop = RESETS && sd[k];
    stretch_join<N, RESETS>(got, s);
    got = s;
  }
  return got;
}

// The state from outside as it is before (FORWARD) or behind a chunk: the other chunks' parts
// on that side, a few for each slice of the block.
template <int N, int LANES, bool RESETS, bool FORWARD, typename Place>
__device__ __forceinline__ void state_at(const RecurArgs& r, const Place& p, long chunk, long chunks, float (&h)[N]) {
  constexpr int SLICES = kWave / LANES * 8;
  const long sites = r.outer * r.inner, at = p.o * r.inner + p.i;
  // the side's chunks first ... first + count - 1, and this slice's of them
  const long first = FORWARD ? 0 : chunk + 1, count = FORWARD ? chunk : chunks - first;
  const long each = (count + SLICES - 1) / SLICES, from = min(count, p.slice * each), to = min(count, from + each);
  Stretch<N> own = stretch_none<N>();
#pragma unroll 2
  for (long c = from; c < to; ++c) {
    const long k = 1 + first + (FORWARD ? c : from + to - 1 - c);
    Stretch<N> s = stretch_none<N>();
#pragma unroll
    for (int j = 0; j < N; ++j) s.a[j] = r.part_a[k * sites + at + j], s.b[j] = r.part_b[k * sites + at + j];
    s.drop = RESETS && r.part_drop[k * r.outer + p.o];
    stretch_join<N, RESETS>(own, s);
    own = s;
  }
  own = block_stretch<N, LANES, 8, RESETS, FORWARD>(p, own);
#pragma unroll
  for (int j = 0; j < N; ++j) h[j] = r.part_b[at + j];
  stretch_apply<N, RESETS>(own, h);
}

// What a chunk does to the state, to its part: every thread has walked its own stretch of the
// chunk.  The first chunk (backward: the last) also leaves the state from outside, so that
// a call may give back a state in its place.
template <int N, int LANES, int WAVES, bool RESETS, bool FORWARD, typename Place>
__device__ __forceinline__ void chunk_part(const RecurArgs& r, const Place& p, const Stretch<N>& own, long chunk,
                                           const float* outside, bool first) {
  const Stretch<N> got = block_stretch<N, LANES, WAVES, RESETS, FORWARD>(p, own);
  if (p.slice) return;
  const long sites = r.outer * r.inner, at = p.o * r.inner + p.i;
#pragma unroll
  for (int j = 0; j < N; ++j) {
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
    if (layout == kHalf && waves == 1) with(g, integral_constant<int, kHalf>(), integral_constant<int, 1>());
    else if (layout == kHalf) with(g, integral_constant<int, kHalf>(), integral_constant<int, 8>());
    else if (layout == kNarrow) with(g, integral_constant<int, kNarrow>(), integral_constant<int, 8>());
    else if (layout == kRow && waves == 1) with(g, integral_constant<int, kRow>(), integral_constant<int, 1>());
    else if (layout == kRow) with(g, integral_constant<int, kRow>(), integral_constant<int, 8>());
    else if (waves == 1) with(g, integral_constant<int, kWide>(), integral_constant<int, 1>());
    else with(g, integral_constant<int, kWide>(), integral_constant<int, 8>());
  };
  if (gate == BL_GATE_EXP) in(std::integral_constant<int, BL_GATE_EXP>());
  else in(std::integral_constant<int, BL_GATE_SIGMOID>());
}

// Steps of a thread in a tile: as many as there are registers for, since every tile has
// stretches to join over lanes and waves, which is 20 instructions a step and channel with
// four steps of two channels each and 12 with eight.
constexpr int recur_each(int layout, int wide, bool backward) {
  if (layout == kRow) return 16 / wide;
  return (layout == kHalf ? 16 : 8) / (backward ? 2 : 1);
}
template <typename T, int LAYOUT, bool BACKWARD>
constexpr int recur_each() {
  return recur_each(LAYOUT, (int)sizeof(T), BACKWARD);
}

// Lanes of channels that a block takes: as many as there are, or a few less, so that the last
// block is not left with fewer channels than a lane has (it would share them with the block
// before); 0 where no number does it.
inline int recur_lanes(const bl_recurrence_desc_t& d, int layout) {
  const int all = layout == kRow ? 1 : layout == kNarrow ? 4 : 16, vec = recur_vec(layout, dtype_bytes(d.dtype));
  if (vec == 1) return all;
  for (int lanes = all; lanes >= all / 2; --lanes) {
    const long rest = d.inner % (lanes * vec);
    if (!rest || rest >= vec) return lanes;
  }
  return 0;
}
// Blocks along sequences and channels (0: the layout does not do).
inline long recur_blocks(const bl_recurrence_desc_t& d, int layout) {
  const long channels = (long)recur_lanes(d, layout) * recur_vec(layout, dtype_bytes(d.dtype));
  return channels ? d.outer * ((d.inner + channels - 1) / channels) : 0;
}

bl_status_t recur_backward(const bl_recurrence_plan_s* p, const RecurArgs& r, hipStream_t s);

}  // namespace blc
