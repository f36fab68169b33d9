// Gated linear recurrence, backward.
//
// What a step passes back, r_t = a_t (dy_t + r_(t+1)), is itself such a recurrence, from
// the last step to the first, with the same products of a.  So a block goes through the
// tiles from the last; in each it joins its threads' stretches both ways in one exchange,
// from the state that the forward pass saved at the tile's start and from what the tiles
// behind pass back, and goes through its steps in registers, forward for h_(t-1) and
// backward for dh_t = dy_t + r_(t+1).  gate, x and dy are read once, dgate and dx written
// once, and y is not needed, whose rounding would otherwise be dgate's.
#include <algorithm>

#include "recur.hpp"

namespace blc {
namespace {

template <typename T, int GATE, int LAYOUT, int WAVES, bool RESETS>
__global__ __launch_bounds__(WAVES* kWave) void k_recur_bwd(RecurArgs r) {
  using S = RecurShape<T, LAYOUT>;
  constexpr int N = S::kVec, EACH = recur_each<T, LAYOUT, true>(), TILE = S::kSlices * WAVES * EACH;
  // products, and the sums forward and backward
  __shared__ float sa[2][WAVES][S::kLanes][N], sb[2][WAVES][S::kLanes][N], sr[2][WAVES][S::kLanes][N];
  __shared__ int sd[2][WAVES];
  const RecurPlace<T, LAYOUT, WAVES> p(r);
  const long chunk = blockIdx.y, begin = chunk * r.chunk, end = min(r.length, begin + r.chunk);
  const long sites = r.outer * r.inner, at = p.o * r.inner + p.i;
  const T* gate = static_cast<const T*>(r.gate) + p.o * r.in_outer + p.i;
  const T* x = static_cast<const T*>(r.x) + p.o * r.in_outer + p.i;
  const T* dy = static_cast<const T*>(r.dy) + p.o * r.out_outer + p.i;
  T* dgate = static_cast<T*>(r.dgate) + p.o * r.in_outer + p.i;
  T* dx = static_cast<T*>(r.dx) + p.o * r.in_outer + p.i;
  const unsigned char* resets = RESETS ? r.resets + p.o * r.length : nullptr;
  float back[N];  // what the tiles behind pass back
  if (gridDim.y > 1) {
    state_at<N, RESETS>(r, p.o, p.i, p.n, gridDim.y - 1, -1, gridDim.y - 1 - chunk, back);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) back[j] = r.dlast && j < p.n ? r.dlast[at + j] : 0.f;
  }
  const long tiles = (end - begin + TILE - 1) / TILE;
  long t = begin + (tiles - 1) * TILE + p.slice * EACH;
  RecurRaw<T, LAYOUT, EACH> g, v, d;
  unsigned bits;
  float h[N];  // the state at the tile's start
  auto load = [&](long from, long there) {
    g.load(gate + from * r.in_step, r.in_step, there, p.n);
    v.load(x + from * r.in_step, r.in_step, there, p.n);
    d.load(dy + from * r.out_step, r.out_step, there, p.n);
    bits = reset_bits<EACH, RESETS>(resets + from, there);
    const long tile = (from - p.slice * EACH) / TILE;
#pragma unroll
    for (int j = 0; j < N; ++j) h[j] = there > -TILE && j < p.n ? r.states[tile * sites + at + j] : 0.f;
  };
  load(t, end - t);
  int turn = 0;
  for (long tile = tiles - 1; tile >= 0; --tile, t -= TILE, turn ^= 1) {
    const long there = end - t;
    float a[EACH][N], rest[EACH][N], xs[EACH][N], ds[EACH][N];
    Stretch<N> own = stretch_none<N>(), rev = stretch_none<N>();
    g.refresh();
    v.refresh();
    d.refresh();
#pragma unroll
    for (int k = 0; k < EACH; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        gate_of<GATE>(g.at(k, j), a[k][j], rest[k][j]);
        xs[k][j] = v.at(k, j);
        ds[k][j] = d.at(k, j);
        if (k >= there) a[k][j] = 1.f, rest[k][j] = 0.f, xs[k][j] = 0.f, ds[k][j] = 0.f;
        const float b = rest[k][j] * xs[k][j];
        own.b[j] = RESETS && (bits >> k & 1) ? b : fmaf(a[k][j], own.b[j], b);
        own.a[j] *= a[k][j];
      }
#pragma unroll
    for (int k = EACH - 1; k >= 0; --k)
#pragma unroll
      for (int j = 0; j < N; ++j) rev.b[j] = RESETS && (bits >> k & 1) ? 0.f : a[k][j] * (ds[k][j] + rev.b[j]);
#pragma unroll
    for (int j = 0; j < N; ++j) rev.a[j] = own.a[j];
    own.drop = rev.drop = RESETS && bits;
    const unsigned now = bits;
    float s[N], back_now[N];  // this thread's state, and what is passed back to it
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = h[j];
    if (tile > 0) load(t - TILE, there + TILE);
    Stretch<N> all, all_rev;
    const Stretch<N> before = wave_others<N, S::kLanes, RESETS, true>(own, all);
    const Stretch<N> behind = wave_others<N, S::kLanes, RESETS, false>(rev, all_rev);
#pragma unroll
    for (int j = 0; j < N; ++j) back_now[j] = back[j];
    if constexpr (WAVES == 1) {
      stretch_apply<N, RESETS>(all_rev, back);
    } else {
      const int l = p.lane % S::kLanes;
      if (p.lane < S::kLanes) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          sa[turn][p.wave][l][j] = all.a[j];
          sb[turn][p.wave][l][j] = all.b[j];
          sr[turn][p.wave][l][j] = all_rev.b[j];
        }
        if (p.lane == 0) sd[turn][p.wave] = all.drop;
      }
      __syncthreads();  // (the other half is written before the next one)
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        Stretch<N> o;
#pragma unroll
        for (int j = 0; j < N; ++j) o.a[j] = sa[turn][w][l][j], o.b[j] = sb[turn][w][l][j];
        o.drop = RESETS && sd[turn][w];
        if (w < p.wave) stretch_apply<N, RESETS>(o, s);
      }
#pragma unroll
      for (int w = WAVES - 1; w >= 0; --w) {
        Stretch<N> o;
#pragma unroll
        for (int j = 0; j < N; ++j) o.a[j] = sa[turn][w][l][j], o.b[j] = sr[turn][w][l][j];
        o.drop = RESETS && sd[turn][w];
        if (w == p.wave)
#pragma unroll
          for (int j = 0; j < N; ++j) back_now[j] = back[j];
        stretch_apply<N, RESETS>(o, back);
      }
    }
    stretch_apply<N, RESETS>(before, s);
    stretch_apply<N, RESETS>(behind, back_now);
    float hs[EACH][N];  // h before each step
#pragma unroll
    for (int k = 0; k < EACH; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        hs[k][j] = RESETS && (now >> k & 1) ? 0.f : s[j];
        s[j] = RESETS && (now >> k & 1) ? rest[k][j] * xs[k][j] : fmaf(a[k][j], s[j], rest[k][j] * xs[k][j]);
      }
    RecurOut<T, LAYOUT, EACH> og, ox;
#pragma unroll
    for (int k = EACH - 1; k >= 0; --k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float dh = ds[k][j] + back_now[j], ah = a[k][j] * dh;
        if (GATE == BL_GATE_SIGMOID) {
          og.set(k, j, ah * rest[k][j] * (hs[k][j] - xs[k][j]));
          ox.set(k, j, dh * rest[k][j]);
        } else {
          og.set(k, j, ah * hs[k][j]);
          ox.set(k, j, dh);
        }
        back_now[j] = RESETS && (now >> k & 1) ? 0.f : ah;
        if (k >= there) back_now[j] = dh;
      }
    og.store(dgate + t * r.in_step, r.in_step, there, p.n);
    ox.store(dx + t * r.in_step, r.in_step, there, p.n);
  }
  if (r.dh0 && chunk == 0 && p.slice == 0) {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < p.n) r.dh0[at + j] = back[j];
  }
}

template <typename T, int GATE, int LAYOUT, bool RESETS>
__global__ __launch_bounds__(8 * kWave) void k_recur_bwd_part(RecurArgs r) {
  using S = RecurShape<T, LAYOUT>;
  constexpr int N = S::kVec, EACH = recur_each<T, LAYOUT, true>(), SLICES = S::kSlices * 8;
  const RecurPlace<T, LAYOUT, 8> p(r);
  const long chunk = blockIdx.y, stretch = r.chunk / SLICES;  // (a multiple of EACH)
  const long begin = chunk * r.chunk + p.slice * stretch, end = min(r.length, begin + stretch);
  const T* gate = static_cast<const T*>(r.gate) + p.o * r.in_outer + p.i;
  const T* dy = static_cast<const T*>(r.dy) + p.o * r.out_outer + p.i;
  Stretch<N> own = stretch_none<N>();
  for (long t = begin + (stretch - EACH); t >= begin; t -= EACH) {
    if (t >= end) continue;
    RecurRaw<T, LAYOUT, EACH> g, d;
    g.load(gate + t * r.in_step, r.in_step, end - t, p.n);
    d.load(dy + t * r.out_step, r.out_step, end - t, p.n);
    const unsigned bits = reset_bits<EACH, RESETS>(RESETS ? r.resets + p.o * r.length + t : nullptr, end - t);
    g.refresh();
    d.refresh();
#pragma unroll
    for (int k = EACH - 1; k >= 0; --k)
      if (k < end - t) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          float a, rest;
          gate_of<GATE>(g.at(k, j), a, rest);
          own.b[j] = RESETS && (bits >> k & 1) ? 0.f : a * (d.at(k, j) + own.b[j]);
          own.a[j] *= a;
        }
      }
    own.drop |= RESETS && bits;
  }
  chunk_part<N, S::kLanes, 8, RESETS, false>(r, p, own, chunk, r.dlast, chunk == (long)gridDim.y - 1);
}

template <typename T>
bl_status_t backward(const bl_recurrence_plan_s* p, RecurArgs r, hipStream_t s) {
  const bl_recurrence_desc_t& d = p->d;
  const double bytes = 5.0 * d.outer * d.length * d.inner * sizeof(T);
  const long lanes = p->layout == kWide ? 16 * (8 / (int)sizeof(T)) : p->layout == kNarrow ? 4 : 1;
  const dim3 grid((unsigned)(d.outer * ((d.inner + lanes - 1) / lanes)), (unsigned)p->chunks[1]);
  r.chunk = p->chunk[1];
  if (p->chunks[1] > 1) {
    const bl_status_t st = timed_launch("recur_bwd_part", bytes * 2 / 5, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      recur_dispatch(d.gate, p->layout, 8, r.resets, [&](auto g, auto l, auto, auto z) {
        hipExtLaunchKernelGGL((k_recur_bwd_part<T, decltype(g)::value, decltype(l)::value, decltype(z)::value>), grid,
                              dim3(8 * kWave), 0, s, e0, e1, 0, r);
      });
    });
    if (st != BL_OK) return st;
  }
  return timed_launch("recur_bwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    recur_dispatch(d.gate, p->layout, p->waves[1], r.resets, [&](auto g, auto l, auto w, auto z) {
      hipExtLaunchKernelGGL((k_recur_bwd<T, decltype(g)::value, decltype(l)::value, decltype(w)::value, decltype(z)::value>),
                            grid, dim3(decltype(w)::value * kWave), 0, s, e0, e1, 0, r);
    });
  });
}

}  // namespace

bl_status_t recur_backward(const bl_recurrence_plan_s* p, const RecurArgs& r, hipStream_t s) {
  if (p->d.dtype == BL_F32) return backward<float>(p, r, s);
  if (p->d.dtype == BL_BF16) return backward<bf16_t>(p, r, s);
  return backward<f16_t>(p, r, s);
}

}  // namespace blc
