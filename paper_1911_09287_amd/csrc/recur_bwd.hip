// Gated linear recurrence, backward.
//
// What a step passes back, r_t = a_t (dy_t + r_(t+1)), is itself such a recurrence, from
// the last step to the first, with the same products of a.  So a block goes through the
// tiles from the last; in each it joins its threads' stretches both ways in one exchange,
// from the state that the forward pass saved at the tile's start and from what the tiles
// behind pass back, and goes through its steps in registers, forward for h_(t-1) and
// backward for dh_t = dy_t + r_(t+1).  gate, x and dy are read once, dgate and dx written
// once, and y is not needed, whose rounding would otherwise be dgate's.  Bound by HBM: 8 x 4096 x
// 1024 bf16 in 99 us, 336 MB at 3.4 TB/s in lines of 64 bytes; 8192 x 1250 fp32 with its steps side
// by side in 45.8 us, 205 MB at 4.5 TB/s.
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
  const long chunk = p.chunk, begin = chunk * r.chunk, end = min(r.length, begin + r.chunk);
  const long sites = r.outer * r.inner, at = p.o * r.inner + p.i;
  const T* gate = static_cast<const T*>(r.gate) + p.o * r.in_outer;
  const T* x = static_cast<const T*>(r.x) + p.o * r.in_outer;
  const T* dy = static_cast<const T*>(r.dy) + p.o * r.out_outer;
  T* dgate = static_cast<T*>(r.dgate) + p.o * r.in_outer;
  T* dx = static_cast<T*>(r.dx) + p.o * r.in_outer;
  const unsigned char* resets = RESETS ? r.resets + p.o * r.length : nullptr;
  float back[N];  // what the tiles behind pass back
  if (WAVES > 1 && gridDim.y > 1) {
    state_at<N, S::kLanes, RESETS, false>(r, p, chunk, gridDim.y, back);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) back[j] = r.dlast ? r.dlast[at + j] : 0.f;
  }
  // a tile's loads are in flight while the one behind it is worked on
  struct Raw {
    RecurRaw<T, LAYOUT, EACH> g, v, d;
    RecurResets<EACH, RESETS> z;
    float h[N];  // the state at the tile's start
  } raw[2];
  const long mine = p.slice * EACH;  // this thread's steps of a tile
  const unsigned in_off = (unsigned)((mine * r.in_step + p.i) * sizeof(T)), out_off = (unsigned)((mine * r.out_step + p.i) * sizeof(T));
  auto load = [&](auto full, Raw& w, long tile) {
    constexpr bool FULL = decltype(full)::value;
    const long t = tile + mine;
    if constexpr (FULL) {
      w.g.load_all(gate + tile * r.in_step, r.in_step, in_off);
      w.v.load_all(x + tile * r.in_step, r.in_step, in_off);
      w.d.load_all(dy + tile * r.out_step, r.out_step, out_off);
    } else {
      w.g.load(gate + t * r.in_step + p.i, r.in_step, end - t);
      w.v.load(x + t * r.in_step + p.i, r.in_step, end - t);
      w.d.load(dy + t * r.out_step + p.i, r.out_step, end - t);
    }
    w.z.template load<FULL>(resets + t, end - t);
    const float* state = r.states + tile / TILE * sites + at;
#pragma unroll
    for (int j = 0; j < N; ++j) w.h[j] = state[j];
  };
  int turn = 0;
  // a tile from w while the one before it is loaded; full: both are there, with all their steps
  auto work = [&](auto full, Raw& w, Raw& following, bool more, long tile) {
    constexpr bool FULL = decltype(full)::value;
    const long t = tile + mine, there = end - t;
    if (FULL || more) load(full, following, tile - TILE);
    const unsigned bits = w.z.bits();
    float a[EACH][N], rest[EACH][N];
    Stretch<N> own = stretch_none<N>(), rev = stretch_none<N>();
    w.g.refresh();
    w.v.refresh();
    w.d.refresh();
#pragma unroll
    for (int k = 0; k < EACH; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        gate_of<GATE>(w.g.at(k, j), a[k][j], rest[k][j]);
        if (!FULL && k >= there) a[k][j] = 1.f, rest[k][j] = 0.f;  // (x and dy are 0 there)
        const float b = rest[k][j] * w.v.at(k, j);
        own.b[j] = RESETS && (bits >> k & 1) ? b : fmaf(a[k][j], own.b[j], b);
        own.a[j] *= a[k][j];
      }
#pragma unroll
    for (int k = EACH - 1; k >= 0; --k)
#pragma unroll
      for (int j = 0; j < N; ++j) rev.b[j] = RESETS && (bits >> k & 1) ? 0.f : a[k][j] * (w.d.at(k, j) + rev.b[j]);
#pragma unroll
    for (int j = 0; j < N; ++j) rev.a[j] = own.a[j];
    own.drop = rev.drop = RESETS && bits;
    float s[N], back_now[N];  // this thread's state, and what is passed back to it
    Stretch<N> all, all_rev;
    const Stretch<N> before = wave_others<N, S::kLanes, RESETS, true>(own, all);
    const Stretch<N> behind = wave_others<N, S::kLanes, RESETS, false>(rev, all_rev);
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = w.h[j], back_now[j] = back[j];
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
      block_sync();  // (the other half is written before the next one)
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
        const float b = rest[k][j] * w.v.at(k, j);
        hs[k][j] = RESETS && (bits >> k & 1) ? 0.f : s[j];
        s[j] = RESETS && (bits >> k & 1) ? b : fmaf(a[k][j], s[j], b);
      }
    RecurOut<T, LAYOUT, EACH> og, ox;
#pragma unroll
    for (int k = EACH - 1; k >= 0; --k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float dh = w.d.at(k, j) + back_now[j], ah = a[k][j] * dh;
        if (GATE == BL_GATE_SIGMOID) {
          og.set(k, j, ah * rest[k][j] * (hs[k][j] - w.v.at(k, j)));
          ox.set(k, j, dh * rest[k][j]);
        } else {
          og.set(k, j, ah * hs[k][j]);
          ox.set(k, j, dh);
        }
        back_now[j] = RESETS && (bits >> k & 1) ? 0.f : ah;
      }
    if constexpr (FULL) {
      og.store_all(dgate + tile * r.in_step, r.in_step, in_off);
      ox.store_all(dx + tile * r.in_step, r.in_step, in_off);
    } else {
      og.store(dgate + t * r.in_step + p.i, r.in_step, there);
      ox.store(dx + t * r.in_step + p.i, r.in_step, there);
    }
    turn ^= 1;
  };
  constexpr std::true_type full;
  constexpr std::false_type any;
  long tile = begin + (end - begin - 1) / TILE * TILE;
  load(any, raw[0], tile);
  for (bool last = true; tile >= begin; last = false) {
    work(any, raw[0], raw[1], tile > begin, tile);
    raw[0] = raw[1];
    tile -= TILE;
    if (!last || !r.near || tile < begin + TILE) continue;
    // (one apart, so that each wait of the loop finds the same accesses behind it)
    work(full, raw[0], raw[1], true, tile);
    for (tile -= TILE; tile >= begin + 2 * TILE; tile -= 2 * TILE) {
      work(full, raw[1], raw[0], true, tile);
      work(full, raw[0], raw[1], true, tile - TILE);
    }
    raw[0] = raw[1];
  }
  if (r.dh0 && chunk == 0 && p.slice == 0) {
#pragma unroll
    for (int j = 0; j < N; ++j) r.dh0[at + j] = back[j];
  }
}

template <typename T, int GATE, int LAYOUT, bool RESETS>
__global__ __launch_bounds__(8 * kWave) void k_recur_bwd_part(RecurArgs r) {
  using S = RecurShape<T, LAYOUT>;
  constexpr int N = S::kVec, EACH = recur_each<T, LAYOUT, true>(), SLICES = S::kSlices * 8;
  const RecurPlace<T, LAYOUT, 8> p(r);
  const long chunk = p.chunk + 1, stretch = r.chunk / SLICES;  // (a multiple of EACH)
  const long first = chunk * r.chunk, begin = first + p.slice * stretch, end = min(r.length, begin + stretch);
  const T* gate = static_cast<const T*>(r.gate) + p.o * r.in_outer;
  const T* dy = static_cast<const T*>(r.dy) + p.o * r.out_outer;
  const unsigned char* resets = RESETS ? r.resets + p.o * r.length : nullptr;
  struct Raw {
    RecurRaw<T, LAYOUT, EACH> g, d;
    RecurResets<EACH, RESETS> z;
  } raw[2];
  Stretch<N> own = stretch_none<N>();
  auto work = [&](Raw& w, long there) {
    w.g.refresh();
    w.d.refresh();
    const unsigned bits = w.z.bits();
#pragma unroll
    for (int k = EACH - 1; k >= 0; --k)
      if (k < there) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          float a, rest;
          gate_of<GATE>(w.g.at(k, j), a, rest);
          own.b[j] = RESETS && (bits >> k & 1) ? 0.f : a * (w.d.at(k, j) + own.b[j]);
          own.a[j] *= a;
        }
      }
    own.drop |= RESETS && bits;
  };
  const long widest = max(r.in_step, r.out_step);
  if (first + r.chunk <= r.length && (r.chunk * widest + r.inner) * (long)sizeof(T) < 1L << 32) {
    // the chunk is whole: the loads of the steps before are in flight while these are worked on
    const unsigned in_off = (unsigned)((p.slice * stretch * r.in_step + p.i) * sizeof(T));
    const unsigned out_off = (unsigned)((p.slice * stretch * r.out_step + p.i) * sizeof(T));
    auto load = [&](Raw& w, long t) {
      w.g.load_all(gate + (first + t) * r.in_step, r.in_step, in_off);
      w.d.load_all(dy + (first + t) * r.out_step, r.out_step, out_off);
      w.z.template load<true>(resets + begin + t, EACH);
    };
    load(raw[0], stretch - EACH);
    for (long t = stretch - EACH; t >= 0; t -= 2 * EACH) {
      if (t > 0) load(raw[1], t - EACH);
      work(raw[0], EACH);
      if (t <= 0) break;
      if (t > EACH) load(raw[0], t - 2 * EACH);
      work(raw[1], EACH);
    }
  } else {
    for (long t = begin + (stretch - EACH); t >= begin; t -= EACH) {
      if (t >= end) continue;
      raw[0].g.load(gate + t * r.in_step + p.i, r.in_step, end - t);
      raw[0].d.load(dy + t * r.out_step + p.i, r.out_step, end - t);
      raw[0].z.template load<false>(resets + t, end - t);
      work(raw[0], end - t);
    }
  }
  chunk_part<N, S::kLanes, 8, RESETS, false>(r, p, own, chunk, r.dlast, chunk == (long)gridDim.y);
}

template <typename T>
bl_status_t backward(const bl_recurrence_plan_s* p, RecurArgs r, hipStream_t s) {
  const bl_recurrence_desc_t& d = p->d;
  const double bytes = 5.0 * d.outer * d.length * d.inner * sizeof(T);
  const dim3 grid((unsigned)recur_blocks(d, p->layout[1]), (unsigned)p->chunks[1]);
  r.chunk = p->chunk[1];
  r.lanes = p->lanes[1];
  if (p->chunks[1] > 1) {
    // (nothing is passed back from the first chunk to another)
    const dim3 parts(grid.x, grid.y - 1);
    const bl_status_t st = timed_launch("recur_bwd_part", bytes * 2 / 5, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      recur_dispatch(d.gate, p->layout[1], 8, r.resets, [&](auto g, auto l, auto, auto z) {
        hipExtLaunchKernelGGL((k_recur_bwd_part<T, decltype(g)::value, decltype(l)::value, decltype(z)::value>), parts,
                              dim3(8 * kWave), 0, s, e0, e1, 0, r);
      });
    });
    if (st != BL_OK) return st;
  }
  return timed_launch("recur_bwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    recur_dispatch(d.gate, p->layout[1], p->waves[1], r.resets, [&](auto g, auto l, auto w, auto z) {
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
