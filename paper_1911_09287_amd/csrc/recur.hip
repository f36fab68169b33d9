// Gated linear recurrence h_t = a_t h_(t-1) + b_t: plan, dispatch and the forward pass.
//
// A stretch of steps takes the state h to A h + B with A the product of its a and B the
// sum of its b, each times the a behind it; two stretches join to one, (A2 A1, A2 B1 + B2).
// So a block reads a tile of steps once, every thread joins its own few steps, the
// stretches before a thread's are joined over lanes and waves, and each thread then goes
// through its steps again in registers.  Bound by HBM: gate and x are read once, y is
// written once: 8 x 4096 x 2048 bf16 in 92.6 us, 403 MB at 4.3 TB/s.  Where sequences are too few for
// the GPU the length is cut into chunks, whose parts a launch before takes, and which reads gate
// and x once more: 1 x 65537 x 256 fp32 in 37.5 + 41.8 us, 335 MB at 4.2 TB/s (one block for each
// 32 channels: eight compute units).
#include <algorithm>
#include <new>

#include "recur.hpp"

namespace blc {
namespace {

template <typename T, int GATE, int LAYOUT, int WAVES, bool RESETS>
__global__ __launch_bounds__(WAVES* kWave) void k_recur_fwd(RecurArgs r) {
  using S = RecurShape<T, LAYOUT>;
  constexpr int N = S::kVec, EACH = recur_each<T, LAYOUT, false>(), TILE = S::kSlices * WAVES * EACH;
  __shared__ float sa[2][WAVES][S::kLanes][N], sb[2][WAVES][S::kLanes][N];
  __shared__ int sd[2][WAVES];
  const RecurPlace<T, LAYOUT, WAVES> p(r);
  const long chunk = p.chunk, begin = chunk * r.chunk, end = min(r.length, begin + r.chunk);
  const long sites = r.outer * r.inner, at = p.o * r.inner + p.i;
  const T* gate = static_cast<const T*>(r.gate) + p.o * r.in_outer;
  const T* x = static_cast<const T*>(r.x) + p.o * r.in_outer;
  T* y = static_cast<T*>(r.y) + p.o * r.out_outer;
  const unsigned char* resets = RESETS ? r.resets + p.o * r.length : nullptr;
  float h[N];  // before the tile
  if (WAVES > 1 && gridDim.y > 1) {
    state_at<N, S::kLanes, RESETS, true>(r, p, chunk, gridDim.y, h);
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) h[j] = r.h0 ? r.h0[at + j] : 0.f;
  }
  // a tile's loads are in flight while the one before it is worked on
  struct Raw {
    RecurRaw<T, LAYOUT, EACH> g, v;
    RecurResets<EACH, RESETS> z;
  } raw[2];
  const long mine = p.slice * EACH;  // this thread's steps of a tile
  const unsigned in_off = (unsigned)((mine * r.in_step + p.i) * sizeof(T)), out_off = (unsigned)((mine * r.out_step + p.i) * sizeof(T));
  auto load = [&](auto full, Raw& w, long tile) {
    constexpr bool FULL = decltype(full)::value;
    const long t = tile + mine;
    if constexpr (FULL) {
      w.g.load_all(gate + tile * r.in_step, r.in_step, in_off);
      w.v.load_all(x + tile * r.in_step, r.in_step, in_off);
    } else {
      w.g.load(gate + t * r.in_step + p.i, r.in_step, end - t);
      w.v.load(x + t * r.in_step + p.i, r.in_step, end - t);
    }
    w.z.template load<FULL>(resets + t, end - t);
  };
  int turn = 0;
  // a tile from w while the following one is loaded; full: both have all their steps
  auto work = [&](auto full, Raw& w, Raw& following, long tile) {
    constexpr bool FULL = decltype(full)::value;
    const long t = tile + mine, there = end - t;
    load(full, following, tile + TILE);
    const unsigned bits = w.z.bits();
    float a[EACH][N], b[EACH][N];
    Stretch<N> own = stretch_none<N>();
    w.g.refresh();
    w.v.refresh();
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
#pragma unroll
      for (int j = 0; j < N; ++j) {
        float rest;
        gate_of<GATE>(w.g.at(k, j), a[k][j], rest);
        b[k][j] = rest * w.v.at(k, j);
        if (!FULL && k >= there) a[k][j] = 1.f, b[k][j] = 0.f;
        own.b[j] = RESETS && (bits >> k & 1) ? b[k][j] : fmaf(a[k][j], own.b[j], b[k][j]);
        own.a[j] *= a[k][j];
      }
    }
    own.drop = RESETS && bits;
    Stretch<N> all;
    const Stretch<N> before = wave_others<N, S::kLanes, RESETS, true>(own, all);
    float s[N];  // this thread's state
#pragma unroll
    for (int j = 0; j < N; ++j) s[j] = h[j];
    if constexpr (WAVES == 1) {
      stretch_apply<N, RESETS>(all, h);
    } else {
      if (p.lane < S::kLanes) {
#pragma unroll
        for (int j = 0; j < N; ++j) sa[turn][p.wave][p.lane][j] = all.a[j], sb[turn][p.wave][p.lane][j] = all.b[j];
        if (p.lane == 0) sd[turn][p.wave] = all.drop;
      }
      block_sync();  // (the other half is written before the next one)
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        Stretch<N> o;
#pragma unroll
        for (int j = 0; j < N; ++j) o.a[j] = sa[turn][w][p.lane % S::kLanes][j], o.b[j] = sb[turn][w][p.lane % S::kLanes][j];
        o.drop = RESETS && sd[turn][w];
        if (w == p.wave)
#pragma unroll
          for (int j = 0; j < N; ++j) s[j] = h[j];
        stretch_apply<N, RESETS>(o, h);
      }
    }
    stretch_apply<N, RESETS>(before, s);
    if (r.states && there > 0 && (t & (r.every - 1)) == 0) {
#pragma unroll
      for (int j = 0; j < N; ++j) r.states[(t >> r.every_log2) * sites + at + j] = s[j];
    }
    RecurOut<T, LAYOUT, EACH> out;
#pragma unroll
    for (int k = 0; k < EACH; ++k)
#pragma unroll
      for (int j = 0; j < N; ++j) {
        s[j] = RESETS && (bits >> k & 1) ? b[k][j] : fmaf(a[k][j], s[j], b[k][j]);
        out.set(k, j, s[j]);
      }
    if constexpr (FULL) out.store_all(y + tile * r.out_step, r.out_step, out_off);
    else out.store(y + t * r.out_step + p.i, r.out_step, there);
    turn ^= 1;
  };
  constexpr std::true_type full;
  constexpr std::false_type any;
  long t = begin;
  load(any, raw[0], t);
  if (r.near && t + 2 * TILE <= end) {
    // (the first one apart, so that each wait of the loop finds the same accesses behind it)
    work(full, raw[0], raw[1], t);
    for (t += TILE; t + 3 * TILE <= end; t += 2 * TILE) {
      work(full, raw[1], raw[0], t);
      work(full, raw[0], raw[1], t + TILE);
    }
    raw[0] = raw[1];
  }
  for (; t < end; t += TILE) {
    work(any, raw[0], raw[1], t);
    raw[0] = raw[1];
  }
  if (r.last && end == r.length && p.slice == 0) {
#pragma unroll
    for (int j = 0; j < N; ++j) r.last[at + j] = h[j];
  }
}

template <typename T, int GATE, int LAYOUT, bool RESETS>
__global__ __launch_bounds__(8 * kWave) void k_recur_fwd_part(RecurArgs r) {
  using S = RecurShape<T, LAYOUT>;
  constexpr int N = S::kVec, EACH = recur_each<T, LAYOUT, false>(), SLICES = S::kSlices * 8;
  const RecurPlace<T, LAYOUT, 8> p(r);
  const long chunk = p.chunk, stretch = r.chunk / SLICES;  // (a multiple of EACH)
  const long first = chunk * r.chunk, begin = first + p.slice * stretch, end = min(r.length, begin + stretch);
  const T* gate = static_cast<const T*>(r.gate) + p.o * r.in_outer;
  const T* x = static_cast<const T*>(r.x) + p.o * r.in_outer;
  const unsigned char* resets = RESETS ? r.resets + p.o * r.length : nullptr;
  struct Raw {
    RecurRaw<T, LAYOUT, EACH> g, v;
    RecurResets<EACH, RESETS> z;
  } raw[2];
  Stretch<N> own = stretch_none<N>();
  auto work = [&](Raw& w, long there) {
    w.g.refresh();
    w.v.refresh();
    const unsigned bits = w.z.bits();
#pragma unroll
    for (int k = 0; k < EACH; ++k)
      if (k < there) {
#pragma unroll
        for (int j = 0; j < N; ++j) {
          float a, rest;
          gate_of<GATE>(w.g.at(k, j), a, rest);
          const float b = rest * w.v.at(k, j);
          own.b[j] = RESETS && (bits >> k & 1) ? b : fmaf(a, own.b[j], b);
          own.a[j] *= a;
        }
      }
    own.drop |= RESETS && bits;
  };
  if (first + r.chunk <= r.length && (r.chunk * r.in_step + r.inner) * (long)sizeof(T) < 1L << 32) {
    // the chunk is whole: the following steps' loads are in flight while these are worked on
    const unsigned off = (unsigned)((p.slice * stretch * r.in_step + p.i) * sizeof(T));
    auto load = [&](Raw& w, long t) {
      w.g.load_all(gate + (first + t) * r.in_step, r.in_step, off);
      w.v.load_all(x + (first + t) * r.in_step, r.in_step, off);
      w.z.template load<true>(resets + begin + t, EACH);
    };
    load(raw[0], 0);
    for (long t = 0; t < stretch; t += 2 * EACH) {
      if (t + EACH < stretch) load(raw[1], t + EACH);
      work(raw[0], EACH);
      if (t + EACH >= stretch) break;
      if (t + 2 * EACH < stretch) load(raw[0], t + 2 * EACH);
      work(raw[1], EACH);
    }
  } else {
    for (long t = begin; t < end; t += EACH) {
      raw[0].g.load(gate + t * r.in_step + p.i, r.in_step, end - t);
      raw[0].v.load(x + t * r.in_step + p.i, r.in_step, end - t);
      raw[0].z.template load<false>(resets + t, end - t);
      work(raw[0], end - t);
    }
  }
  chunk_part<N, S::kLanes, 8, RESETS, true>(r, p, own, chunk, r.h0, chunk == 0);
}

// Few steps of many channels: a thread walks all of its channels' steps.
template <typename T, int GATE, bool RESETS>
__global__ __launch_bounds__(kThreads) void k_recur_serial(RecurArgs r, int vec_per) {
  constexpr int N = 8 / (int)sizeof(T);
  const long q = (long)blockIdx.x * kThreads + threadIdx.x, o = q / vec_per, i = (q - o * vec_per) * N, n = r.inner - i;
  if (o >= r.outer) return;
  const long sites = r.outer * r.inner, at = o * r.inner + i;
  const T* gate = static_cast<const T*>(r.gate) + o * r.in_outer + i;
  const T* x = static_cast<const T*>(r.x) + o * r.in_outer + i;
  T* y = static_cast<T*>(r.y) + o * r.out_outer + i;
  float h[N];
#pragma unroll
  for (int j = 0; j < N; ++j) h[j] = r.h0 && j < n ? r.h0[at + j] : 0.f;
  for (long t = 0; t < r.length; ++t) {
    Held<T, N> g, v;
    g.load(gate + t * r.in_step, n);
    v.load(x + t * r.in_step, n);
    const bool drop = RESETS && r.resets[o * r.length + t];
    if (r.states && (t & (r.every - 1)) == 0) {
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < n) r.states[(t >> r.every_log2) * sites + at + j] = h[j];
    }
    g.refresh();
    v.refresh();
    Pack<T, N> out;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      float a, rest;
      gate_of<GATE>(g[j], a, rest);
      h[j] = drop ? rest * v[j] : fmaf(a, h[j], rest * v[j]);
      out.v[j] = (T)h[j];
    }
    store_part(y + t * r.out_step, n, out);
  }
  if (r.last) {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < n) r.last[at + j] = h[j];
  }
}

// A state of no steps: the one from outside.
__global__ void k_recur_none(const float* from, float* to, long n) {
  const long i = (long)blockIdx.x * kThreads + threadIdx.x;
  if (i < n) to[i] = from ? from[i] : 0.f;
}

constexpr long kUnits = 256;  // compute units
// Up to this many steps a thread walks them alone.
constexpr long kSerialSteps = 8;

template <typename T>
bl_status_t forward(const bl_recurrence_plan_s* p, RecurArgs r, hipStream_t s) {
  const bl_recurrence_desc_t& d = p->d;
  const double bytes = 3.0 * d.outer * d.length * d.inner * sizeof(T);
  if (d.length <= kSerialSteps) {
    constexpr int N = 8 / (int)sizeof(T);
    const int per = (int)((d.inner + N - 1) / N);
    const dim3 grid((unsigned)((d.outer * per + kThreads - 1) / kThreads));
    return timed_launch("recur_fwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      recur_dispatch(d.gate, kWide, 1, r.resets, [&](auto g, auto, auto, auto z) {
        hipExtLaunchKernelGGL((k_recur_serial<T, decltype(g)::value, decltype(z)::value>), grid, dim3(kThreads), 0, s,
                              e0, e1, 0, r, per);
      });
    });
  }
  const dim3 grid((unsigned)recur_blocks(d, p->layout[0]), (unsigned)p->chunks[0]);
  r.chunk = p->chunk[0];
  r.lanes = p->lanes[0];
  if (p->chunks[0] > 1) {
    // (nothing follows the last chunk)
    const dim3 parts(grid.x, grid.y - 1);
    const bl_status_t st = timed_launch("recur_fwd_part", bytes * 2 / 3, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      recur_dispatch(d.gate, p->layout[0], 8, r.resets, [&](auto g, auto l, auto, auto z) {
        hipExtLaunchKernelGGL((k_recur_fwd_part<T, decltype(g)::value, decltype(l)::value, decltype(z)::value>), parts,
                              dim3(8 * kWave), 0, s, e0, e1, 0, r);
      });
    });
    if (st != BL_OK) return st;
  }
  return timed_launch("recur_fwd", bytes, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    recur_dispatch(d.gate, p->layout[0], p->waves[0], r.resets, [&](auto g, auto l, auto w, auto z) {
      hipExtLaunchKernelGGL((k_recur_fwd<T, decltype(g)::value, decltype(l)::value, decltype(w)::value, decltype(z)::value>),
                            grid, dim3(decltype(w)::value * kWave), 0, s, e0, e1, 0, r);
    });
  });
}

RecurArgs args_of(const bl_recurrence_plan_s* p, void* ws) {
  RecurArgs r{};
  const bl_recurrence_desc_t& d = p->d;
  r.outer = d.outer;
  r.length = d.length;
  r.inner = d.inner;
  r.in_outer = d.in_outer;
  r.in_step = d.in_step;
  r.out_outer = d.out_outer;
  r.out_step = d.out_step;
  r.every = p->every;
  while (1L << r.every_log2 < r.every) ++r.every_log2;
  const long tile = 8L * kWave * 8;  // (steps of any tile, at most)
  r.near = (tile * std::max(d.in_step, d.out_step) + d.inner) * dtype_bytes(d.dtype) < 1LL << 32;
  const long parts = std::max(p->chunks[0], p->chunks[1]) + 1, sites = d.outer * d.inner;
  r.part_a = static_cast<float*>(ws);
  r.part_b = r.part_a + parts * sites;
  r.part_drop = reinterpret_cast<unsigned char*>(r.part_b + parts * sites);
  return r;
}

}  // namespace

bl_status_t recur_none(const float* from, float* to, long n, hipStream_t s) {
  if (!to) return BL_OK;
  return timed_launch("recur_none", 8.0 * n, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL(k_recur_none, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, s, e0, e1, 0,
                          from, to, n);
  });
}

}  // namespace blc

using namespace blc;

extern "C" bl_status_t bl_recurrence_plan_create(bl_recurrence_plan_t* out, const bl_recurrence_desc_t* desc) {
  if (!out || !desc) return BL_ERR_INVALID_ARG;
  *out = nullptr;
  bl_recurrence_desc_t d = *desc;
  if (d.outer < 0 || d.length < 0 || d.inner < 1 || !known_dtype(d.dtype)) return BL_ERR_INVALID_ARG;
  if (d.gate != BL_GATE_SIGMOID && d.gate != BL_GATE_EXP) return BL_ERR_INVALID_ARG;
  if (d.in_outer < 0 || d.in_step < 0 || d.out_outer < 0 || d.out_step < 0) return BL_ERR_INVALID_ARG;
  const long long most = (1LL << 31) - 1;
  if (d.outer > most || d.inner > most || d.length > most || d.outer * d.inner > most) return BL_ERR_UNSUPPORTED;
  if (!d.in_step) d.in_step = d.inner;
  if (!d.out_step) d.out_step = d.inner;
  // (no offset of an element may leave 62 bits)
  const __int128 bound = (__int128)1 << 60;
  if ((__int128)d.in_step * d.length > bound || (__int128)d.out_step * d.length > bound) return BL_ERR_UNSUPPORTED;
  if (!d.in_outer) d.in_outer = d.length * d.in_step;
  if (!d.out_outer) d.out_outer = d.length * d.out_step;
  if ((__int128)d.in_outer * d.outer > bound || (__int128)d.out_outer * d.outer > bound) return BL_ERR_UNSUPPORTED;
  // steps and sequences may interleave, but no two elements may share a place: the
  // larger of two strides spans what the smaller one covers
  auto apart = [&](long long step, long long per) {
    if (d.length > 1 && step < d.inner) return false;
    if (d.outer <= 1 || !d.length) return true;
    return per >= step ? per >= (d.length - 1) * step + d.inner
                       : per >= d.inner && (d.length <= 1 || step >= (d.outer - 1) * per + d.inner);
  };
  if (!apart(d.in_step, d.in_outer) || !apart(d.out_step, d.out_outer)) return BL_ERR_INVALID_ARG;
  bl_recurrence_plan_s* p = new (std::nothrow) bl_recurrence_plan_s{};
  if (!p) return BL_ERR_OOM;
  p->d = d;
  const bool row = d.inner == 1 && d.in_step == 1 && d.out_step == 1;
  long most_threads = 0;
  for (int i = 0; i < 2; ++i) {
    double best = 0.0;
    auto consider = [&](int layout, double rate) {
      const long lanes = recur_lanes(d, layout), blocks = std::max(recur_blocks(d, layout), 1L);
      if (!lanes) return;
      const long slices = layout == kRow ? kWave : layout == kNarrow ? 16 : 4;
      const long tile = slices * recur_each(layout, dtype_bytes(d.dtype), i), part = 8 * tile;  // of a wave, of eight
      // one wave a block: rows in such a number that they fill the GPU, or sequences of one tile
      const int waves = layout != kNarrow && (d.length <= tile || (layout == kRow && blocks >= 2048)) ? 1 : 8;
      // fewer blocks than compute units (each has registers for one): chunks of four tiles at
      // least, whose loads of a part more (all but one chunk's gates and values or dy) are
      // weighed against the units that have none
      const long most = waves == 1 || blocks >= kUnits ? 1 : std::max(1L, std::min<long>(4 * kUnits / blocks, d.length / (4 * part)));
      for (long n = 1; n <= most; ++n) {
        const long all = n * blocks, turns = (all + kUnits - 1) / kUnits;
        const double full = most > 1 ? (double)all / (double)(turns * kUnits) : std::min(1.0, (double)blocks / kUnits);
        const double more = (i ? 2.0 / 5.0 : 2.0 / 3.0) * (double)(n - 1) / (double)n;
        const double speed = rate * full / (1.0 + more);
        if (speed <= best * 1.02) continue;
        best = speed;
        p->layout[i] = layout;
        p->lanes[i] = (int)lanes;
        p->waves[i] = waves;
        p->chunk[i] = n > 1 ? ((d.length + n - 1) / n + part - 1) / part * part : std::max<long>(d.length, 1);
        p->chunks[i] = n > 1 ? (d.length + p->chunk[i] - 1) / p->chunk[i] : 1;
      }
    };
    if (row) consider(kRow, 1.0);
    if (!row && d.inner > 4) {
      // lines of 64 bytes against 128: bf16, 8 x 4096 x 1024 forward 3.4 TB/s, twice the channels
      // 4.2, backward (which is short of registers with 128) 3.5 and 4.0
      consider(kWide, 1.0);
      consider(kHalf, i ? 0.9 : 0.8);
    }
    if (!row && (d.inner <= 4 || best == 0.0)) consider(kNarrow, 1.0);
    const long blocks = std::max(recur_blocks(d, p->layout[i]), 1L);
    most_threads = std::max(most_threads, blocks * p->waves[i] * kWave);
  }
  if (most_threads >= 1LL << 32) {  // (a launch has fewer)
    delete p;
    return BL_ERR_UNSUPPORTED;
  }
  // a state at every tile of the backward pass
  p->every = (row ? kWave : p->layout[1] == kNarrow ? 16 : 4) * recur_each(p->layout[1], dtype_bytes(d.dtype), true) * p->waves[1];
  const size_t parts = std::max(p->chunks[0], p->chunks[1]);
  p->bytes = parts > 1 ? (parts + 1) * ((size_t)d.outer * d.inner * 8 + d.outer) : 0;
  *out = p;
  return BL_OK;
}

extern "C" bl_status_t bl_recurrence_plan_destroy(bl_recurrence_plan_t p) {
  if (!p) return BL_ERR_INVALID_ARG;
  delete p;
  return BL_OK;
}

extern "C" bl_status_t bl_recurrence_workspace_size(bl_recurrence_plan_t p, size_t* bytes) {
  if (!p || !bytes) return BL_ERR_INVALID_ARG;
  *bytes = p->bytes;
  return BL_OK;
}

extern "C" bl_status_t bl_recurrence_states_size(bl_recurrence_plan_t p, long long* elements) {
  if (!p || !elements) return BL_ERR_INVALID_ARG;
  *elements = (p->d.length + p->every - 1) / p->every * p->d.outer * p->d.inner;
  return BL_OK;
}

extern "C" bl_status_t bl_recurrence_forward(bl_recurrence_plan_t p, const void* gate, const void* x,
                                             const unsigned char* resets, const float* h0, void* y, float* last,
                                             float* states, void* ws, void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  const bl_recurrence_desc_t& d = p->d;
  if (!d.outer) return BL_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!d.length) return recur_none(h0, last, d.outer * d.inner, s);
  if (!gate || !x || !y || (p->bytes && (!ws || !aligned(ws)))) return BL_ERR_INVALID_ARG;
  RecurArgs r = args_of(p, ws);
  r.gate = gate;
  r.x = x;
  r.resets = resets;
  r.h0 = h0;
  r.y = y;
  r.last = last;
  r.states = states;
  if (d.dtype == BL_F32) return forward<float>(p, r, s);
  if (d.dtype == BL_BF16) return forward<bf16_t>(p, r, s);
  return forward<f16_t>(p, r, s);
}

extern "C" bl_status_t bl_recurrence_backward(bl_recurrence_plan_t p, const void* gate, const void* x,
                                              const unsigned char* resets, const float* states, const void* dy,
                                              const float* dlast, void* dgate, void* dx, float* dh0, void* ws,
                                              void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  const bl_recurrence_desc_t& d = p->d;
  if (!d.outer) return BL_OK;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!d.length) return recur_none(dlast, dh0, d.outer * d.inner, s);
  if (!gate || !x || !states || !dy || !dgate || !dx || (p->bytes && (!ws || !aligned(ws)))) return BL_ERR_INVALID_ARG;
  RecurArgs r = args_of(p, ws);
  r.gate = gate;
  r.x = x;
  r.resets = resets;
  r.states = const_cast<float*>(states);
  r.dy = dy;
  r.dlast = dlast;
  r.dgate = dgate;
  r.dx = dx;
  r.dh0 = dh0;
  return recur_backward(p, r, s);
}
