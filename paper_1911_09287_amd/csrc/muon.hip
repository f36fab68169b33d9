// Orthogonalised update of many matrices: plan, momentum, norms and the order of launches.
//
// A launch takes momentum and squares of slabs of 4096 elements, a second divides by the
// norm and lays the matrices out for the products (muon_gemm.hip), the last of which writes
// the parameters.  The matrices of a launch are part of its arguments, so that nothing is
// copied to the device beforehand and a captured step replays.
//
// Steps may be joined: with A = X X^T, the next step's is B A B, so that a few steps need X
// only for the first A and for X = (... B2 B1) X, and square products in between, which are
// symmetric since all are polynomials of A.  Of m by 4 m that is 19 / 32 of the single steps'
// operations, of squares the same.  But what rounds in A grows by B B where B A B is formed
// and not from X: a joined run ends before its B's product may exceed 48 (three usual steps).
// Where a gradient has a few strong directions, five usual steps of 50 x 128 ... 256 x 640 in fp32
// are off by 0.9 to 1.8e-6 of the norm one by one, by 2.1 to 3.8e-6 in runs of three and two, by 1.5e-5 to
// 1e-4 in longer ones: and that only if the square matrices are symmetric to the last bit.
#include <algorithm>
#include <cmath>
#include <new>

#include "muon.hpp"

namespace blc {
namespace {

// Sum over a block, in each thread.
__device__ __forceinline__ double block_sum(double sum, double (&red)[kThreads / kWave]) {
  for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / kWave; ++w) sum += red[w];
  return sum;
}

// The new momentum of a slab, and the sum of its u's squares in double precision (which
// holds the squares of all fp32 values).  A thread's loads are all in flight together.
template <typename G>
__global__ __launch_bounds__(kThreads) void k_muon_momentum(MuonList list, MuonArgs a) {
  constexpr int kEach = kMuonSlab / kThreads / 4;
  __shared__ double red[kThreads / kWave];
  const unsigned at = muon_find(list.first, list.count, blockIdx.x);
  const MuonItem& it = list.item[at];
  const long size = (long)it.rows * it.cols, from = (long)(blockIdx.x - list.first[at]) * kMuonSlab + threadIdx.x * 4;
  const G* g = static_cast<const G*>(it.g) + from;
  float* m = a.momentum ? a.momentum + it.start + from : nullptr;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  Held<G, 4> gv[kEach];
  Held<float, 4> mv[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    gv[k].load(g + k * kThreads * 4, size - from - k * kThreads * 4);
    mv[k].load(m + k * kThreads * 4, m ? size - from - k * kThreads * 4 : 0);
  }
  double sum = 0.0;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    gv[k].refresh();
    mv[k].refresh();
    Pack<float, 4> next;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      next.v[j] = fmaf(a.beta, mv[k][j], gs * gv[k][j]);
      const double u = muon_update_of(gv[k][j], next.v[j], gs, a);  // (0 where there is none)
      sum = fma(u, u, sum);
    }
    if (m) store_part(m + k * kThreads * 4, size - from - k * kThreads * 4, next);
  }
  sum = block_sum(sum, red);
  if (threadIdx.x == 0) a.squares[blockIdx.x] = sum;
}

// X and its transpose: a block takes 64 x 64 elements of a matrix as it lies in memory.
struct MuonSlabs {
  unsigned first[kMuonList + 1];  // first slab of each matrix
};
constexpr int kLayRow = kMuonPad + 1;
// Eight values of the tile, `step` apart, as high and low parts of a row of the layout.
__device__ __forceinline__ void lay_eight(const float* v, int step, char* row, int c) {
  Pack<f16_t, 8> hi, lo;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float x = v[j * step];
    hi.v[j] = (f16_t)x;
    lo.v[j] = (f16_t)(x - (float)hi.v[j]);
  }
  f16_t* to = reinterpret_cast<f16_t*>(row + c / 32 * 128 + c % 32 * 2);
  store_pack(to, hi);
  store_pack(to + 32, lo);
}
template <typename G>
__global__ __launch_bounds__(kThreads) void k_muon_lay(MuonList list, MuonSlabs slabs, MuonArgs a) {
  constexpr int kEach = kMuonPad * kMuonPad / 4 / kThreads;
  __shared__ double red[kThreads / kWave];
  __shared__ float tile[kMuonPad * kLayRow];
  const unsigned at = muon_find(list.first, list.count, blockIdx.x);
  const MuonItem& it = list.item[at];
  const unsigned across = it.tall ? it.m : it.n, block = blockIdx.x - list.first[at];
  const int r0 = (int)(block / across) * kMuonPad, c0 = (int)(block % across) * kMuonPad, cols = it.cols;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  const int c = c0 + threadIdx.x % 16 * 4;
  Held<G, 4> gv[kEach];
  Held<float, 4> mv[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int r = r0 + k * 16 + threadIdx.x / 16;
    const long e = (long)r * cols + c, n = r < it.rows ? cols - c : 0;
    gv[k].load(static_cast<const G*>(it.g) + e, n);
    mv[k].load(a.momentum + it.start + e, a.momentum ? n : 0);
  }
  double sum = 0.0;
  for (unsigned k = slabs.first[at] + threadIdx.x; k < slabs.first[at + 1]; k += kThreads) sum += a.squares[k];
  sum = block_sum(sum, red);
  const double inv = muon_inverse(sum, a.eps);
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    gv[k].refresh();
    mv[k].refresh();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = k * 16 + threadIdx.x / 16;
      const bool there = r0 + r < it.rows && c + j < cols;
      tile[r * kLayRow + threadIdx.x % 16 * 4 + j] = there ? (float)((double)muon_update_of(gv[k][j], mv[k][j], gs, a) * inv) : 0.f;
    }
  }
  __syncthreads();
  const MuonPlaces w = muon_places(it.m, it.n);
  char* part = a.ws + (size_t)it.off * 256;
  // as it lies, and its transpose: X and t0 or, tall, the other way round
  const size_t mm = muon_row(it.m), nn = muon_row(it.n), as_row = it.tall ? mm : nn, turned_row = it.tall ? nn : mm;
  char* as = part + (it.tall ? w.t0 : w.x) + r0 * as_row + c0 * 4;
  char* turned = part + (it.tall ? w.x : w.t0) + c0 * turned_row + r0 * 4;
#pragma unroll
  for (int k = 0; k < kMuonPad * kMuonPad / 8 / kThreads; ++k) {
    const int i = k * (kThreads / 8) + threadIdx.x / 8, j = threadIdx.x % 8 * 8;
    lay_eight(tile + i * kLayRow + j, 1, as + i * as_row, j);
    lay_eight(tile + j * kLayRow + i, kLayRow, turned + i * turned_row, j);
  }
}

// Largest |a + b y + c y^2| over 0 ... y, and of t times that with y = t^2 over 0 ... t.
double most_of_poly(double a, double b, double c, double y) {
  double most = std::max(std::fabs(a), std::fabs(a + (b + c * y) * y));
  const double turn = c != 0.0 ? -b / (2.0 * c) : -1.0;
  if (turn > 0.0 && turn < y) most = std::max(most, std::fabs(a + (b + c * turn) * turn));
  return most;
}
double most_of_step(double a, double b, double c, double t) {
  auto at = [&](double x) { return std::fabs(x * (a + (b + c * x * x) * x * x)); };
  double most = at(t);
  // where its derivative a + 3 b y + 5 c y^2 is 0
  const double qa = 5.0 * c, qb = 3.0 * b, root = qb * qb - 4.0 * qa * a;
  double y[2] = {-1.0, -1.0};
  if (qa == 0.0) y[0] = qb != 0.0 ? -a / qb : -1.0;
  else if (root >= 0.0) y[0] = (-qb + std::sqrt(root)) / (2.0 * qa), y[1] = (-qb - std::sqrt(root)) / (2.0 * qa);
  for (double v : y)
    if (v > 0.0 && v < t * t) most = std::max(most, at(std::sqrt(v)));
  return most;
}

constexpr double kUsual[3] = {3.4445, -4.7750, 2.0315};
constexpr double kMostSingular = 1.75;
constexpr double kMostJoined = 48.0;  // of a joined run's B's product
// Tiles that a launch needs to go by larger ones.  One X = B X of 2048 x 2048 (256 tiles of 128)
// takes 78 us with 128-wide tiles, 95 with 64, 139 with 256; of 512 x 8192 28.9 with 128, 31.5 with
// 64; of 20 of 1024 x 4096 7 % less with 256 than with 128.  The lower 136 tiles of 128
// of one 2048 x 2048 gram take 72 us, its 528 of 64 only 58.
constexpr unsigned kFillSquare = 512, kFill128 = 256, kFill256 = 1024;

bl_status_t run(const bl_muon_plan_s* p, void* const* out, const void* const* grads, MuonArgs a, void* ws, hipStream_t s) {
  a.ws = static_cast<char*>(ws);
  a.squares = reinterpret_cast<double*>(a.ws + p->off_squares);
  MuonList list;
  MuonShapes shapes;
  MuonSlabs slabs;
  for (const auto& batch : p->batches) {
    const int count = (int)batch.of.size();
    double gram = 0.0, poly = 0.0, apply = 0.0, values = 0.0;
    list.count = shapes.count = count;
    for (int k = 0; k < count; ++k) {
      const auto& x = p->matrices[batch.of[k]];
      MuonItem& it = list.item[k];
      it.p = out[batch.of[k]];
      it.g = grads[batch.of[k]];
      it.start = x.start;
      it.rows = (int)x.rows;
      it.cols = (int)x.cols;
      it.scale = (float)x.scale;
      it.off = shapes.off[k] = batch.off[k];
      it.tall = x.rows > x.cols;
      it.decay = x.decay;
      const long long m = std::min(x.rows, x.cols), n = std::max(x.rows, x.cols);
      it.m = shapes.m[k] = (unsigned short)((m + kMuonPad - 1) / kMuonPad);
      it.n = shapes.n[k] = (unsigned short)((n + kMuonPad - 1) / kMuonPad);
      gram += 3.0 * m * m * n;
      poly += 3.0 * m * m * m;
      apply += 6.0 * m * m * n;
      values += (double)m * n;
    }
    if (p->small) {
      MuonSmallSteps small{};
      small.count = (int)p->joined.size();
      for (int k = 0; k < small.count; ++k) {
        const auto& step = p->joined[k];
        small.step[k] = {(float)(step.a * step.hold_b), (float)(step.b * step.hold_b / kHoldA),
                         (float)(step.c * step.hold_b / ((double)kHoldA * kHoldA)), step.hold_b, step.hold_q, step.first, step.last};
      }
      const bl_status_t st = muon_small(p->param_dtype, p->grad_dtype, list, small, a, 5.0 * (gram + poly + apply), s);
      if (st != BL_OK) return st;
      continue;
    }
    // first[] of a launch whose blocks of matrix k are blocks(k); how many there are
    auto lay = [&](unsigned* first, auto&& blocks) {
      unsigned n = 0;
      for (int k = 0; k <= kMuonList; ++k) {
        first[k] = n;
        if (k < count) n += (unsigned)blocks(k);
      }
      return n;
    };
    auto slab_count = [&](int k) { return ((long)list.item[k].rows * list.item[k].cols + kMuonSlab - 1) / kMuonSlab; };
    unsigned blocks = lay(list.first, slab_count);
    lay(slabs.first, slab_count);
    auto typed = [&](auto&& go) {
      if (p->grad_dtype == BL_F32) go(float());
      else if (p->grad_dtype == BL_BF16) go(bf16_t());
      else go(f16_t());
    };
    bl_status_t st = timed_launch("muon_momentum", values * 8.0, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      typed([&](auto g) {
        hipExtLaunchKernelGGL(k_muon_momentum<decltype(g)>, dim3(blocks), dim3(kThreads), 0, s, e0, e1, 0, list, a);
      });
    });
    if (st != BL_OK) return st;
    blocks = lay(list.first, [&](int k) { return (unsigned)list.item[k].m * list.item[k].n; });
    st = timed_launch("muon_lay", values * 16.0, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      typed([&](auto g) {
        hipExtLaunchKernelGGL(k_muon_lay<decltype(g)>, dim3(blocks), dim3(kThreads), 0, s, e0, e1, 0, list, slabs, a);
      });
    });
    auto triangle = [&](int side) {
      return lay(shapes.first, [&](int i) {
        const unsigned m = (shapes.m[i] * 64u + side - 1) / side;
        return m * (m + 1) / 2;
      });
    };
    auto all = [&](unsigned* first, int side) {
      return lay(first, [&](int i) {
        return (shapes.m[i] * 64u + side - 1) / side * ((shapes.n[i] * 64u + side - 1) / side);
      });
    };
    const int square_side = triangle(128) >= kFillSquare ? 128 : 64;
    const int apply_side = all(shapes.first, 256) >= kFill256 ? 256 : all(shapes.first, 128) >= kFill128 ? 128 : 64;
    const auto& steps = batch.joined ? p->joined : p->single;
    MuonProduct q{};
    q.ws = a.ws;
    q.q2 = -1;
    int product = kSlotB;  // of the joined steps
    for (size_t k = 0; st == BL_OK && k < steps.size(); ++k) {
      const auto& step = steps[k];
      const bool end = k + 1 == steps.size();
      auto go = [&](int mode, double flops) {
        if (st == BL_OK) st = muon_product(mode, square_side, shapes, blocks, flops, q, s);
      };
      blocks = triangle(square_side);
      if (step.first) {
        q.out = kSlotA;
        q.scale = kHoldA / (kHoldX * kHoldX);
        go(kGram, gram);
      }
      const int b = step.first && !step.last ? kSlotQ0 : kSlotB;
      q.p = kSlotA;
      q.out = b;
      q.a = (float)(step.a * step.hold_b);
      q.b = (float)(step.b * step.hold_b / kHoldA);
      q.c = (float)(step.c * step.hold_b / ((double)kHoldA * kHoldA));
      go(kPoly, poly);
      q.p = b;
      // the product so far times B, and A B, then B (A B)
      const int next = step.first ? b : product == kSlotQ0 ? kSlotQ1 : kSlotQ0;
      const float scale = step.first ? 0.f : step.hold_q / (step.hold_b * steps[k - 1].hold_q);
      if (!step.last) {
        q.q = kSlotA;
        q.out = kSlotAB;
        q.scale = 1.f / step.hold_b;
        q.q2 = step.first ? -1 : product;
        q.out2 = next;
        q.scale2 = scale;
        go(kSquare, q.q2 < 0 ? poly : 2.0 * poly);
        q.q = kSlotAB;
        q.out = kSlotA;
        q.q2 = -1;
        go(kSquare, poly);
      } else if (!step.first) {
        q.q = product;
        q.out = next;
        q.scale = scale;
        go(kSquare, poly);
      }
      product = next;
      if (!step.last || st != BL_OK) continue;
      q.p = product;
      q.scale = 1.f / step.hold_q;  // (X keeps its power of two)
      if (end) {
        q.scale /= kHoldX;
        blocks = all(list.first, apply_side);
        st = muon_update(p->param_dtype, apply_side, list, blocks, apply, q, a, s);
      } else {
        blocks = all(shapes.first, apply_side);
        st = muon_product(kApply, apply_side, shapes, blocks, apply, q, s);
        q.turn ^= 1;
      }
    }
    if (st != BL_OK) return st;
  }
  return BL_OK;
}

}  // namespace
}  // namespace blc

using namespace blc;

extern "C" bl_status_t bl_muon_plan_create(bl_muon_plan_t* out, const bl_muon_desc_t* d) {
  if (!out || !d) return BL_ERR_INVALID_ARG;
  *out = nullptr;
  if (d->count < 0 || (d->count && (!d->rows || !d->cols))) return BL_ERR_INVALID_ARG;
  if (d->param_dtype != BL_F32 && d->param_dtype != BL_BF16) return BL_ERR_INVALID_ARG;
  if (!known_dtype(d->grad_dtype) || d->steps < 1 || d->steps > kMuonSteps) return BL_ERR_INVALID_ARG;
  for (int i = 0; i < d->count; ++i) {
    if (d->rows[i] < 0 || d->cols[i] < 0) return BL_ERR_INVALID_ARG;
    if (d->scale && !std::isfinite(d->scale[i])) return BL_ERR_INVALID_ARG;
    if (!d->rows[i] || !d->cols[i]) continue;
    if (d->rows[i] > 65536 || d->cols[i] > 65536 || d->rows[i] * d->cols[i] >= 1LL << 31) return BL_ERR_UNSUPPORTED;
  }
  bl_muon_plan_s* p = new (std::nothrow) bl_muon_plan_s();
  if (!p) return BL_ERR_OOM;
  p->param_dtype = d->param_dtype;
  p->grad_dtype = d->grad_dtype;
  try {
    auto hold = [](double most) { return (float)std::exp2(std::min(14.0, std::floor(std::log2(60000.0 / most)))); };
    double most = 1.0;
    for (int k = 0; k < d->steps; ++k) {
      const double* c = d->coef ? d->coef + 3 * k : kUsual;
      bool good = std::isfinite(c[0]) && std::isfinite(c[1]) && std::isfinite(c[2]);
      const double poly = good ? most_of_poly(c[0], c[1], c[2], most * most) : 0.0;
      most = good ? most_of_step(c[0], c[1], c[2], most) : 0.0;
      if (!(good && most <= kMostSingular && poly > 0.0 && poly <= 1e4)) {
        delete p;
        return BL_ERR_INVALID_ARG;
      }
      p->single.push_back({c[0], c[1], c[2], hold(poly), poly, true, true, hold(poly)});
    }
    double run = 1.0;
    for (size_t k = 0; k < p->single.size(); ++k) {
      auto step = p->single[k];
      step.first = k == 0 || run * step.most_b > kMostJoined;
      if (step.first && k) p->joined.back().last = true;
      run = step.first ? step.most_b : run * step.most_b;
      step.last = k + 1 == p->single.size();
      step.hold_q = hold(run);
      p->joined.push_back(step);
    }
    std::vector<int> order;  // of those that are not empty: the longest sums first
    for (int i = 0; i < d->count; ++i) {
      const long long r = d->rows[i], c = d->cols[i];
      const double scale = d->scale ? d->scale[i] : std::sqrt(std::max(1.0, c ? (double)r / (double)c : 1.0));
      p->matrices.push_back({r, c, p->total, scale, (unsigned char)(!d->decay || d->decay[i])});
      p->total += (r * c + 63) / 64 * 64;
      if (r && c) order.push_back(i);
    }
    auto longer = [&](int i, int j) {
      const auto &x = p->matrices[i], &y = p->matrices[j];
      return std::max(x.rows, x.cols) > std::max(y.rows, y.cols);
    };
    std::stable_sort(order.begin(), order.end(), longer);
    auto sides = [&](int i, unsigned& m, unsigned& n) {
      const auto& x = p->matrices[i];
      m = (unsigned)((std::min(x.rows, x.cols) + kMuonPad - 1) / kMuonPad);
      n = (unsigned)((std::max(x.rows, x.cols) + kMuonPad - 1) / kMuonPad);
    };
    // joined steps for matrices at least twice as long as high, single ones for the others; where
    // either are too few to fill the GPU, what takes fewer operations for all
    double single = 0.0, joined = 0.0;
    unsigned long long tiles[2] = {0, 0};
    for (int i : order) {
      unsigned m, n;
      sides(i, m, n);
      const double runs = std::count_if(p->joined.begin(), p->joined.end(), [](auto& x) { return x.first; });
      const double count = (double)p->single.size(), mm = 0.5 * m * m;
      single += count * mm * (3.0 * n + m);
      joined += runs * mm * 3.0 * n + mm * m * (count + 3.0 * (count - runs));
      tiles[n >= 2 * m] += (unsigned long long)((m + 1) / 2) * ((m + 1) / 2 + 1) / 2;
    }
    p->small = true;
    for (int i : order) {
      const auto& x = p->matrices[i];
      p->small &= std::min(x.rows, x.cols) <= kSmallShort && std::max(x.rows, x.cols) <= kSmallLong;
    }
    const bool apart = tiles[0] >= kFillSquare && tiles[1] >= kFillSquare;
    if (apart)
      std::stable_partition(order.begin(), order.end(), [&](int i) {
        unsigned m, n;
        sides(i, m, n);
        return n >= 2 * m;
      });
    for (int i : order) {
      const long long r = d->rows[i], c = d->cols[i];
      unsigned m, n;
      sides(i, m, n);
      const bool join = apart ? n >= 2 * m : joined < single;
      if (p->batches.empty() || p->batches.back().of.size() == kMuonList || p->batches.back().joined != join ||
          p->batches.back().bytes + muon_places(m, n).bytes > kMuonBytes) {
        p->batches.emplace_back();
        p->batches.back().joined = join;
      }
      auto& b = p->batches.back();
      b.of.push_back(i);
      b.off.push_back((unsigned)(b.bytes / 256));
      b.bytes += muon_places(m, n).bytes;
      b.slabs += (r * c + kMuonSlab - 1) / kMuonSlab;
    }
  } catch (const std::bad_alloc&) {
    delete p;
    return BL_ERR_OOM;
  }
  long slabs = 0;
  for (const auto& b : p->batches) {
    p->off_squares = std::max(p->off_squares, b.bytes);
    slabs = std::max(slabs, b.slabs);
  }
  p->bytes = p->off_squares + (size_t)slabs * sizeof(double);
  *out = p;
  return BL_OK;
}

extern "C" bl_status_t bl_muon_plan_destroy(bl_muon_plan_t p) {
  if (!p) return BL_ERR_INVALID_ARG;
  delete p;
  return BL_OK;
}

extern "C" bl_status_t bl_muon_state_size(bl_muon_plan_t p, size_t* bytes, long long* total, long long* start) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (bytes) *bytes = (size_t)p->total * sizeof(float);
  if (total) *total = p->total;
  if (start)
    for (size_t i = 0; i < p->matrices.size(); ++i) start[i] = p->matrices[i].start;
  return BL_OK;
}

extern "C" bl_status_t bl_muon_workspace_size(bl_muon_plan_t p, size_t* bytes) {
  if (!p || !bytes) return BL_ERR_INVALID_ARG;
  *bytes = p->bytes;
  return BL_OK;
}

namespace {
bool whole(const bl_muon_plan_s* p, void* const* out, const void* const* grads, void* ws) {
  if (!out || !grads || !ws || !aligned(ws)) return false;
  for (size_t i = 0; i < p->matrices.size(); ++i)
    if (p->matrices[i].rows && p->matrices[i].cols && (!out[i] || !grads[i])) return false;
  return true;
}
}  // namespace

extern "C" bl_status_t bl_muon_step(bl_muon_plan_t p, void* const* params, const void* const* grads, void* state,
                                    void* ws, const bl_muon_args_t* args, void* stream) {
  if (!p || !args) return BL_ERR_INVALID_ARG;
  const bl_muon_args_t& r = *args;
  if (!(r.momentum >= 0.0 && r.momentum < 1.0) || !(r.eps > 0.0) || !std::isfinite(r.eps)) return BL_ERR_INVALID_ARG;
  if (!(r.weight_decay >= 0.0) || !std::isfinite(r.weight_decay)) return BL_ERR_INVALID_ARG;
  if (!r.live && (!(r.lr >= 0.0) || !std::isfinite(r.lr) || r.step < 1)) return BL_ERR_INVALID_ARG;
  if (p->batches.empty()) return BL_OK;
  if (!whole(p, params, grads, ws) || !state || !aligned(state)) return BL_ERR_INVALID_ARG;
  MuonArgs a{};
  a.momentum = static_cast<float*>(state);
  a.grad_scale = r.grad_scale;
  a.live = r.live;
  a.lr = r.lr;
  a.wd = r.weight_decay;
  a.eps = r.eps;
  a.beta = (float)r.momentum;
  a.nesterov = r.nesterov;
  a.seed = r.seed;
  a.key = r.seed * 0x6A09E667u + (unsigned)r.step * 0xBB67AE85u;
  return run(p, params, grads, a, ws, static_cast<hipStream_t>(stream));
}

extern "C" bl_status_t bl_muon_orthogonalize(bl_muon_plan_t p, void* const* out, const void* const* grads, void* ws,
                                             double eps, void* stream) {
  if (!p || !(eps > 0.0) || !std::isfinite(eps)) return BL_ERR_INVALID_ARG;
  if (p->batches.empty()) return BL_OK;
  if (!whole(p, out, grads, ws)) return BL_ERR_INVALID_ARG;
  MuonArgs a{};
  a.eps = eps;
  a.set = 1;
  return run(p, out, grads, a, ws, static_cast<hipStream_t>(stream));
}
