// Orthogonalised update of many matrices: plan, momentum, norms and the order of launches.
//
// A launch takes momentum and squares of slabs of 4096 elements, a second divides by the
// norm and lays the matrices out for the products, and three launches a Newton-Schulz step
// (muon_gemm.hip) follow, the last of which writes the parameters.  The matrices of a
// launch are part of its arguments, so that nothing is copied to the device beforehand and
// a captured step replays.
#include <algorithm>
#include <cmath>
#include <new>

#include "muon.hpp"

namespace blc {
namespace {

// u of element e (of a matrix whose momentum lies at m, or null).
template <typename G>
__device__ __forceinline__ float update_of(const G* g, const float* m, size_t e, float gs, const MuonArgs& a) {
  const float v = gs * to_f32(g[e]);
  if (!m) return v;
  return a.nesterov ? fmaf(a.beta, m[e], v) : m[e];
}

// The new momentum of a slab, and the sum of its u's squares in double precision (which
// holds the squares of all fp32 values).
template <typename G>
__global__ __launch_bounds__(kThreads) void k_muon_momentum(MuonList list, MuonArgs a) {
  __shared__ double red[kThreads / kWave];
  const unsigned at = muon_find(list.first, list.count, blockIdx.x);
  const MuonItem& it = list.item[at];
  const size_t size = (size_t)it.rows * it.cols, from = (size_t)(blockIdx.x - list.first[at]) * kMuonSlab;
  const size_t end = min(size, from + kMuonSlab);
  const G* g = static_cast<const G*>(it.g);
  float* m = a.momentum ? a.momentum + it.start : nullptr;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  double sum = 0.0;
  for (size_t e = from + threadIdx.x; e < end; e += kThreads) {
    if (m) m[e] = fmaf(a.beta, m[e], gs * to_f32(g[e]));
    const double u = update_of(g, m, e, gs, a);
    sum += u * u;
  }
  for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = sum;
  __syncthreads();
  if (threadIdx.x) return;
  sum = 0.0;
  for (int w = 0; w < kThreads / kWave; ++w) sum += red[w];
  a.squares[blockIdx.x] = sum;
}

// X and its transpose: a block takes 32 x 32 elements.  `slab`: first slab of each matrix.
struct MuonSlabs {
  unsigned first[kMuonList + 1];
};
constexpr int kLay = 32;
template <typename G>
__global__ __launch_bounds__(kThreads) void k_muon_lay(MuonList list, MuonSlabs slabs, MuonArgs a) {
  __shared__ double red[kThreads / kWave];
  __shared__ float tile[kLay][kLay + 1];
  const unsigned at = muon_find(list.first, list.count, blockIdx.x);
  const MuonItem& it = list.item[at];
  double sum = 0.0;
  for (unsigned k = slabs.first[at] + threadIdx.x; k < slabs.first[at + 1]; k += kThreads) sum += a.squares[k];
  for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
  if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < kThreads / kWave; ++w) sum += red[w];
  // (what is not finite makes all of the matrix NaN)
  const double inv = sum < (double)INFINITY ? 1.0 / (sqrt(sum) + a.eps) : (double)NAN;
  const G* g = static_cast<const G*>(it.g);
  const float* m = a.momentum ? a.momentum + it.start : nullptr;
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  // the matrix as it lies in memory, padded: rows by cols, of which the longer is n
  const unsigned across = (it.tall ? it.m : it.n) * (kMuonTile / kLay), block = blockIdx.x - list.first[at];
  const int r0 = (int)(block / across) * kLay, c0 = (int)(block % across) * kLay;
  for (int k = threadIdx.x; k < kLay * kLay; k += kThreads) {
    const int r = r0 + k / kLay, c = c0 + k % kLay;
    float v = 0.f;
    if (r < it.rows && c < it.cols)
      v = (float)((double)update_of(g, m, (size_t)r * it.cols + c, gs, a) * inv) * kHoldX;
    tile[k / kLay][k % kLay] = v;
  }
  __syncthreads();
  const MuonPlaces w = muon_places(it.m, it.n);
  char* part = a.ws + (size_t)it.off * 256;
  // as it lies, and its transpose: X and t[0] or, tall, the other way round
  const size_t mm = (size_t)it.m * kMuonTile * 4, nn = (size_t)it.n * kMuonTile * 4;
  f16_t* as = reinterpret_cast<f16_t*>(part + (it.tall ? w.t0 : w.x));
  f16_t* turned = reinterpret_cast<f16_t*>(part + (it.tall ? w.x : w.t0));
  const size_t as_row = (it.tall ? mm : nn) / 2, turned_row = (it.tall ? nn : mm) / 2;
  for (int k = threadIdx.x; k < kLay * kLay; k += kThreads) {
    const int i = k / kLay, j = k % kLay;
    const float v = tile[i][j], t = tile[j][i];
    const f16_t vh = (f16_t)v, th = (f16_t)t;
    // 32 values of a row: their high parts, then their low ones
    f16_t* pv = as + (size_t)(r0 + i) * as_row + (size_t)c0 * 2 + j;
    f16_t* pt = turned + (size_t)(c0 + i) * turned_row + (size_t)r0 * 2 + j;
    pv[0] = vh;
    pv[32] = (f16_t)(v - (float)vh);
    pt[0] = th;
    pt[32] = (f16_t)(t - (float)th);
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
      it.m = shapes.m[k] = (unsigned short)((m + kMuonTile - 1) / kMuonTile);
      it.n = shapes.n[k] = (unsigned short)((n + kMuonTile - 1) / kMuonTile);
      gram += 3.0 * m * m * n;
      poly += 3.0 * m * m * m;
      apply += 6.0 * m * m * n;
      values += (double)m * n;
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
    blocks = lay(list.first, [&](int k) { return (unsigned)list.item[k].m * list.item[k].n * 16; });
    st = timed_launch("muon_lay", values * 16.0, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
      typed([&](auto g) {
        hipExtLaunchKernelGGL(k_muon_lay<decltype(g)>, dim3(blocks), dim3(kThreads), 0, s, e0, e1, 0, list, slabs, a);
      });
    });
    for (size_t k = 0; st == BL_OK && k < p->steps.size(); ++k) {
      const auto& step = p->steps[k];
      MuonProduct q{};
      q.ws = a.ws;
      q.turn = (int)(k % 2);
      q.scale = kHoldA / (kHoldX * kHoldX);
      blocks = lay(shapes.first, [&](int i) { return (unsigned)shapes.m[i] * (shapes.m[i] + 1) / 2; });
      st = muon_product(kGram, shapes, blocks, gram, q, s);
      if (st != BL_OK) return st;
      q.a = (float)(step.a * step.scale_b);
      q.b = (float)(step.b * step.scale_b / kHoldA);
      q.c = (float)(step.c * step.scale_b / ((double)kHoldA * kHoldA));
      st = muon_product(kPoly, shapes, blocks, poly, q, s);
      if (st != BL_OK) return st;
      const bool last = k + 1 == p->steps.size();
      q.scale = 1.f / step.scale_b;  // (X keeps its power of two)
      if (last) {
        q.scale /= kHoldX;
        blocks = lay(list.first, [&](int i) { return (unsigned)shapes.m[i] * shapes.n[i]; });
        st = muon_update(p->param_dtype, list, blocks, apply, q, a, s);
      } else {
        blocks = lay(shapes.first, [&](int i) { return (unsigned)shapes.m[i] * shapes.n[i]; });
        st = muon_product(kApply, shapes, blocks, apply, q, s);
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
      // the largest power of two that keeps B below fp16's largest value, up to 2^14
      p->steps.push_back({c[0], c[1], c[2], (float)std::exp2(std::min(14.0, std::floor(std::log2(60000.0 / poly))))});
    }
    for (int i = 0; i < d->count; ++i) {
      const long long r = d->rows[i], c = d->cols[i];
      const double scale = d->scale ? d->scale[i] : std::sqrt(std::max(1.0, c ? (double)r / (double)c : 1.0));
      p->matrices.push_back({r, c, p->total, scale, (unsigned char)(!d->decay || d->decay[i])});
      p->total += (r * c + 63) / 64 * 64;
      if (!r || !c) continue;
      const unsigned m = (unsigned)((std::min(r, c) + kMuonTile - 1) / kMuonTile);
      const unsigned n = (unsigned)((std::max(r, c) + kMuonTile - 1) / kMuonTile);
      if (p->batches.empty() || p->batches.back().of.size() == kMuonList ||
          p->batches.back().bytes + muon_places(m, n).bytes > kMuonBytes)
        p->batches.emplace_back();
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
