// Layer norm over the middle axis of [outer][size][inner]: plan, dispatch and
// the last sum of the weights' gradients.
#include <cmath>
#include <new>

#include "norm.hpp"

namespace blc {
namespace {

// Sums of partial rows part[parts][2 size] by columns: 64 columns and SLICES slices
// of the rows a block, each slice in order with four loads in flight, then the
// slices in order.  (One thread a column would wait for many parts in turn; few
// parts leave slices without work: 10 parts of 200704 columns 14 us with 16 slices, 4
// with one.)  512 parts of 2048 columns take 4 us.
constexpr int kCols = 64;
constexpr long long kMostColumns = 64LL * ((1LL << 26) - 1);  // a launch has fewer than 2^32 threads
template <typename T, int SLICES>
__global__ __launch_bounds__(kCols* SLICES) void k_norm_sum(const float* part, int parts, long size, void* dw,
                                                            void* db, bool wide) {
  __shared__ float red[SLICES][kCols];
  const int col = threadIdx.x % kCols, slice = threadIdx.x / kCols;
  const long n = 2 * size, c = (long)blockIdx.x * kCols + col;
  float acc[4] = {};
  if (c < n) {
    int r = slice;
    for (; r + 3 * SLICES < parts; r += 4 * SLICES) {
      float v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = part[(size_t)(r + k * SLICES) * n + c];
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[k] += v[k];
    }
    for (int k = 0; r < parts; r += SLICES, ++k) acc[k] += part[(size_t)r * n + c];
  }
  float sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
  if (SLICES > 1) {
    red[slice][col] = sum;
    __syncthreads();
    if (slice) return;
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < SLICES; ++k) sum += red[k][col];
  }
  if (c >= n) return;
  void* out = c < size ? dw : db;
  const long i = c < size ? c : c - size;
  if (!out) return;
  if (wide) static_cast<float*>(out)[i] = sum;
  else static_cast<T*>(out)[i] = (T)sum;
}

}  // namespace

bl_status_t norm_sum_parts(const bl_norm_plan_s* p, const NormPtrs& a, int parts, hipStream_t s) {
  if (!a.dw && !a.db) return BL_OK;
  const unsigned blocks = (unsigned)((2 * p->d.size + kCols - 1) / kCols);
  const bool wide = p->d.wdtype == BL_F32, few = parts <= 16;
  return timed_launch("norm_sum", 8.0 * parts * p->d.size, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    auto go = [&](auto kernel, int slices) {
      hipExtLaunchKernelGGL(kernel, dim3(blocks), dim3(kCols * slices), 0, s, e0, e1, 0, a.part, parts,
                            (long)p->d.size, a.dw, a.db, wide);
    };
    if (p->d.dtype == BL_F16) few ? go(k_norm_sum<f16_t, 1>, 1) : go(k_norm_sum<f16_t, 16>, 16);
    else few ? go(k_norm_sum<bf16_t, 1>, 1) : go(k_norm_sum<bf16_t, 16>, 16);
  });
}

}  // namespace blc

using namespace blc;

extern "C" bl_status_t bl_norm_plan_create(bl_norm_plan_t* out, const bl_norm_desc_t* desc) {
  if (!out || !desc) return BL_ERR_INVALID_ARG;
  *out = nullptr;
  bl_norm_desc_t d = *desc;
  if (d.outer < 0 || d.size < 1 || d.inner < 1 || !known_dtype(d.dtype)) return BL_ERR_INVALID_ARG;
  if (d.wdtype != BL_F32 && d.wdtype != d.dtype) return BL_ERR_INVALID_ARG;
  if (!(d.eps >= 0.0) || !std::isfinite(d.eps)) return BL_ERR_INVALID_ARG;
  if (d.x_stride < 0 || d.y_stride < 0) return BL_ERR_INVALID_ARG;
  const long long most = (1LL << 31) - 1;
  if (d.size > most || d.inner > most || d.size * d.inner > most) return BL_ERR_UNSUPPORTED;
  if (2 * d.size > kMostColumns) return BL_ERR_UNSUPPORTED;  // (one thread a column of dw and db: few parts)
  if (d.outer > most || d.outer * d.inner > most) return BL_ERR_UNSUPPORTED;
  if (!d.x_stride) d.x_stride = d.size * d.inner;
  if (!d.y_stride) d.y_stride = d.size * d.inner;
  if (d.outer > 1 && (d.x_stride < d.size * d.inner || d.y_stride < d.size * d.inner)) return BL_ERR_INVALID_ARG;
  bl_norm_plan_s* p = new (std::nothrow) bl_norm_plan_s{};
  if (!p) return BL_ERR_OOM;
  p->d = d;
  const bl_status_t st = !d.outer ? BL_OK : d.inner == 1 ? norm_rows_plan(p) : norm_maps_plan(p);
  if (st != BL_OK) {
    delete p;
    return st;
  }
  *out = p;
  return BL_OK;
}

extern "C" bl_status_t bl_norm_plan_destroy(bl_norm_plan_t p) {
  if (!p) return BL_ERR_INVALID_ARG;
  delete p;
  return BL_OK;
}

extern "C" bl_status_t bl_norm_workspace_size(bl_norm_plan_t p, size_t* bytes) {
  if (!p || !bytes) return BL_ERR_INVALID_ARG;
  *bytes = p->bytes;
  return BL_OK;
}

extern "C" bl_status_t bl_norm_forward(bl_norm_plan_t p, const void* x, const void* w, const void* b, void* y,
                                       float* stats, void* ws, void* stream) {
  if (!p || (p->d.outer && (!x || !y || (p->bytes && (!ws || !aligned(ws)))))) return BL_ERR_INVALID_ARG;
  if (!p->d.outer) return BL_OK;
  NormPtrs a{};
  a.x = x;
  a.w = w;
  a.b = b;
  a.y = y;
  a.stats = stats;
  a.sums = reinterpret_cast<float*>(static_cast<char*>(ws) + p->off_sums);
  hipStream_t s = static_cast<hipStream_t>(stream);
  return p->d.inner == 1 ? norm_rows_forward(p, a, s) : norm_maps_forward(p, a, s);
}

extern "C" bl_status_t bl_norm_backward(bl_norm_plan_t p, const void* dy, const void* x, const void* w,
                                        const float* stats, void* dx, void* dw, void* db, void* ws, void* stream) {
  if (!p || (p->d.outer && (!dy || !x || !stats || !dx || (p->bytes && (!ws || !aligned(ws)))))) return BL_ERR_INVALID_ARG;
  NormPtrs a{};
  a.x = x;
  a.dy = dy;
  a.w = w;
  a.dx = dx;
  a.dw = dw;
  a.db = db;
  a.stats = const_cast<float*>(stats);
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + p->off_part);
  a.sums = reinterpret_cast<float*>(static_cast<char*>(ws) + p->off_sums);
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!p->d.outer) return norm_sum_parts(p, a, 0, s);
  return p->d.inner == 1 ? norm_rows_backward(p, a, s) : norm_maps_backward(p, a, s);
}
