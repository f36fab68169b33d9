// Group norm with an activation: plan, dispatch and the joins of partial sums.
//
// Statistics span a sample's sites, and a group's channels may be one of 16 bits or all:
// blocks take all channels of some sites (channels last) or sites of some channels (first),
// leave what each channel gives there, and a launch of a wave a group joins it (or, where it is
// little, every block that needs it for itself); a further launch applies the result.  So x (backward: x and dy) is read twice, which memory bounds.  Where
// a block's registers can hold whole groups of a sample they are read once, by one launch.
//
// Kernels' times, bf16 (bytes as moved, with the second reading): 128 x 3136 x 64 channels last
// forward 13.7 + 20.3 us, 154 MB; 32 x 3136 x 256 backward 31.2 + 4.9 + 28.4 us, 257
// MB; in one launch fp32 channels first 64 x 256 x 512 backward 27.8 us, 101 MB, and 4.5 for the
// weights' gradients.
#include <algorithm>
#include <cmath>
#include <new>

#include "gnorm.hpp"

namespace blc {
namespace {

// Entry i of a group's parts: chunk i / each of the channel i % each, and its sites.
__device__ __forceinline__ const float* part_at(const GroupNormArgs& a, long n, long g, unsigned i, float& sites) {
  const unsigned k = i / (unsigned)a.each, c = i - k * (unsigned)a.each;
  sites = (float)min(a.chunk, a.sites - (long)k * a.chunk);
  return a.part + (((n * a.chunks + k) * a.channels) + g * a.each + c) * 2;
}

// A wave a group, or a block (WAVES 4) where the parts are many: the mean of the parts' means,
// then the squares about it.
template <int WAVES>
__global__ __launch_bounds__(kThreads) void k_gnorm_join_fwd(GroupNormArgs a) {
  __shared__ float red[2][kThreads / kWave];
  const long q = WAVES > 1 ? (long)blockIdx.x : (long)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;
  if (q >= a.batch * a.groups) return;
  const long n = q / a.groups, g = q - n * a.groups;
  const unsigned entries = (unsigned)(a.each * a.chunks), first = threadIdx.x % (WAVES * kWave);
  const float size = (float)a.sites * (float)a.each;
  float sum = 0.f, m2 = 0.f;
#pragma unroll 4
  for (unsigned i = first; i < entries; i += WAVES * kWave) {
    float sites;
    const float* v = part_at(a, n, g, i, sites);
    sum = fmaf(sites, v[0], sum);
  }
  const float mean = (WAVES > 1 ? block_sum(sum, red[0]) : wave_sum(sum)) / size;
#pragma unroll 4
  for (unsigned i = first; i < entries; i += WAVES * kWave) {
    float sites;
    const float* v = part_at(a, n, g, i, sites);
    const float d = v[0] - mean;
    m2 += fmaf(sites * d, d, v[1]);
  }
  m2 = WAVES > 1 ? block_sum(m2, red[1]) : wave_sum(m2);
  if (first) return;
  a.stats[q] = mean;
  a.stats[a.batch * a.groups + q] = 1.f / sqrtf(m2 / size + a.eps);
}

// A wave a group: the sums of each channel over the sample, and the group's means of u = dz w
// and of u h.  Every product and sum rounds by itself, so that a group of one value, whose
// u is its mean, has a gradient of 0.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_gnorm_join_bwd(GroupNormArgs a) {
#pragma clang fp contract(off)
  const long q = (long)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;
  if (q >= a.batch * a.groups) return;
  const long n = q / a.groups, g = q - n * a.groups;
  const unsigned lane = threadIdx.x % kWave;
  // as many lanes on a channel as leave none idle
  unsigned on = kWave;
  while (on > 1 && on / 2 * (unsigned)a.each >= kWave) on /= 2;
  float s1 = 0.f, s2 = 0.f;
  for (unsigned first = 0; first < (unsigned)a.each; first += kWave / on) {
    const unsigned c = first + lane / on;
    float sums[2] = {};
    if (c < (unsigned)a.each)
      gnorm_pairs_sum(a.part + (n * a.chunks * a.channels + g * a.each + c) * 2, a.channels * 2, lane % on, a.chunks, on,
                      a.chunks, sums);
    const float dz = wave_sum(sums[0], (int)on), dh = wave_sum(sums[1], (int)on);
    if (c < (unsigned)a.each && lane % on == 0) {
      const long at = g * a.each + c;
      a.own[(n * a.channels + at) * 2] = dz;
      a.own[(n * a.channels + at) * 2 + 1] = dh;
      const float w = weight_at<T>(a.w, a.wide, at, 1.f);
      s1 += w * dz;
      s2 += w * dh;
    }
  }
  s1 = wave_sum(s1);
  s2 = wave_sum(s2);
  if (lane) return;
  const float size = (float)a.sites * (float)a.each;
  a.sums[2 * q] = s1 / size;
  a.sums[2 * q + 1] = s2 / size;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_gnorm_weights(GroupNormArgs a) {
  gnorm_weights_block<T>(a, blockIdx.x);
}

// Block k + weights' blocks times slab: its channels' sums over a slab.
__global__ __launch_bounds__(kThreads) void k_gnorm_slabs(GroupNormArgs a, long slab) {
  const unsigned across = (unsigned)((a.channels + kWave - 1) / kWave), q = blockIdx.x / across;
  gnorm_rows_sum(a.own, a.channels, q * slab, min(a.own_rows, (q + 1) * slab), blockIdx.x - q * across,
                 [&](long c, float db, float dw) {
                   float* to = a.slabs + (q * a.channels + c) * 2;
                   to[0] = db;
                   to[1] = dw;
                 });
}

unsigned blocks_for(long n, long each) { return (unsigned)((n + each - 1) / each); }

GroupNormArgs args_of(const bl_group_norm_plan_s* p, void* ws) {
  GroupNormArgs a{};
  const bl_group_norm_desc_t& d = p->d;
  char* at = static_cast<char*>(ws);
  a.part = reinterpret_cast<float*>(at + p->off_part);
  a.sums = reinterpret_cast<float*>(at + p->off_sums);
  a.own = reinterpret_cast<float*>(at + p->off_own);
  a.slabs = reinterpret_cast<float*>(at + p->off_slabs);
  a.batch = a.own_rows = d.batch;
  a.sites = d.sites;
  a.channels = d.channels;
  a.groups = d.groups;
  a.each = p->each;
  a.x_stride = d.x_stride;
  a.y_stride = d.y_stride;
  a.chunk = p->chunk;
  a.chunks = p->chunks;
  a.lanes = p->lanes;
  a.tiles = p->tiles;
  a.wide = d.wdtype == BL_F32;
  a.eps = (float)d.eps;
  return a;
}

}  // namespace

bl_status_t gnorm_join_forward(const GroupNormArgs& a, hipStream_t s) {
  return timed_launch("gnorm_join", 8.0 * a.batch * a.chunks * a.channels, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    if (a.each * a.chunks > 8 * kWave && a.batch * a.groups < 4096)
      hipExtLaunchKernelGGL(k_gnorm_join_fwd<4>, dim3((unsigned)(a.batch * a.groups)), dim3(kThreads), 0, s, e0, e1, 0, a);
    else
      hipExtLaunchKernelGGL(k_gnorm_join_fwd<1>, dim3(blocks_for(a.batch * a.groups, kThreads / kWave)), dim3(kThreads), 0,
                            s, e0, e1, 0, a);
  });
}

bl_status_t gnorm_join_backward(const GroupNormArgs& a, int dtype, hipStream_t s) {
  return timed_launch("gnorm_join", 8.0 * a.batch * a.chunks * a.channels, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    const dim3 grid(blocks_for(a.batch * a.groups, kThreads / kWave));
    if (dtype == BL_F16) hipExtLaunchKernelGGL(k_gnorm_join_bwd<f16_t>, grid, dim3(kThreads), 0, s, e0, e1, 0, a);
    else hipExtLaunchKernelGGL(k_gnorm_join_bwd<bf16_t>, grid, dim3(kThreads), 0, s, e0, e1, 0, a);
  });
}

bl_status_t gnorm_weights(const GroupNormArgs& a, int dtype, hipStream_t s) {
  if (!a.dw && !a.db) return BL_OK;
  return timed_launch("gnorm_weights", 8.0 * a.batch * a.channels, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    const dim3 grid(gnorm_weights_blocks(a));
    if (dtype == BL_F16) hipExtLaunchKernelGGL(k_gnorm_weights<f16_t>, grid, dim3(kThreads), 0, s, e0, e1, 0, a);
    else hipExtLaunchKernelGGL(k_gnorm_weights<bf16_t>, grid, dim3(kThreads), 0, s, e0, e1, 0, a);
  });
}

bl_status_t gnorm_slabs(const bl_group_norm_plan_s* p, GroupNormArgs& a, hipStream_t s) {
  if (!p->slabs || (!a.dw && !a.db)) return BL_OK;
  const bl_status_t st = timed_launch("gnorm_slabs", 8.0 * a.batch * a.channels, 0.0, s, [&](hipEvent_t e0, hipEvent_t e1) {
    hipExtLaunchKernelGGL(k_gnorm_slabs, dim3(gnorm_weights_blocks(a) * (unsigned)p->slabs), dim3(kThreads), 0, s, e0, e1, 0,
                          a, p->slab);
  });
  a.own = a.slabs;
  a.own_rows = p->slabs;
  return st;
}

}  // namespace blc

using namespace blc;

extern "C" bl_status_t bl_group_norm_plan_create(bl_group_norm_plan_t* out, const bl_group_norm_desc_t* desc) {
  if (!out || !desc) return BL_ERR_INVALID_ARG;
  *out = nullptr;
  bl_group_norm_desc_t d = *desc;
  if (d.batch < 0 || d.sites < 1 || d.channels < 1 || d.groups < 1 || d.channels % d.groups) return BL_ERR_INVALID_ARG;
  if (!known_dtype(d.dtype) || (d.wdtype != BL_F32 && d.wdtype != d.dtype)) return BL_ERR_INVALID_ARG;
  if ((d.layout != BL_CHANNELS_LAST && d.layout != BL_CHANNELS_FIRST) || d.act < BL_ACT_NONE || d.act > BL_ACT_SILU)
    return BL_ERR_INVALID_ARG;
  if (!(d.eps >= 0.0) || !std::isfinite(d.eps) || d.x_stride < 0 || d.y_stride < 0) return BL_ERR_INVALID_ARG;
  const long long most = (1LL << 31) - 1;
  if (d.sites > most || d.channels > most || d.sites * d.channels > most) return BL_ERR_UNSUPPORTED;
  if (d.batch > most || d.batch * d.channels > most) return BL_ERR_UNSUPPORTED;
  const long long flat = d.sites * d.channels;
  if (!d.x_stride) d.x_stride = flat;
  if (!d.y_stride) d.y_stride = flat;
  if (d.batch > 1 && (d.x_stride < flat || d.y_stride < flat)) return BL_ERR_INVALID_ARG;
  if (d.x_stride > 1LL << 58 || d.y_stride > 1LL << 58) return BL_ERR_UNSUPPORTED;
  if (d.batch > 1 && std::max(d.x_stride, d.y_stride) > (1LL << 60) / d.batch) return BL_ERR_UNSUPPORTED;
  bl_group_norm_plan_s* p = new (std::nothrow) bl_group_norm_plan_s{};
  if (!p) return BL_ERR_OOM;
  p->d = d;
  p->each = d.channels / d.groups;
  const long most_vec = 16 / dtype_bytes(d.dtype);
  if (d.layout == BL_CHANNELS_LAST) {
    p->vec = (int)most_vec;
    while (d.channels % p->vec) p->vec /= 2;
    const long lanes = d.channels / p->vec;
    p->lanes = (int)std::min<long>(lanes, kThreads);
    p->tiles = (int)((lanes + kThreads - 1) / kThreads);
    const long slices = kThreads / p->lanes;
    // chunks of eight sites a thread at least, as many as bring 512 blocks onto the GPU (two a
    // compute unit; with 2048 the apply launches of 128 x 3136 x 64 forward and 32 x 3136 x 256
    // backward, bf16, take 23.1 and 33.4 us, not 20.5 and 28.3, the sums the same), and more
    // where accesses are narrow (182 x 7250 x 5 fp32 forward: 28 us with 512, 21 with 2048)
    const long fill = std::min(2048L, 512 * (most_vec / p->vec)), have = std::min<long>(d.batch * p->tiles, fill);
    const long blocks = std::max(1L, fill / std::max(1L, have));
    p->chunk = std::max<long>((d.sites + blocks - 1) / blocks, slices * 8);
  } else {
    p->vec = (int)most_vec;
    p->tiles = 1;
    // as many lanes of a wave as a channel's sites fill, or a block where they are more than
    // eight accesses of each (217 x 180 x 899 fp16: a block a channel 207 us, a wave 80)
    p->lanes = kWave;
    while (p->lanes > 1 && p->lanes / 2 * most_vec >= d.sites) p->lanes /= 2;
    if (d.sites > 8 * kWave * most_vec) p->lanes = kThreads;
    const long blocks = std::max(1L, 2048 / std::max<long>(1, std::min<long>(d.batch * d.channels, 2048)));
    p->chunk = p->lanes < kThreads ? d.sites
                                   : std::max<long>((d.sites + blocks - 1) / blocks, kThreads * most_vec * 4);
    p->chunk = (p->chunk + most_vec - 1) / most_vec * most_vec;
  }
  d.layout == BL_CHANNELS_LAST ? gnorm_last_whole(p) : gnorm_first_whole(p);
  // (few groups that are large go over more of the GPU in parts)
  const __int128 wholes = (__int128)d.batch * p->whole_tiles;
  for (int i = 0; i < 2; ++i)
    if (wholes >= 1LL << 22 || (wholes < 128 && p->whole_threads[i] > kThreads)) p->whole_threads[i] = 0;
  p->chunk = std::min<long>(p->chunk, d.sites);
  p->chunks = (int)((d.sites + p->chunk - 1) / p->chunk);
  p->joins[0] = d.layout == BL_CHANNELS_LAST && p->tiles == 1 && d.channels * p->chunks <= kMostJoined &&
                p->each * p->chunks <= kMostOfGroup;
  const long most_rows = kMostOwn * (kThreads / gnorm_rows_cols(d.channels));
  p->joins[1] = p->joins[0] && d.batch * p->chunks <= most_rows;
  if (!p->joins[1] && d.batch > most_rows) {
    p->slab = std::max<long>(most_rows / (kMostOwn / kLeastOwn), (d.batch + kMostSlabs - 1) / kMostSlabs);
    p->slabs = (d.batch + p->slab - 1) / p->slab;
  }
  const size_t groups = (size_t)d.batch * d.groups, channels = (size_t)d.batch * d.channels;
  p->off_part = 0;
  p->off_sums = round_up(channels * p->chunks * 8, 16);
  p->off_own = p->off_sums + round_up(groups * 8, 16);
  p->off_slabs = p->off_own + round_up(channels * 8, 16);
  p->bytes = d.batch ? p->off_slabs + (size_t)p->slabs * d.channels * 8 : 0;
  // a launch has fewer than 2^32 threads
  const __int128 blocks = d.layout == BL_CHANNELS_LAST
                              ? (__int128)d.batch * p->chunks * p->tiles
                              : ((__int128)d.batch * d.channels + kThreads / p->lanes - 1) / (kThreads / p->lanes) * p->chunks;
  const long sums = (d.channels + kWave - 1) / kWave;  // (blocks that sum the weights' gradients)
  if (blocks + sums >= 1LL << 24 || (__int128)d.batch * d.groups >= (1LL << 24) * 4 || (__int128)p->each * p->chunks >= 1LL << 31) {
    delete p;
    return BL_ERR_UNSUPPORTED;
  }
  *out = p;
  return BL_OK;
}

extern "C" bl_status_t bl_group_norm_plan_destroy(bl_group_norm_plan_t p) {
  if (!p) return BL_ERR_INVALID_ARG;
  delete p;
  return BL_OK;
}

extern "C" bl_status_t bl_group_norm_workspace_size(bl_group_norm_plan_t p, size_t* bytes) {
  if (!p || !bytes) return BL_ERR_INVALID_ARG;
  *bytes = p->bytes;
  return BL_OK;
}

extern "C" bl_status_t bl_group_norm_forward(bl_group_norm_plan_t p, const void* x, const void* w, const void* b, void* y,
                                             float* stats, void* ws, void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (!p->d.batch) return BL_OK;
  if (!x || !y || (p->bytes && (!ws || !aligned(ws)))) return BL_ERR_INVALID_ARG;
  GroupNormArgs a = args_of(p, ws);
  a.x = x;
  a.w = w;
  a.b = b;
  a.y = y;
  a.stats = stats ? stats : a.sums;  // (the backward call's sums are as many)
  hipStream_t s = static_cast<hipStream_t>(stream);
  return p->d.layout == BL_CHANNELS_LAST ? gnorm_last_forward(p, a, s) : gnorm_first_forward(p, a, s);
}

extern "C" bl_status_t bl_group_norm_backward(bl_group_norm_plan_t p, const void* dy, const void* x, const void* w,
                                              const void* b, const float* stats, void* dx, void* dw, void* db, void* ws,
                                              void* stream) {
  if (!p) return BL_ERR_INVALID_ARG;
  if (p->d.batch && (!dy || !x || !stats || !dx || (p->bytes && (!ws || !aligned(ws))))) return BL_ERR_INVALID_ARG;
  GroupNormArgs a = args_of(p, ws);
  a.x = x;
  a.dy = dy;
  a.w = w;
  a.b = b;
  a.stats = const_cast<float*>(stats);
  a.dx = dx;
  a.dw = dw;
  a.db = db;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (!p->d.batch) return gnorm_weights(a, p->d.dtype, s);
  return p->d.layout == BL_CHANNELS_LAST ? gnorm_last_backward(p, a, s) : gnorm_first_backward(p, a, s);
}
