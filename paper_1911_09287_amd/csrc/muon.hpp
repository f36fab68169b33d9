// Orthogonalised update: plan and launch arguments (muon.hip: plan, momentum, norms and
// dispatch; muon_gemm.hip: the Newton-Schulz products).
#pragma once

#include <vector>

#include "ops.hpp"

namespace blc {

constexpr int kMuonList = 64;   // matrices of a launch: their list is part of the kernel's arguments
constexpr int kMuonPad = 64;    // matrices are padded to multiples of it with zeros
constexpr int kMuonSlab = 4096;  // elements of a block that takes squares
constexpr int kMuonSteps = 16;
constexpr size_t kMuonBytes = 1ull << 36; // of a launch's matrices, which keeps its blocks far below 2^24

// A matrix of a launch.  m and n: its shorter and longer side in 64s; `tall`: it has
// more rows than columns and is taken by its transpose.
struct MuonItem {
  void* p;
  const void* g;
  long long start;  // in the momentum's layout
  int rows, cols;
  float scale;
  unsigned off;     // of its part of the workspace, in 256 bytes
  unsigned short m, n, tall, decay;
};

struct MuonList {
  int count;
  unsigned first[kMuonList + 1];  // blocks before each matrix's; past the last one all are the number of blocks
  MuonItem item[kMuonList];
};

// What the products alone need.
struct MuonShapes {
  int count;
  unsigned first[kMuonList + 1];  // (a launch of two products reads a product's number of blocks at its end)
  unsigned off[kMuonList];
  unsigned short m[kMuonList], n[kMuonList];
};

struct MuonArgs {
  char* ws;        // matrices' parts
  double* squares; // a sum of squares for each slab
  float* momentum; // null: u is the gradient
  const float* grad_scale;
  const double* live;
  double lr, wd, eps;
  float beta;
  int nesterov, set;  // set: the result is the parameter
  unsigned key, seed;
};

// A product's launch.  Square matrices [m][m] are kept in slots of a matrix's part.
struct MuonProduct {
  char* ws;
  int p, q, out;     // slots of the operands and the result (gram: out; poly: p, out; apply: p)
  float scale;       // of the accumulated sum
  int q2, out2;      // square: a second product p q2 in the same launch, or q2 < 0
  float scale2;
  float a, b, c;     // poly: of I, A and A A, with the powers of two
  int turn;          // apply: which of X's two transposes is read
};

// The steps of a launch that takes whole matrices (a, b, c as in a product's launch).
struct MuonSmallSteps {
  struct Step {
    float a, b, c, hold_b, hold_q;
    int first, last;
  };
  int count;
  Step step[kMuonSteps];
};
constexpr long long kSmallShort = 64, kSmallLong = 1024;  // sides of the matrices it takes

}  // namespace blc

struct bl_muon_plan_s {
  struct Matrix {
    long long rows, cols, start;
    double scale;
    unsigned char decay;
  };
  struct Step {
    double a, b, c;
    float hold_b;   // power of two that B is held with
    double most_b;  // its largest singular value's bound
    bool first, last;  // of the steps that X is multiplied by at once
    float hold_q;   // power of two that their product up to this step is held with
  };
  // Matrices that are taken together, by their numbers.
  struct Batch {
    std::vector<int> of;
    std::vector<unsigned> off;
    size_t bytes;
    long slabs;
    bool joined;  // by joined steps, not single ones
  };
  std::vector<Matrix> matrices;
  std::vector<Step> single, joined;
  bool small;  // a block takes a matrix
  std::vector<Batch> batches;
  int param_dtype, grad_dtype;
  long long total;
  size_t bytes, off_squares;
};

namespace blc {

// Values are held as two fp16 parts, high and low, 32 of a row's high parts and then their
// low ones side by side.  X is held times 2^15 (no singular value of it is above 1.75),
// A = X X^T and A B (no singular value above 1.75^2) times 2^14.
constexpr float kHoldX = 32768.f, kHoldA = 16384.f;
// Slots of square matrices: A, B, A B and the product of a few steps' B, in turn.
enum MuonSlot { kSlotA, kSlotB, kSlotAB, kSlotQ0, kSlotQ1, kSlots };

// Bytes of a row of n 64s.
__host__ __device__ inline size_t muon_row(unsigned n) { return (size_t)n * kMuonPad * 4; }
// Byte offsets in a matrix's part: X [m][n], its transpose twice and the slots [m][m].
struct MuonPlaces {
  size_t x, t0, t1, square, each, bytes;
  __host__ __device__ size_t t(int turn) const { return turn ? t1 : t0; }
  __host__ __device__ size_t slot(int s) const { return square + s * each; }
};
__host__ __device__ inline MuonPlaces muon_places(unsigned m, unsigned n) {
  const size_t x = (size_t)m * kMuonPad * muon_row(n), s = (size_t)m * kMuonPad * muon_row(m);
  return MuonPlaces{0, x, 2 * x, 3 * x, s, 3 * x + kSlots * s};
}

__device__ __forceinline__ unsigned muon_find(const unsigned* first, int count, unsigned block) {
  int lo = 0, hi = count;  // first[lo] <= block < first[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (first[mid] <= block) lo = mid;
    else hi = mid;
  }
  return (unsigned)lo;
}

// 16 bits that round a bfloat16 parameter, from the element's place (the AdamW step's hash).
__device__ __forceinline__ unsigned muon_dither(unsigned long long place, unsigned key) {
  unsigned x = (unsigned)place * 0x9E3779B9u + key;
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  x ^= x >> 16;
  return (x * 0x6A09E667u) >> 16;
}

// u of an element from its gradient and (new) momentum.
__device__ __forceinline__ float muon_update_of(float g, float m, float gs, const MuonArgs& a) {
  return !a.momentum ? gs * g : a.nesterov ? fmaf(a.beta, m, gs * g) : m;
}
// What u is multiplied by, from the sum of its squares: what is not finite makes all of the matrix NaN, and
// zeros stay zeros though 1 / eps may be infinite.
__device__ __forceinline__ double muon_inverse(double sum, double eps) {
  if (sum == 0.0) return 0.0;
  return (sum < (double)INFINITY ? 1.0 / (sqrt(sum) + eps) : (double)NAN) * kHoldX;
}
// The parameter from its old value and x of X, or x itself (set).
template <typename P>
__device__ __forceinline__ P muon_next(float old, float x, unsigned long long place, float keep, float rate, unsigned key,
                                       bool set) {
  if (set) return (P)x;
  const float next = fmaf(-rate, x, old * keep);
  if constexpr (sizeof(P) == 4) {
    return next;
  } else {
    const unsigned bits = __float_as_uint(next);
    const bool finite = (bits & 0x7F800000u) != 0x7F800000u;
    const unsigned up = finite ? bits + muon_dither(place, key) : bits | (next != next ? 0x400000u : 0u);
    return __builtin_bit_cast(bf16_t, (unsigned short)(up >> 16));
  }
}
template <typename P>
__device__ __forceinline__ void muon_put(P* p, size_t e, float x, unsigned long long start, float keep, float rate,
                                         unsigned key, bool set) {
  p[e] = muon_next<P>(set ? 0.f : to_f32(p[e]), x, start + e, keep, rate, key, set);
}

bl_status_t muon_small(int param_dtype, int grad_dtype, const MuonList& list, const MuonSmallSteps& steps,
                       const MuonArgs& a, double flops, hipStream_t s);

enum MuonMode { kGram, kPoly, kSquare, kApply };
// side: of the tiles, 64, 128 or 256 (256: not where the result is symmetric).
bl_status_t muon_product(int mode, int side, const MuonShapes& shapes, unsigned blocks, double flops, const MuonProduct& q,
                         hipStream_t s);
// The last step's product, and the parameters' update from its tiles.
bl_status_t muon_update(int param_dtype, int side, const MuonList& list, unsigned blocks, double flops, const MuonProduct& q,
                        const MuonArgs& a, hipStream_t s);

}  // namespace blc
