/*
 * bltrain.h -- what a training step or an answer needs around the band-limited
 * convolution layer of blconv.h: layer norm, the log probabilities that a
 * classifier's or a language model's loss is made of, and the AdamW update of
 * many tensors, for AMD Instinct MI355X (gfx950).
 *
 * Ownership: as in blconv.h, the caller owns every device buffer and creating
 * and querying a plan makes no HIP call.  Compute calls allocate nothing, keep
 * nothing from one call for the next, make no host synchronisation and enqueue
 * their kernels on `stream` (a hipStream_t, NULL = the default stream) of the
 * current device, which has to be the buffers' own, so they can be captured in a
 * HIP graph.  A workspace is scratch: its contents before
 * and after a call mean nothing.  Workspaces and AdamW's state must be aligned to
 * 16 bytes (else BL_ERR_INVALID_ARG); tensors need the alignment of their element
 * type only.
 *
 * Errors: every call returns a bl_status_t.  Arguments are validated on the
 * host before anything is enqueued; a call that returns an error other than
 * BL_ERR_HIP (a failed launch) has enqueued no kernel.
 *
 * Arithmetic: values are converted to fp32 when they are loaded; sums,
 * statistics, moments and norms are held in fp32 and a result is rounded once,
 * to nearest even, when it is stored (AdamW's parameters of 16 bits and moments
 * of 8 bits: by a dither, see there).  Sums are taken in an order that depends
 * on sizes alone: the same call on the same values gives the same bits.
 *
 * Threading: a plan is immutable; calls with distinct outputs and workspaces
 * may run concurrently from several threads and streams.
 */
#ifndef BLTRAIN_H
#define BLTRAIN_H

#include "blconv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define BL_F32 0
#define BL_BF16 1
#define BL_F16 2

/* ---- layer norm -------------------------------------------------------------
 *
 * Over the middle axis of x [outer][size][inner]: at every (o, i)
 *
 *   mean = sum_j x[o][j][i] / size,   rstd = 1 / sqrt(sum_j (x - mean)^2 / size + eps)
 *   y[o][j][i] = (x[o][j][i] - mean) rstd w[j] + b[j]
 *
 * inner = 1 normalises rows; inner = length or H W normalises the channels at
 * each position of the convolution layer's [N][C][L] or [N][C][H][W] maps;
 * size = C H W, inner = 1 a whole sample.
 *
 * x and dx have `dtype` and lie outer slices x_stride elements apart (0: dense,
 * size inner); y and dy likewise with y_stride.  w, b, dw, db [size] have
 * `wdtype`: fp32, or dtype. */
typedef struct {
  long long outer;  /* >= 0; 0: the calls do nothing but zero dw and db */
  long long size;   /* >= 1 */
  long long inner;  /* >= 1; size * inner < 2^31 */
  int dtype, wdtype;
  double eps;       /* >= 0 */
  long long x_stride, y_stride;
} bl_norm_desc_t;

typedef struct bl_norm_plan_s* bl_norm_plan_t;

/* BL_ERR_UNSUPPORTED: size * inner >= 2^31, size > 2^31 - 32, outer * inner >= 2^31, or
 * rows (inner = 1) of over 16384 elements in such a number that they are cut into 2^24
 * chunks. */
bl_status_t bl_norm_plan_create(bl_norm_plan_t* out, const bl_norm_desc_t* desc);
bl_status_t bl_norm_plan_destroy(bl_norm_plan_t plan);
/* Workspace bytes of either call (0: ws may be NULL). */
bl_status_t bl_norm_workspace_size(bl_norm_plan_t plan, size_t* bytes);

/* y, and in stats [2][outer][inner] (fp32; NULL: not wanted) mean and rstd.
 * w NULL: 1, b NULL: 0.  y may be x (the same pointer and strides). */
bl_status_t bl_norm_forward(bl_norm_plan_t plan, const void* x, const void* w, const void* b, void* y, float* stats,
                            void* ws, void* stream);

/* Gradients of <dy, y>: with h = (x - mean) rstd and u = dy w,
 *   dx = rstd (u - mean_j u - h mean_j (u h)),
 *   dw[j] = sum over outer and inner of dy h,  db[j] = sum of dy.
 * stats: what bl_norm_forward gave.  dw or db NULL: not wanted; w NULL: 1. dx
 * may be dy or x (the same pointer and strides). */
bl_status_t bl_norm_backward(bl_norm_plan_t plan, const void* dy, const void* x, const void* w, const float* stats,
                             void* dx, void* dw, void* db, void* ws, void* stream);

/* ---- log probabilities ------------------------------------------------------
 *
 * Of rows of logits z [rows][classes] (`dtype`, rows `stride` elements apart, 0:
 * dense), with m = max_j z_j, q_j = exp(z_j - m) / sum_k exp(z_k - m):
 *
 *   logp = log q_t for the row's target t,   entropy = -sum_j q_j log q_j,
 *
 * and the `top` classes of largest z, in falling order, with their log q; of
 * equal values the lower class comes first (-0 equals 0; a NaN counts as larger
 * than any number).
 *
 * A class ruled out is a logit of minus infinity: its q is 0.  A row that rules
 * out every class has logp = -infinity, entropy 0, gradients 0 and, as top
 * classes, the first ones at -infinity.  A row that holds a NaN or +infinity
 * gives NaN.  A target outside [0, classes) marks a row without one: its logp is
 * 0 and its g_logp is not used.  Where `top` exceeds `classes` the places
 * left over hold class -1 at -infinity. */
typedef struct {
  long long rows;    /* >= 0 */
  long long classes; /* >= 1, < 2^31 */
  int top;           /* 0 ... 64 */
  int dtype;
  long long stride, grad_stride; /* of logits and of their gradient */
} bl_logprob_desc_t;

typedef struct bl_logprob_plan_s* bl_logprob_plan_t;

/* BL_ERR_UNSUPPORTED: top > 64, classes or rows >= 2^31. */
bl_status_t bl_logprob_plan_create(bl_logprob_plan_t* out, const bl_logprob_desc_t* desc);
bl_status_t bl_logprob_plan_destroy(bl_logprob_plan_t plan);
bl_status_t bl_logprob_workspace_size(bl_logprob_plan_t plan, size_t* bytes); /* of the forward call */

/* logp [rows]; stats [3][rows]: m, log sum_k exp(z_k - m) and the entropy (fp32;
 * for the backward call); top_logp [rows][top] and top_index [rows][top] where
 * top > 0.  targets NULL: no row has one.  logp or stats NULL: not wanted. */
bl_status_t bl_logprob_forward(bl_logprob_plan_t plan, const void* logits, const long long* targets, float* logp,
                               float* stats, float* top_logp, long long* top_index, void* ws, void* stream);

/* Gradient of sum_rows g_logp logp + g_entropy entropy with respect to the logits:
 *   dz_j = g_logp ([j = t] - q_j) - g_entropy q_j (log q_j + entropy).
 * g_logp or g_entropy NULL: 0.  dlogits (`dtype`, grad_stride) may be the logits
 * themselves where the strides agree. */
bl_status_t bl_logprob_backward(bl_logprob_plan_t plan, const void* logits, const long long* targets,
                                const float* stats, const float* g_logp, const float* g_entropy, void* dlogits,
                                void* stream);

/* ---- AdamW ------------------------------------------------------------------
 *
 * One step over `count` tensors, elementwise, with s = *grad_scale and t = step:
 *
 *   g = s grad,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g g
 *   p = p (1 - lr weight_decay) - (lr / (1 - beta1^t)) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 *
 * (weight decay where the tensor's decay byte is set.)  Parameters are fp32 or
 * bfloat16, gradients fp32, bfloat16 or fp16.  With eps = 0 a value without any
 * gradient so far becomes NaN (0 / 0), and one whose g g is below fp32's least
 * subnormal value infinite.
 *
 * State: one device buffer of the caller's, filled with zero bytes before the
 * first step.  Tensor i's moments start at element start[i] of both moments'
 * arrays, a multiple of 1024, so that `total` elements are held.
 *
 * bits = 32: the moments are fp32.
 * bits = 8: blocks of 128 elements of a tensor share a power of two S, the
 * largest that does not exceed the block's largest finite magnitude, and at
 * least 2^-96.  m is held as a sign bit, 4 bits of exponent and 3 of fraction:
 * with e = code >> 3 and f = code & 7, |m| = S 2^(e - 14) (1 + f / 8), for
 * e = 0 S 2^-13 f / 8; v as 5 bits of exponent and 3 of fraction, S 2^(e - 30)
 * (1 + f / 8), for e = 0 S 2^-29 f / 8.  The code of all ones is NaN, which
 * stands for everything not finite.  Eight steps a factor of two round each
 * value by up to 6 %, and a change of v by 0.1 % a step would never pass
 * rounding to nearest: values are rounded down or up by chance so that they are
 * held right on average, by 16 bits of a hash of the element's place in the
 * layout, `seed` and the step.  A positive v is never held as 0 (a later step
 * would divide m by eps alone).  The parameters' step uses m and v before they
 * are rounded.  Parameters in bfloat16 are rounded by the same kind of chance.
 *
 * The hash, in 32-bit words: x = element * 0x9E3779B9 + key with key = seed *
 * 0x6A09E667 + step * 0xBB67AE85; x = (x ^ x >> 15) * 0xBB67AE85; x ^= x >> 16.
 * The low 16 bits round m, the high ones v, the high ones of x * 0x6A09E667 p. */
typedef struct {
  int count;                 /* >= 0 */
  const long long* sizes;    /* [count] elements, >= 0 (host memory, copied) */
  const unsigned char* decay; /* [count] 1: weight decay applies; NULL: to all */
  int param_dtype;           /* BL_F32 or BL_BF16 */
  int grad_dtype;
  int bits;                  /* of the moments: 32 or 8 */
} bl_adamw_desc_t;

typedef struct {
  double lr, beta1, beta2, eps, weight_decay;
  long long step;          /* 1 in the first step */
  unsigned seed;           /* of the dither */
  const float* grad_scale; /* device; NULL: 1 */
  const double* live;      /* device {lr, step} in the place of the two above, read when
                              the kernels run, so that a captured step can go on; or NULL.
                              Moments of 8 bits take about twice the time with it */
} bl_adamw_args_t;

typedef struct bl_adamw_plan_s* bl_adamw_plan_t;

/* BL_ERR_UNSUPPORTED: a tensor of more than 2^34 - 1024 elements, or 2^31 or more blocks of 1024. */
bl_status_t bl_adamw_plan_create(bl_adamw_plan_t* out, const bl_adamw_desc_t* desc);
bl_status_t bl_adamw_plan_destroy(bl_adamw_plan_t plan);
/* Bytes of the state, elements of each moment's array, and start[count] (any may be NULL). */
bl_status_t bl_adamw_state_size(bl_adamw_plan_t plan, size_t* bytes, long long* total, long long* start);
/* Byte offsets of m, v and, with bits = 8, of the fp32 powers of two of their blocks. */
bl_status_t bl_adamw_state_layout(bl_adamw_plan_t plan, size_t* off_m, size_t* off_v, size_t* off_m_scale,
                                  size_t* off_v_scale);

/* params, grads: host arrays of `count` device pointers (those of empty tensors
 * may be NULL).  Parameters and state are updated in place. */
bl_status_t bl_adamw_step(bl_adamw_plan_t plan, void* const* params, const void* const* grads, void* state,
                          const bl_adamw_args_t* args, void* stream);

/* The moments as values, m and v [total] each: fp32 with bits = 32, bfloat16 with
 * bits = 8 (which holds every 8-bit value exactly); and from fp32 values, rounded
 * to nearest with bits = 8 (half away from zero; S is the largest power of two
 * below the block's largest magnitude, so that values which bl_adamw_get_moments
 * gave are held again exactly; a negative v is held as NaN).  Elements between the tensors must be 0 in what is
 * set, as they are in what is given. */
bl_status_t bl_adamw_get_moments(bl_adamw_plan_t plan, const void* state, void* m, void* v, void* stream);
bl_status_t bl_adamw_set_moments(bl_adamw_plan_t plan, void* state, const float* m, const float* v, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BLTRAIN_H */
