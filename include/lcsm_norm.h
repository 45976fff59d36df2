/*
 * lcsm_norm.h -- C ABI of the norms around a block, fused with the block's
 * gate, its residual scale and the sum (include lcsm.h for the error codes and
 * element types).
 *
 * Operation, for every row (token) of D values, with o the block's output, g
 * its gate and r the residual before the block:
 *
 *   v  = o * act(g)                 act: silu(g) = g / (1 + e^{-g}),
 *                                   sigmoid(g) = 1 / (1 + e^{-g}), or no gate
 *   q  = post(v)                    the norm after the block, each of `groups`
 *                                   equal parts of the row on its own
 *   r' = alpha r + scale * q        the residual after the block
 *   n  = pre(r')                    the norm before the next block (whole row)
 *
 * where a norm is one of
 *   LCSM_NORM_NONE   v
 *   LCSM_NORM_RMS    w * v / sqrt(mean(v^2) + eps) + b
 *   LCSM_NORM_LAYER  w * (v - mean(v)) / sqrt(var(v) + eps) + b
 * with weights w and biases b over the D values of a row.  One pass: o, g and
 * r are read once, r' and n written once; everything between is fp32 in
 * registers (n is the norm of r' before it is rounded), and the variance is
 * that of the differences from the mean.
 *
 * A context holds the weights of M layers.  Conventions as in lcsm.h: device
 * pointers, asynchronous on the context's stream, LCSM_* return codes,
 * arguments validated before any device work is queued, not thread safe.  No
 * call but lcsm_norm_init allocates: all may be recorded into a graph.
 */
#ifndef LCSM_NORM_H
#define LCSM_NORM_H

#include <stddef.h>

#include "lcsm.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LCSM_NORM_NONE 0
#define LCSM_NORM_RMS 1
#define LCSM_NORM_LAYER 2

#define LCSM_ACT_NONE 0
#define LCSM_ACT_SILU 1
#define LCSM_ACT_SIGMOID 2

typedef struct lcsm_norm lcsm_norm;

typedef struct lcsm_norm_shape {
  int M;         /* layers */
  int D;         /* values a row, at most 32768 */
  int post, pre; /* LCSM_NORM_* */
  int act;       /* LCSM_ACT_* */
  int groups;    /* parts of a row that the norm after the block takes apart (divides D, <= 1024) */
  int dtype;     /* type of o, g and n */
  int res_dtype; /* type of r and r': dtype or LCSM_F32 */
  float alpha, eps;
  int reserved[2]; /* must be zero */
} lcsm_norm_shape;

/* Create a context.  Weights are device fp32 [M][D]; NULL stands for ones
 * (post_w, pre_w, scale) or zeros (post_b, pre_b).  They are copied during the
 * call's stream work; the caller may free them once the stream has passed
 * lcsm_norm_init.  The library allocates the copies (4 M D bytes each).
 * Errors: LCSM_EINVAL (sizes out of range, unknown kinds or types, eps < 0,
 * alpha or eps not finite), LCSM_ENOMEM, LCSM_EDEVICE; *out is NULL on
 * failure. */
int lcsm_norm_init(lcsm_norm** out, const lcsm_norm_shape* shape, const float* post_w,
                   const float* post_b, const float* scale, const float* pre_w, const float* pre_b,
                   void* stream);

/* Rows of a call; a row is contiguous, rows are `_stride` elements apart.
 *   o        [rows][D]; NULL: no block before (r' = alpha r; g must be NULL)
 *   g        [rows][D]; needed where o is given and act is not LCSM_ACT_NONE,
 *            else NULL
 *   r        [rows][D]
 *   r_out    receives r', may be r itself (same stride); NULL: not kept
 *   n        receives pre(r'), may be o or g itself (same stride); NULL: not
 *            computed
 * Otherwise the buffers do not overlap. */
typedef struct lcsm_norm_io {
  const void *o, *g, *r;
  void *r_out, *n;
  size_t o_stride, g_stride, r_stride, r_out_stride, n_stride;
} lcsm_norm_io;

/* One pass over `rows` rows with the weights of `layer`.  rows = 0 queues
 * nothing.  Errors: LCSM_EINVAL (null pointers, layer, rows or strides out of
 * range), LCSM_ESTATE after a fault (until lcsm_norm_reset), LCSM_EDEVICE. */
int lcsm_norm_block(lcsm_norm* ctx, int layer, int rows, const lcsm_norm_io* io);

/* Clears a fault.  Errors: LCSM_EINVAL. */
int lcsm_norm_reset(lcsm_norm* ctx);

/* Release the context (waits for its stream).  NULL is ignored. */
void lcsm_norm_destroy(lcsm_norm* ctx);

/* Text of the last error recorded on this context ("" if none). */
const char* lcsm_norm_last_error(const lcsm_norm* ctx);

#ifdef __cplusplus
}
#endif

#endif /* LCSM_NORM_H */
