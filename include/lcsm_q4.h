/*
 * lcsm_q4.h -- C ABI of matrix-vector products with 4-bit weights and group
 * scales (include lcsm.h for the error codes and element types), for the
 * projections of layers that generate token by token, whose time is the read
 * of their weights.
 *
 * Operation: for each of M layers a matrix of N rows of K weights
 *
 *     w[n,k] = scale[n, k / group] (code[n,k] - zero[n, k / group])
 *     y[r,n] = bias[n] + sum_k w[n,k] x[r,k]
 *
 * with codes 0 .. 15, zeros 0 .. 15 (8 where none are given) and any number of
 * rows r.  x is multiplied by code - 8, exactly (and what zeros other than 8
 * leave of its sums is added); sums are fp32, and y is rounded once to x's type.
 * A row of x with values that are not finite gives a row of y that is not
 * finite; other rows are not touched by it.  Sums are taken over up to 128
 * inputs before they are scaled: they are within fp32 for any codes and zeros
 * where |x| stays below 1.7e35, and beyond that a row may be not finite where
 * the formula's is.
 *
 * Conventions as in lcsm.h: device pointers, asynchronous on the context's
 * stream, LCSM_* return codes, arguments validated before any device work is
 * queued, not thread safe.  No call but lcsm_q4_init allocates: all may be
 * recorded into a graph.
 */
#ifndef LCSM_Q4_H
#define LCSM_Q4_H

#include <stddef.h>

#include "lcsm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lcsm_q4 lcsm_q4;

typedef struct lcsm_q4_shape {
  int M;           /* layers */
  int N, K;        /* outputs and inputs of a matrix (<= 2^24, N K <= 2^40) */
  int group;       /* weights of a row that share a scale: 32, 64 or a multiple of 128 */
  int scale_dtype; /* type of the scales */
  int reserved[3]; /* must be zero */
} lcsm_q4_shape;

/* Device bytes of the workspace: the codes, scales and zeros laid out anew
 * (rows rounded up to 16, weights of a row to 128), and the biases.  Host
 * only.  Errors: LCSM_EINVAL. */
int lcsm_q4_workspace_bytes(const lcsm_q4_shape* shape, size_t* bytes);

/* Create a context.  With ng = ceil(K / group):
 *   codes   device [M][N][ceil(K/2)] bytes, the even k in the low four bits
 *   scales  device [M][N][ng] of scale_dtype
 *   zeros   device [M][N][ng] bytes (their low four bits count), NULL: all 8
 *   bias    device [M][N] fp32, NULL: none
 * All are laid out anew during the call's stream work; the caller may free
 * them once the stream has passed lcsm_q4_init.  workspace: at least
 * lcsm_q4_workspace_bytes bytes, 256-byte aligned, owned by the caller until
 * lcsm_q4_destroy; NULL makes the library allocate it.
 * Errors: LCSM_EINVAL, LCSM_ENOMEM, LCSM_EDEVICE; *out is NULL on failure. */
int lcsm_q4_init(lcsm_q4** out, const lcsm_q4_shape* shape, const void* codes, const void* scales,
                 const void* zeros, const float* bias, void* stream, void* workspace,
                 size_t workspace_bytes);

/* y [rows][N] = x [rows][K] times the layer's matrix, both of type dtype; a
 * row is contiguous, rows are `_stride` elements apart.  x and y do not
 * overlap.  rows = 0 queues nothing, more than 2^20 - 16 are refused.
 * Errors: LCSM_EINVAL (null pointers,
 * layer, rows, dtype or strides out of range), LCSM_ESTATE after a fault
 * (until lcsm_q4_reset), LCSM_EDEVICE. */
int lcsm_q4_matvec(lcsm_q4* ctx, int layer, int rows, int dtype, const void* x, size_t x_stride,
                   void* y, size_t y_stride);

/* Codes and scales of fp32 weights, without zeros (device w [rows][K], codes
 * [rows][ceil(K/2)], scales [rows][ceil(K / group)] of scale_dtype):
 *     scale = max |w| / 7 of the group, rounded to scale_dtype,
 *     code  = 8 + w / scale rounded to the nearest (ties to even), within
 *             0 .. 15; 8 where the scale is zero or not finite.
 * A group with a value that is not finite, or beyond 7 times what scale_dtype
 * holds, has a scale that is not finite, and so weights that are not.  An odd
 * K leaves the high bits of a row's last byte 8.  Needs no context; the work is
 * queued on `stream`.  Errors: LCSM_EINVAL, LCSM_EDEVICE. */
int lcsm_q4_quantize(const float* w, int rows, int K, int group, int scale_dtype, void* codes,
                     void* scales, void* stream);

/* Clears a fault.  Errors: LCSM_EINVAL. */
int lcsm_q4_reset(lcsm_q4* ctx);

/* Release the context (waits for its stream).  NULL is ignored. */
void lcsm_q4_destroy(lcsm_q4* ctx);

/* Text of the last error recorded on this context ("" if none). */
const char* lcsm_q4_last_error(const lcsm_q4* ctx);

#ifdef __cplusplus
}
#endif

#endif /* LCSM_Q4_H */
