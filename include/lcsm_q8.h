/*
 * lcsm_q8.h -- C ABI of products with 8-bit weights and rows that are
 * quantized to 8 bits on the way, for the projections of prompts and of
 * batches of tokens (include lcsm.h for the error codes and element types;
 * lcsm_q4.h for weights of 4 bits).
 *
 * Operation: for each of M layers a matrix of N rows of K codes with a scale
 * for each row (output), and any rows x:
 *
 *     s[r]   = max_k |x[r,k]| / 127, rounded to fp32
 *     c[r,k] = x[r,k] / s[r] rounded to the nearest (ties to even), within
 *              -127 .. 127; 0 where s[r] is zero
 *     y[r,n] = s[r] scale[n] sum_k c[r,k] code[n,k] + bias[n]
 *
 * The sum is exact (32-bit integers), so that it does not depend on how it is
 * taken; y is rounded once to x's type.  A row of x with a value that is not
 * finite gives a row of y that is not finite; other rows are not touched by it.
 * Scales of outputs stay below 2^96 in magnitude.
 *
 * Conventions as in lcsm.h: device pointers, asynchronous on the context's
 * stream, LCSM_* return codes, arguments validated before any device work is
 * queued, not thread safe.  No call but lcsm_q8_init allocates: all may be
 * recorded into a graph.  The workspace holds a call's codes, so graphs that
 * record calls of one context run one after another.
 */
#ifndef LCSM_Q8_H
#define LCSM_Q8_H

#include <stddef.h>

#include "lcsm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lcsm_q8 lcsm_q8;

typedef struct lcsm_q8_shape {
  int M;           /* layers */
  int N, K;        /* outputs (<= 2^24) and inputs (<= 2^17) of a matrix, N K <= 2^40 */
  int max_rows;    /* rows of the largest call, 1 .. 2^24 */
  int reserved[4]; /* must be zero */
} lcsm_q8_shape;

/* Device bytes of the workspace: the codes laid out anew (rows rounded up to
 * 16, inputs to 128), scales and biases, and the codes and scales of a call's
 * rows.  Host only.  Errors: LCSM_EINVAL. */
int lcsm_q8_workspace_bytes(const lcsm_q8_shape* shape, size_t* bytes);

/* Create a context.
 *   codes   device int8 [M][N][K]
 *   scales  device fp32 [M][N]
 *   bias    device fp32 [M][N], NULL: none
 * All are laid out anew during the call's stream work; the caller may free
 * them once the stream has passed lcsm_q8_init.  workspace: at least
 * lcsm_q8_workspace_bytes bytes, 256-byte aligned, owned by the caller until
 * lcsm_q8_destroy; NULL makes the library allocate it.
 * Errors: LCSM_EINVAL, LCSM_ENOMEM, LCSM_EDEVICE; *out is NULL on failure. */
int lcsm_q8_init(lcsm_q8** out, const lcsm_q8_shape* shape, const void* codes, const float* scales,
                 const float* bias, void* stream, void* workspace, size_t workspace_bytes);

/* y [rows][N] from x [rows][K], both of type dtype; a row is contiguous, rows
 * are `_stride` elements apart.  x and y do not overlap.  rows = 0 queues
 * nothing.  Errors: LCSM_EINVAL (null pointers, layer, dtype or strides out of
 * range, rows below zero or above max_rows, more than 2^42 outputs),
 * LCSM_ESTATE after a fault (until lcsm_q8_reset), LCSM_EDEVICE. */
int lcsm_q8_matmul(lcsm_q8* ctx, int layer, int rows, int dtype, const void* x, size_t x_stride,
                   void* y, size_t y_stride);

/* Codes and scales of fp32 weights (device w [rows][K], codes int8 [rows][K],
 * scales fp32 [rows]) by the rule above.  A row with a value that is not finite
 * has a scale that is NaN and codes of zero.  Needs no context; the work is
 * queued on `stream`.  Errors: LCSM_EINVAL, LCSM_EDEVICE. */
int lcsm_q8_quantize(const float* w, int rows, int K, void* codes, float* scales, void* stream);

/* Clears a fault.  Errors: LCSM_EINVAL. */
int lcsm_q8_reset(lcsm_q8* ctx);

/* Release the context (waits for its stream).  NULL is ignored. */
void lcsm_q8_destroy(lcsm_q8* ctx);

/* Text of the last error recorded on this context ("" if none). */
const char* lcsm_q8_last_error(const lcsm_q8* ctx);

#ifdef __cplusplus
}
#endif

#endif /* LCSM_Q8_H */
