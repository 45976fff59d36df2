/*
 * lcsm_rot.h -- C ABI of the norms of queries and keys for each head with the
 * rotation by their positions (include lcsm.h for the error codes and element
 * types, lcsm_norm.h for the kinds of norms).
 *
 * Operation, for every row (token) at position t and every head of P values x
 * of its queries, then its keys:
 *
 *   v = norm(x)                        of the head's P values, times the weights
 *                                      w of queries or of keys:
 *     LCSM_NORM_NONE   x
 *     LCSM_NORM_RMS    w * x / sqrt(mean(x^2) + eps)
 *     LCSM_NORM_LAYER  w * (x - mean(x)) / sqrt(var(x) + eps)
 *   (a, b) -> (a cos(t f_j) - b sin(t f_j), b cos(t f_j) + a sin(t f_j))
 *                                      for each pair j < rotary / 2 of v:
 *     LCSM_PAIRS_HALF      a = v[j],   b = v[j + rotary / 2]
 *     LCSM_PAIRS_ADJACENT  a = v[2 j], b = v[2 j + 1]
 *
 * and the values from `rotary` on as they are in v.  One pass: a head is read
 * once and written once.  Sums and values are fp32, an output is rounded once;
 * the angle is taken modulo a turn in fp64, so that far positions lose nothing.
 * Heads do not touch each other; where there is a norm, a head's sum of squares
 * stays below 2^128.
 *
 * A context holds the weights of M layers and the frequencies f_j that they
 * share.  Conventions as in lcsm.h: device pointers, asynchronous on the
 * context's stream, LCSM_* return codes, arguments validated before any device
 * work is queued, not thread safe.  No call but lcsm_rot_init allocates: all may
 * be recorded into a graph.
 */
#ifndef LCSM_ROT_H
#define LCSM_ROT_H

#include <stddef.h>

#include "lcsm.h"
#include "lcsm_norm.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LCSM_PAIRS_HALF 0
#define LCSM_PAIRS_ADJACENT 1

typedef struct lcsm_rot lcsm_rot;

typedef struct lcsm_rot_shape {
  int M;                /* layers */
  int P;                /* values of a head, at most 512 */
  int q_heads, k_heads; /* 1 .. 65536 and 0 .. 65536 */
  int rotary;           /* values of a head that are turned: even, 0 .. P */
  int pairs;            /* LCSM_PAIRS_* */
  int norm;             /* LCSM_NORM_* */
  int dtype;            /* type of queries and keys */
  float eps;
  int reserved[3]; /* must be zero */
} lcsm_rot_shape;

/* Device bytes of the workspace: the frequencies and both weights.  Host only.
 * Errors: LCSM_EINVAL (sizes out of range, unknown kinds or types, eps < 0 or
 * not finite). */
int lcsm_rot_workspace_bytes(const lcsm_rot_shape* shape, size_t* bytes);

/* Create a context.  freqs: device fp64 [rotary / 2], radians a position (may
 * be NULL with rotary 0); q_w, k_w: device fp32 [M][P], NULL: ones.  They are
 * copied during the call's stream work; the caller may free them once the
 * stream has passed lcsm_rot_init.  workspace: at least
 * lcsm_rot_workspace_bytes bytes, 256-byte aligned, owned by the caller until
 * lcsm_rot_destroy; NULL makes the library allocate it.
 * Errors: LCSM_EINVAL, LCSM_ENOMEM, LCSM_EDEVICE; *out is NULL on failure. */
int lcsm_rot_init(lcsm_rot** out, const lcsm_rot_shape* shape, const double* freqs, const float* q_w,
                  const float* k_w, void* stream, void* workspace, size_t workspace_bytes);

/* Rows of a call; a row is contiguous, rows are `_stride` elements apart (at
 * least the row's length): slices of one wide projection's rows can be handed
 * in as they are.
 *   q [rows][q_heads P], k [rows][k_heads P] (ignored with k_heads 0)
 *   q_out, k_out  receive the results; q_out may be q itself and k_out k
 *                 (same stride)
 *   positions     device int[rows] (may be NULL with rotary 0)
 * Otherwise the buffers do not overlap. */
typedef struct lcsm_rot_io {
  const void *q, *k;
  void *q_out, *k_out;
  size_t q_stride, k_stride, q_out_stride, k_out_stride;
  const int* positions;
} lcsm_rot_io;

/* One pass over `rows` rows with the weights of `layer`.  rows = 0 queues
 * nothing.  Errors: LCSM_EINVAL (null pointers, layer, rows or strides out of
 * range), LCSM_ESTATE after a fault (until lcsm_rot_reset), LCSM_EDEVICE. */
int lcsm_rot_apply(lcsm_rot* ctx, int layer, int rows, const lcsm_rot_io* io);

/* Clears a fault.  Errors: LCSM_EINVAL. */
int lcsm_rot_reset(lcsm_rot* ctx);

/* Release the context (waits for its stream).  NULL is ignored. */
void lcsm_rot_destroy(lcsm_rot* ctx);

/* Text of the last error recorded on this context ("" if none). */
const char* lcsm_rot_last_error(const lcsm_rot* ctx);

#ifdef __cplusplus
}
#endif

#endif /* LCSM_ROT_H */
