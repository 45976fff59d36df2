/*
 * lcsm_ssm.h -- C ABI of the selective state space mixer with its short
 * causal convolution (include lcsm.h for the error codes and element types):
 * a mixer whose state has a fixed size, for layers that stand beside the
 * long convolutions of lcsm.h.
 *
 * Operation: a layer has H heads of P channels (D = H P), states of N values
 * per channel, and G groups of H / G neighbouring heads that share B and C.
 * Of every token t it is given the C = D + 2 G N channels xbc_t (the D
 * channels x, then G rows of N of B, then G of C), the H values dt_t and the
 * gate z_t of D channels.  With W taps w[c,k] (w[c,W-1] is the tap of the
 * current token) and silu(v) = v / (1 + e^{-v}), softplus(v) = ln(1 + e^v):
 *
 *   u_t[c]     = silu(conv_b[c] + sum_{k<W} w[c,k] xbc_{t-W+1+k}[c])
 *   (x_t, B_t, C_t) = u_t,   s_t[h] = softplus(dt_t[h] + dt_bias[h])
 *   S_t[h,p,n] = e^{s_t[h] A[h]} S_{t-1}[h,p,n] + s_t[h] x_t[h,p] B_t[g,n]
 *   y_t[h,p]   = (sum_n C_t[g,n] S_t[h,p,n] + skip[h] x_t[h,p]) silu(z_t[h,p])
 *
 * with g = h / (H / G).  A context holds, for each of M layers, `slots`
 * sequences' states: S in fp32 and the last W-1 tokens' xbc (the window) as
 * they came.  Calls name the slot that each sequence is read from and the one
 * it is written to, so that a sequence is continued in place, begun, or
 * continued in a copy.  Sums, decays and states are fp32 whatever the type of
 * the activations; outputs are rounded to it once.
 *
 * A value that is not finite makes only those outputs and states not finite
 * that depend on it: no earlier token, no other sequence.
 *
 * Conventions as in lcsm.h: device pointers, asynchronous on the context's
 * stream, LCSM_* return codes, arguments validated before any device work is
 * queued, not thread safe.  No call but lcsm_ssm_init allocates: all may be
 * recorded into a graph.
 */
#ifndef LCSM_SSM_H
#define LCSM_SSM_H

#include <stddef.h>

#include "lcsm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lcsm_ssm lcsm_ssm;

typedef struct lcsm_ssm_shape {
  int M;          /* layers */
  int slots;      /* sequences whose states the context holds; no call takes more sequences */
  int H, P, N, G; /* heads, channels per head, states per channel (<= 256), groups (G divides H) */
  int W;          /* taps of the short convolution, 1 .. 4 */
  int dtype;      /* type of the activations: LCSM_F32, LCSM_BF16 or LCSM_F16 */
  int max_tokens; /* tokens of the largest prompt call; 0: steps only */
  int reserved[3]; /* must be zero */
} lcsm_ssm_shape;

/* Device bytes of the workspace: the states 4 M slots H P N, the windows,
 * copies of the parameters, and for prompt calls beyond 192 tokens what all
 * heads share of every 64 tokens (about 12 G N + 300 G + 17 H bytes a token) and
 * the states of the segments that a call is cut into.  Host only.
 * Errors: LCSM_EINVAL for a bad shape (sizes < 1, P > 4096, N > 256, W > 4, G not a
 * divisor of H, an unknown type, D + 2 G N > 2^24, slots > 65535, H > 65535,
 * G + H / 32 > 65534 with max_tokens > 192, max_tokens < 0 or > 2^26, or a
 * workspace beyond 2^46 bytes). */
int lcsm_ssm_workspace_bytes(const lcsm_ssm_shape* shape, size_t* bytes);

/* Create a context with all states and windows zero.
 *   conv_w   device [M][C][W] fp32;  conv_b  [M][C], NULL: zero
 *   A        [M][H], the heads' decay rates (negative for a decay)
 *   skip     [M][H], NULL: zero;     dt_bias [M][H], NULL: zero
 * All are copied during the call's stream work; the caller may free them once
 * the stream has passed lcsm_ssm_init.  stream: hipStream_t (NULL = the null
 * stream).  workspace: at least lcsm_ssm_workspace_bytes bytes, 256-byte
 * aligned, owned by the caller until lcsm_ssm_destroy; NULL makes the library
 * allocate it.  Errors: LCSM_EINVAL, LCSM_ENOMEM, LCSM_EDEVICE; *out is NULL
 * on failure. */
int lcsm_ssm_init(lcsm_ssm** out, const lcsm_ssm_shape* shape, const float* conv_w,
                  const float* conv_b, const float* A, const float* skip, const float* dt_bias,
                  void* stream, void* workspace, size_t workspace_bytes);

/* What a call reads and writes, rows of tokens in the context's type.  A row
 * is contiguous, rows are `_stride` elements apart (at least the row's
 * length, at most 2^24): slices of one wide projection's rows can be handed in
 * as they are.
 *   xbc [rows][D + 2 G N], dt [rows][H], z [rows][D] or NULL (no gate),
 *   y [rows][D] receives the outputs; it may be z itself (same stride), and
 *   overlaps nothing else.
 *   src  device int[n]: the slot that sequence i's state and window are read
 *        from, -1: zero (a new sequence).  NULL: slot i.
 *   dst  device int[n]: the slot that they are written to, -1: not kept.
 *        NULL: slot i.
 * Values outside -1 .. slots-1 count as -1.  A slot that a sequence of the
 * call is written to is read by no other sequence of it and written by none. */
typedef struct lcsm_ssm_io {
  const void *xbc, *dt, *z;
  void* y;
  size_t xbc_stride, dt_stride, z_stride, y_stride;
  const int *src, *dst;
} lcsm_ssm_io;

/* One token of each of n sequences (rows = n).  n = 0 queues nothing.
 * Errors: LCSM_EINVAL (null pointers, layer, n or strides out of range),
 * LCSM_ESTATE after a fault, LCSM_EDEVICE. */
int lcsm_ssm_step_layer(lcsm_ssm* ctx, int layer, int n, const lcsm_ssm_io* io);

/* Prompts, or further pieces of them: the tokens of n sequences one after
 * another, rows = T.
 *   offsets  device int[n + 1]: sequence i is rows offsets[i] .. offsets[i+1]
 *            (none where these are equal: its state moves from src to dst
 *            unchanged).  NULL: n must be 1, the sequence is all T rows.
 * Offsets have to rise within 0 .. T; others give wrong values, but nothing is
 * read or written outside the rows.  A row that no sequence has keeps its y.
 * Errors: as lcsm_ssm_step_layer; LCSM_EINVAL for T > max_tokens. */
int lcsm_ssm_prompt_layer(lcsm_ssm* ctx, int layer, int T, int n, const int* offsets,
                          const lcsm_ssm_io* io);

/* Views of a layer's states, fp32 [slots][H][P][N], and windows, in the
 * context's type [slots][W-1][C], oldest token first (valid until
 * lcsm_ssm_destroy; read and written in the order of the context's stream).
 * Host only.  Errors: LCSM_EINVAL. */
int lcsm_ssm_state(lcsm_ssm* ctx, int layer, float** state);
int lcsm_ssm_window(lcsm_ssm* ctx, int layer, void** window);

/* All states and windows zero; clears a fault.  Errors: LCSM_EINVAL,
 * LCSM_EDEVICE. */
int lcsm_ssm_reset(lcsm_ssm* ctx);

/* Release the context (waits for its stream).  NULL is ignored. */
void lcsm_ssm_destroy(lcsm_ssm* ctx);

/* Text of the last error recorded on this context ("" if none). */
const char* lcsm_ssm_last_error(const lcsm_ssm* ctx);

#ifdef __cplusplus
}
#endif

#endif /* LCSM_SSM_H */
