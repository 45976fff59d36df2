/*
 * lcsm_lin.h -- C ABI of linear attention with a decay for each head (include
 * lcsm.h for the error codes and element types): a mixer whose state has a
 * fixed size, as that of lcsm_ssm.h, for layers that stand beside the long
 * convolutions of lcsm.h.
 *
 * Operation: a layer has G states of K x V values, each with its decay e^g, and
 * H heads of queries, of which H / G neighbouring ones read one state.  Of
 * every token t it is given the queries q_t [H][K], the keys k_t [G][K] and the
 * values v_t [G][V]:
 *
 *   S_t[s] = e^{g[s]} S_{t-1}[s] + k_t[s] v_t[s]^T
 *   y_t[h] = scale q_t[h] S_t[s],    s = h / (H / G)
 *
 * A context holds, for each of M layers, `slots` sequences' states in fp32.
 * Calls name the slot that each sequence is read from and the one it is
 * written to, so that a sequence is continued in place, begun, or continued in
 * a copy.  Sums, decays and states are held in fp32 whatever the type of
 * queries, keys and values; outputs are rounded to it once.  Prompts make their
 * products on the matrix units, of parts of 16 bits: those that states are
 * made of, and all of fp32, to some 2^-24 of the factors.  Where outputs have
 * 16 bits, the scores q k and the states that queries are multiplied with
 * enter their products rounded to 2^-16, and of two fp16 values' product (and
 * of their products with scores and states) that of the lower parts, up to
 * 2^-16, is left out: shares of the magnitudes that are summed, which stay
 * below the outputs' rounding unless the sum is far smaller than those.  Single
 * tokens are fp32 throughout.
 *
 * A value that is not finite makes only those outputs and states not finite
 * that depend on it: no earlier token, no other sequence, no other head.
 * Values of fp32 stay below 2^127 in magnitude (above, what they reach may be
 * not finite where the formula's is).
 *
 * Conventions as in lcsm.h: device pointers, asynchronous on the context's
 * stream, LCSM_* return codes, arguments validated before any device work is
 * queued, not thread safe.  No call but lcsm_lin_init allocates: all may be
 * recorded into a graph; graphs that record prompts of one context share its
 * workspace and run one after another.
 */
#ifndef LCSM_LIN_H
#define LCSM_LIN_H

#include <stddef.h>

#include "lcsm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct lcsm_lin lcsm_lin;

typedef struct lcsm_lin_shape {
  int M;          /* layers */
  int slots;      /* sequences whose states the context holds (<= 32768); no call takes more sequences */
  int H, G;       /* heads of queries, states (G divides H, H <= 65535) */
  int K, V;       /* keys (<= 256) and values (<= 4096) of a state */
  int dtype;      /* type of queries, keys, values and outputs: LCSM_F32, LCSM_BF16 or LCSM_F16 */
  int max_tokens; /* tokens of the largest prompt call (<= 2^26); 0: steps only */
  float scale;    /* of the outputs, finite */
  int reserved[3]; /* must be zero */
} lcsm_lin_shape;

/* Device bytes of the workspace: the states 4 M slots G K V, the decays, and
 * for prompt calls the states of the segments that a call is cut into.  Host
 * only.  Errors: LCSM_EINVAL for a bad shape (sizes out of range, H (K + V)
 * beyond 2^24, a workspace beyond 2^46 bytes). */
int lcsm_lin_workspace_bytes(const lcsm_lin_shape* shape, size_t* bytes);

/* Create a context with all states zero.  decay: device fp32 [M][G], the
 * natural logarithms g of the states' decays (at most 0 for a decay; minus
 * infinity: a state holds its last token only).  With g above 0 a state grows:
 * prompts are right while e^(g n) is below 2^127, n the tokens of the call's
 * longest sequence rounded up to 64; beyond, outputs and states may be not
 * finite where the formula's are.  They are copied during the call's stream
 * work; the caller may free them once the stream has passed lcsm_lin_init.  stream: hipStream_t (NULL = the null stream).  workspace: at
 * least lcsm_lin_workspace_bytes bytes, 256-byte aligned, owned by the caller
 * until lcsm_lin_destroy; NULL makes the library allocate it.
 * Errors: LCSM_EINVAL, LCSM_ENOMEM, LCSM_EDEVICE; *out is NULL on failure. */
int lcsm_lin_init(lcsm_lin** out, const lcsm_lin_shape* shape, const float* decay, void* stream,
                  void* workspace, size_t workspace_bytes);

/* What a call reads and writes, rows of tokens in the context's type.  A row
 * is contiguous, rows are `_stride` elements apart (at least the row's
 * length, at most 2^24): slices of one wide projection's rows can be handed in
 * as they are.
 *   q [rows][H K], k [rows][G K], v [rows][G V], y [rows][H V]
 *   y receives the outputs and overlaps nothing else.
 *   src  device int[n]: the slot that sequence i's state is read from, -1:
 *        zero (a new sequence).  NULL: slot i.
 *   dst  device int[n]: the slot that it is written to, -1: not kept.
 *        NULL: slot i.
 * Values outside -1 .. slots-1 count as -1.  A slot that a sequence of the
 * call is written to is read by no other sequence of it and written by none. */
typedef struct lcsm_lin_io {
  const void *q, *k, *v;
  void* y;
  size_t q_stride, k_stride, v_stride, y_stride;
  const int *src, *dst;
} lcsm_lin_io;

/* One token of each of n sequences (rows = n).  n = 0 queues nothing.
 * Errors: LCSM_EINVAL (null pointers, layer, n or strides out of range),
 * LCSM_ESTATE after a fault, LCSM_EDEVICE. */
int lcsm_lin_step_layer(lcsm_lin* ctx, int layer, int n, const lcsm_lin_io* io);

/* Prompts, or further pieces of them: the tokens of n sequences one after
 * another, rows = T.
 *   offsets  device int[n + 1]: sequence i is rows offsets[i] .. offsets[i+1]
 *            (none where these are equal: its state moves from src to dst
 *            unchanged).  NULL: n must be 1, the sequence is all T rows.
 * Offsets have to rise within 0 .. T; others give wrong values, but nothing is
 * read or written outside the rows.  A row that no sequence has keeps its y.
 * Errors: as lcsm_lin_step_layer; LCSM_EINVAL for T > max_tokens. */
int lcsm_lin_prompt_layer(lcsm_lin* ctx, int layer, int T, int n, const int* offsets,
                          const lcsm_lin_io* io);

/* View of a layer's states, fp32 [slots][G][K][V] (valid until
 * lcsm_lin_destroy; read and written in the order of the context's stream).
 * Host only.  Errors: LCSM_EINVAL. */
int lcsm_lin_state(lcsm_lin* ctx, int layer, float** state);

/* All states zero; clears a fault.  Errors: LCSM_EINVAL, LCSM_EDEVICE. */
int lcsm_lin_reset(lcsm_lin* ctx);

/* Release the context (waits for its stream).  NULL is ignored. */
void lcsm_lin_destroy(lcsm_lin* ctx);

/* Text of the last error recorded on this context ("" if none). */
const char* lcsm_lin_last_error(const lcsm_lin* ctx);

#ifdef __cplusplus
}
#endif

#endif /* LCSM_LIN_H */
