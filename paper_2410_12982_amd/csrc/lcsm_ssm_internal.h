// What the host side and the kernels of the state space mixer share.
#pragma once

#include "lcsm_elem.h"
#include "lcsm_ssm.h"

namespace lcsm {

// One layer's call as the kernels see it.  Channels of a row: D of x, G N of B,
// G N of C.
struct SsmCall {
  int H, P, N, G, W, D, C;
  int slots, T, n;
  int step;  // row i is the one token of sequence i
  const int *offsets, *src, *dst;  // offsets NULL: one sequence of T rows
  const void *xbc, *dt, *z;
  void* y;
  size_t xbc_stride, dt_stride, z_stride, y_stride;
  const float *conv_w, *conv_b, *A, *skip, *dt_bias;  // of the layer
  float* state;                                       // [slots][H][P][N]
  void* window;                                       // [slots][W-1][C]
};

__device__ __forceinline__ int ssm_slot(const int* list, int i, int slots) {
  const int s = list ? list[i] : i;
  return s >= 0 && s < slots ? s : -1;
}

// Rows [t0, t1) of sequence i.
__device__ __forceinline__ void ssm_rows(const SsmCall& c, int i, int& t0, int& t1) {
  t0 = c.step ? i : 0;
  t1 = c.step ? i + 1 : c.T;
  if (c.offsets) {
    t0 = min(max(c.offsets[i], 0), c.T);
    t1 = min(max(c.offsets[i + 1], t0), c.T);
  }
}

}  // namespace lcsm
