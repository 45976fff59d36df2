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

// ---- prompts in chunks (lcsm_ssm_prompt.h)

constexpr int kSsmQ = 64;     // positions of a chunk
constexpr int kSsmWaves = 4;  // waves of a workgroup, 32 channels of a head each

// Operands of one chunk and group for NT blocks of 32 states, in bytes; a
// fragment of 64 lanes is 1024.  C: [position / 16][state block], B: [state /
// 16][position block], G = tril(C B^T): the six blocks of 16 x 32 positions
// that are not above the diagonal; all low parts PART (GPART) after the high
// ones.
template <int NT>
struct SsmBlock {
  static constexpr int PART = 4096 * NT, GPART = 6144;
  static constexpr int C = 0, B = 2 * PART, G = 4 * PART, BYTES = G + 2 * GPART;
};
inline size_t ssm_block_bytes(int N) {
  return N <= 32 ? SsmBlock<1>::BYTES : N <= 64 ? SsmBlock<2>::BYTES : N <= 128 ? SsmBlock<4>::BYTES : SsmBlock<8>::BYTES;
}

struct SsmScratch {
  char* bc;       // [blocks][G] SsmBlock
  float* states;  // [segments][H][P][N]: what a segment adds to the state after it
  float* decay;   // [segments][H]: and what it leaves of the one before it
  int blocks, segments;  // upper bounds of the call's chunks and segments
  int per;               // chunks a segment
  int pair, quads;       // two channels of a row, four states are aligned as one load
};

hipError_t ssm_prompt_f32(const SsmCall& c, const SsmScratch& w, hipStream_t st);
hipError_t ssm_prompt_bf16(const SsmCall& c, const SsmScratch& w, hipStream_t st);
hipError_t ssm_prompt_f16(const SsmCall& c, const SsmScratch& w, hipStream_t st);

}  // namespace lcsm
