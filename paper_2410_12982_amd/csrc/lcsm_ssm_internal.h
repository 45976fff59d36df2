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
  int* tickets;                                       // [slots][G], zero between calls
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

constexpr size_t kSsmMaxStride = kMaxStride;

template <class E>
__device__ __forceinline__ float load_one(__amdgpu_buffer_rsrc_t r, unsigned at) {
  if constexpr (sizeof(E) == 4) return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0));
  else return (float)__builtin_bit_cast(E, (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0));
}

// ---- prompts in chunks (lcsm_ssm_prompt.h)

constexpr int kSsmQ = 64;  // positions of a chunk

// bf16 parts of a value in a product: all of fp32's bits.
constexpr int kSsmParts = 3;

// Operands of one chunk and group for NT blocks of 32 states, in bytes; a
// fragment of 64 lanes is 1024.  C: [position / 16][state block], B: [state /
// 16][position block], G = tril(C B^T): the six blocks of 16 x 32 positions
// that are not above the diagonal; every one part after part.  C and B of NB state blocks at a time are what LDS holds (STAGE).
template <int NT>
struct SsmBlock {
  static constexpr int NB = NT < 2 ? NT : 2, STAGES = NT / NB;
  static constexpr int PART = 4096 * NB, GPART = 6144;
  static constexpr int STAGE = 2 * kSsmParts * PART, G = STAGES * STAGE, GBYTES = kSsmParts * GPART;
  static constexpr int BYTES = G + GBYTES;
  static constexpr int c_at(int tt, int cc) { return cc / NB * STAGE + (tt * NB + cc % NB) * 1024; }
  static constexpr int b_at(int a, int b) { return a / (2 * NB) * STAGE + kSsmParts * PART + (a % (2 * NB) * 2 + b) * 1024; }
  static constexpr int g_at(int f) { return G + f * 1024; }
};

// What a workgroup of `waves` keeps in LDS: a stage (C and B; B alone where only
// the states are wanted), G of the chunk, and what each wave's positions have of
// its head.  TWICE: two of the first and the last, so that the next ones are
// fetched before these have been used; where they are small, two workgroups a
// compute unit take turns instead (4 x 2048 tokens of 24 heads x 64 x 64 in fp32
// 103 against 109 us; 16384 tokens of 64 heads x 64 x 128 with two parts a value
// 401 twice, 440 once and four waves).
template <int NT, bool OUT>
struct SsmLds {
  typedef SsmBlock<NT> Blk;
  static constexpr int C = OUT ? kSsmParts * Blk::PART : 0, STAGE = C + kSsmParts * Blk::PART;
  static constexpr bool TWICE = Blk::STAGES > 1;
  static constexpr int G = (TWICE ? 2 : 1) * STAGE, WAVES = G + (OUT ? Blk::GBYTES : 0);
  static constexpr int SCAL = 4 * kSsmQ * (int)sizeof(float);
  static constexpr int bytes(int waves) { return WAVES + (TWICE ? 2 : 1) * waves * SCAL; }
};

inline int ssm_blocks_of(int N) { return N <= 32 ? 1 : N <= 64 ? 2 : N <= 128 ? 4 : 8; }
inline size_t ssm_block_bytes(int N) { return (size_t)kSsmParts * (8192 * ssm_blocks_of(N) + 6144); }
// Waves of a workgroup, 32 channels of a head each: they share the operands in
// LDS.  256 registers are what they have up to N = 128, 512 above.
inline int ssm_waves(int N) { return N > 64 && N <= 128 ? 8 : 4; }

struct SsmScratch {
  void* windows;  // [sequences][W-1][C]: the windows that the call begins from
  char* bc;       // [blocks][G] SsmBlock
  float* scal;    // [blocks][H][4][64]: what a chunk's positions have of a head
  double* lq;     // [blocks][H][2]: log2 of the decays of a chunk's halves
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
