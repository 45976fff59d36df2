// What the host side and the kernels of linear attention share.
#pragma once

#include "lcsm_elem.h"
#include "lcsm_lin.h"

namespace lcsm {

// One layer's call as the kernels see it.
struct LinCall {
  int H, G, K, V;
  int slots, T, n;
  float scale;
  const int *offsets, *src, *dst;  // offsets NULL: one sequence of T rows
  const void *q, *k, *v;
  void* y;
  size_t q_stride, k_stride, v_stride, y_stride;
  const float* decay;  // of the layer
  float* state;        // [slots][G][K][V]
};

// How a prompt call is cut: segments of `per` chunks.
struct LinCut {
  float* states;  // [segments][G][K][V]: what a segment adds to the state after it, then the state before it
  int per, segments;  // segments: an upper bound
  int direct;         // rows are whole and aligned eights: they can go from memory straight into LDS
  int wide;           // so many outputs are whole and aligned as one: 8 (of 16 bits), 4 or 1
};

__device__ __forceinline__ int lin_slot(const int* list, int i, int slots) {
  const int s = list ? list[i] : i;
  return s >= 0 && s < slots ? s : -1;
}

// Rows [t0, t1) of sequence i.
__device__ __forceinline__ void lin_rows(const LinCall& c, int i, int& t0, int& t1) {
  t0 = 0;
  t1 = c.T;
  if (c.offsets) {
    t0 = min(max(c.offsets[i], 0), c.T);
    t1 = min(max(c.offsets[i + 1], t0), c.T);
  }
}

// A state after so many tokens: S' = keep S + by S, by a factor that is as exact
// for decays next to one (by = e^a - 1, keep = 1) as for strong ones (by = e^a,
// keep = 0).
struct LinDecay {
  float by, keep;
  __device__ LinDecay() {}
  __device__ explicit LinDecay(double a) {  // a: the logarithm; NaN is kept
    keep = a > -0.7 && a < 0.7 ? 1.f : 0.f;
    by = (float)(keep != 0.f ? expm1(a) : exp(a));
  }
  __device__ float operator()(float s) const { return fmaf(s, by, keep != 0.f ? s : 0.f); }
};

// Positions of a chunk (the kernels' lin_chunk).
inline int lin_blocks_of(int K) { return K <= 32 ? 1 : K <= 64 ? 2 : K <= 128 ? 4 : 8; }
inline int lin_chunk_of(int dtype, int K) { return dtype == LCSM_BF16 && K <= 128 ? 64 : 32; }
// Waves of a workgroup, 32 values of a state each.
constexpr int kLinWaves = 4;

hipError_t lin_prompt_f32(const LinCall& c, const LinCut& w, hipStream_t st);
hipError_t lin_prompt_bf16(const LinCall& c, const LinCut& w, hipStream_t st);
hipError_t lin_prompt_f16(const LinCall& c, const LinCut& w, hipStream_t st);

}  // namespace lcsm
