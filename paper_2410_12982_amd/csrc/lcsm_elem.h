// Element types of the operators that take more than fp32, and what their
// kernels share.  Arithmetic is fp32: elements are widened when loaded and
// rounded (to nearest, ties to even) once when stored.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lcsm.h"

namespace lcsm {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

inline bool dtype_ok(int t) { return t == LCSM_F32 || t == LCSM_BF16 || t == LCSM_F16; }
inline size_t dtype_size(int t) { return t == LCSM_F32 ? 4 : 2; }

// f(element) with the element type of a code (dtype_ok).
template <class F>
auto with_dtype(int t, F&& f) {
  switch (t) {
    case LCSM_BF16: return f(bf16_t());
    case LCSM_F16: return f(f16_t());
    default: return f(float());
  }
}

__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }
// The reciprocal is good to an ulp.
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + exp2_hw(-1.44269504f * v)); }
__device__ __forceinline__ float silu(float v) { return v * sigmoid(v); }
__device__ __forceinline__ float softplus(float v) { return v > 20.0f ? v : log1pf(__expf(v)); }

}  // namespace lcsm
