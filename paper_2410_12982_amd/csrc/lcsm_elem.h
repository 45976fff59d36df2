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

constexpr size_t kMaxStride = (size_t)1 << 24;  // elements between rows

// A buffer that is the same for all lanes (which the compiler does not always
// see, and then loops over the lanes' values at every access).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t uniform_buffer(const void* p, unsigned bytes) {
  const uint64_t at = reinterpret_cast<uint64_t>(p);
  const unsigned lo = __builtin_amdgcn_readfirstlane((unsigned)at), hi = __builtin_amdgcn_readfirstlane((unsigned)(at >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t)hi << 32 | lo), 0,
                                           __builtin_amdgcn_readfirstlane((int)bytes), 0x00027000);
}

// Rows as a buffer of whole rows from a base row on: what lies past its end
// reads as zero and is not stored.  `rows` of them, `width` elements in the
// last; kMaxStride keeps the offsets of 40 rows of fp32, and of 64 of 16 bits,
// below 2^32.
template <class E>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const void* p, size_t row, size_t stride, int rows,
                                                             int width) {
  const unsigned bytes = rows > 0 ? (unsigned)((rows - 1) * stride + width) * (unsigned)sizeof(E) : 0u;
  return uniform_buffer(static_cast<const E*>(p) + row * stride, bytes);
}

// 16 bytes a lane from `lane_at` + `at` of a buffer into LDS, one lane after
// another.  The compiler does not wait for these where LDS is read.
__device__ __forceinline__ void fetch_to_lds(__amdgpu_buffer_rsrc_t r, unsigned lane_at, unsigned at, char* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)to, 16, (int)lane_at, (int)at, 0, 0);
}

// All waves past their LDS accesses; transfers and stores of global memory stay on
// their way, which __syncthreads may wait for.  (The wait is one that the compiler
// sees, so that it does not wait again, for later reads too.)
__device__ __forceinline__ void barrier_for_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// At most N memory instructions of this wave on their way, the older ones done.
template <int N>
__device__ __forceinline__ void wait_memory_but() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ __forceinline__ float exp2_hw(float v) { return __builtin_amdgcn_exp2f(v); }
// The reciprocal is good to an ulp.
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.0f + exp2_hw(-1.44269504f * v)); }
__device__ __forceinline__ float silu(float v) { return v * sigmoid(v); }
__device__ __forceinline__ float softplus(float v) { return v > 20.0f ? v : log1pf(__expf(v)); }

}  // namespace lcsm
