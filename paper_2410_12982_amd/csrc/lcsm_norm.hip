// Norms around a block with its gate, residual scale and sum (lcsm_norm.h).
//
// A row is held in the registers of TPR threads from its first load to its last
// store, so that it is read and written once; the statistics are sums over
// those registers (the variance a second sum, of the differences from the
// mean).  Memory bounds it: 16384 rows of 2048 bf16 values with an fp32 residual
// take 90 us, 4.5 TB/s of the 403 MB that have to move (a large copy reaches
// 4.8); a few rows take the 6 us of a launch and its two round trips.  Rows that
// are not aligned to 16 bytes, or not of whole eights, go through the same
// kernels with accesses of the elements' alignment: 2047 values 134 us (232 one
// element at a time), 1025 57 (98).
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>

#include "lcsm_elem.h"
#include "lcsm_norm.h"

namespace lcsm {
namespace {

constexpr int kNormMaxD = 32768;
constexpr int kNormMaxGroups = 1024;

struct NormCall {
  int rows, D, groups, post, pre, act;
  float alpha, eps;
  const void *o, *g, *r;
  void *r_out, *n;
  size_t o_stride, g_stride, r_stride, r_out_stride, n_stride;
  const float *post_w, *post_b, *scale, *pre_w, *pre_b;  // of the layer, NULL where not given
};

constexpr int kVec = 8;  // elements of a thread side by side

// Eight elements from p, of which `have` (at least one) are there, the others
// zero.  WHOLE: all are, and p is aligned to 16 bytes; else p has the alignment
// of one element, which wide accesses of global memory allow.
template <bool WHOLE, class E>
__device__ __forceinline__ void load(const E* p, int have, float (&v)[kVec]) {
  struct __attribute__((packed, aligned(WHOLE ? 16 : sizeof(E)))) Pack {
    E e[kVec];
  };
  if (WHOLE || have >= kVec) {
    const Pack k = *reinterpret_cast<const Pack*>(p);
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = (float)k.e[i];
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = i < have ? (float)p[i] : 0.f;
  }
}
template <bool WHOLE, class E>
__device__ __forceinline__ void store(E* p, int have, const float (&v)[kVec]) {
  struct __attribute__((packed, aligned(WHOLE ? 16 : sizeof(E)))) Pack {
    E e[kVec];
  };
  if (WHOLE || have >= kVec) {
    Pack k;
#pragma unroll
    for (int i = 0; i < kVec; ++i) k.e[i] = (E)v[i];
    *reinterpret_cast<Pack*>(p) = k;
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i < have) p[i] = (E)v[i];
  }
}

// Sum over the TPR threads of a row, in a fixed order; every thread gets it.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* part) {
#pragma unroll
  for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
  if constexpr (TPR > 64) {
    __syncthreads();  // the last sum's parts have been read
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) v += part[w];
  }
  return v;
}

template <class E, class RE, bool WHOLE, int NV, int TPR, bool GROUPED>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_norm(NormCall c) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;  // rows a workgroup
  constexpr int VEC = kVec, FP = VEC * NV;
  __shared__ float part[TPR / 64];
  extern __shared__ float all[];  // GROUPED: the row, then mean and factor of every group; of each row
  const int lane = (int)threadIdx.x % TPR;
  const size_t row = ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * RPB + threadIdx.x / TPR;
  // rows past the last one are computed again by whoever takes them, and not
  // stored: every thread meets every barrier
  const bool live = row < (size_t)c.rows;
  const size_t at = live ? row : (size_t)c.rows - 1;
  const int D = c.D;
  float* lds = all + (size_t)(threadIdx.x / TPR) * (D + 2 * c.groups);
  auto index = [&](int k) { return (k * TPR + lane) * VEC; };

  float v[FP], res[FP];
  {
    const RE* r = static_cast<const RE*>(c.r) + at * c.r_stride;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float t[VEC] = {};
      if (index(k) < D) load<WHOLE>(r + index(k), D - index(k), t);
#pragma unroll
      for (int e = 0; e < VEC; ++e) res[k * VEC + e] = c.alpha * t[e];
    }
  }
  if (c.o) {
    const E* o = static_cast<const E*>(c.o) + at * c.o_stride;
    const E* g = static_cast<const E*>(c.g) + at * c.g_stride;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float t[VEC] = {}, u[VEC] = {};
      if (index(k) < D) {
        load<WHOLE>(o + index(k), D - index(k), t);
        if (c.act != LCSM_ACT_NONE) load<WHOLE>(g + index(k), D - index(k), u);
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        float f = 1.f;
        if (c.act != LCSM_ACT_NONE) f = sigmoid(u[e]);
        if (c.act == LCSM_ACT_SILU) f *= u[e];
        v[k * VEC + e] = t[e] * f;
      }
    }
    if (c.post != LCSM_NORM_NONE) {
      if constexpr (GROUPED) {
        // the row meets in LDS, every wave takes groups of it
        const int per = D / c.groups;
        int team = 64;  // lanes a group: several groups a wave where they are short
        while (team > per) team /= 2;
        auto team_sum = [&](float x) {
          for (int m = 1; m < team; m *= 2) x += __shfl_xor(x, m);
          return x;
        };
        const int who = lane % team;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (index(k) + e < D) lds[index(k) + e] = v[k * VEC + e];
        __syncthreads();
        // (all lanes take every turn: their sums go through each other's registers)
        for (int q0 = 0; q0 < c.groups; q0 += TPR / team) {
          const int q = q0 + lane / team;
          const float* x = lds + min(q, c.groups - 1) * per;
          float mean = 0.f, var = 0.f;
          if (c.post == LCSM_NORM_LAYER) {
            for (int i = who; i < per; i += team) mean += x[i];
            mean = team_sum(mean) / per;
          }
          for (int i = who; i < per; i += team) var += (x[i] - mean) * (x[i] - mean);
          var = team_sum(var) / per;
          if (who == 0 && q < c.groups) {
            lds[D + 2 * q] = mean;
            lds[D + 2 * q + 1] = 1.f / sqrtf(var + c.eps);
          }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const int q = min(index(k) + e, D - 1) / per;
            v[k * VEC + e] = (v[k * VEC + e] - lds[D + 2 * q]) * lds[D + 2 * q + 1];
          }
      } else {
        float mean = 0.f, var = 0.f;
        if (c.post == LCSM_NORM_LAYER) {
#pragma unroll
          for (int i = 0; i < FP; ++i) mean += v[i];  // (zeros past the row)
          mean = row_sum<TPR>(mean, part) / D;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (index(k) + e < D) var += (v[k * VEC + e] - mean) * (v[k * VEC + e] - mean);
        const float f = 1.f / sqrtf(row_sum<TPR>(var, part) / D + c.eps);
#pragma unroll
        for (int i = 0; i < FP; ++i) v[i] = (v[i] - mean) * f;
      }
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      if (index(k) >= D) continue;
      float w[VEC], b[VEC], s[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) w[e] = s[e] = 1.f, b[e] = 0.f;
      if (c.post_w) load<WHOLE>(c.post_w + index(k), D - index(k), w);
      if (c.post_b) load<WHOLE>(c.post_b + index(k), D - index(k), b);
      if (c.scale) load<WHOLE>(c.scale + index(k), D - index(k), s);
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (WHOLE || index(k) + e < D) res[k * VEC + e] = fmaf(s[e], fmaf(v[k * VEC + e], w[e], b[e]), res[k * VEC + e]);
    }
  }
  if (c.r_out && live) {
    RE* r = static_cast<RE*>(c.r_out) + at * c.r_out_stride;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float t[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) t[e] = res[k * VEC + e];
      if (index(k) < D) store<WHOLE>(r + index(k), D - index(k), t);
    }
  }
  if (!c.n) return;
  float mean = 0.f, f = 1.f;
  if (c.pre == LCSM_NORM_LAYER) {
#pragma unroll
    for (int i = 0; i < FP; ++i) mean += res[i];
    mean = row_sum<TPR>(mean, part) / D;
  }
  if (c.pre != LCSM_NORM_NONE) {
    float var = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (index(k) + e < D) var += (res[k * VEC + e] - mean) * (res[k * VEC + e] - mean);
    f = 1.f / sqrtf(row_sum<TPR>(var, part) / D + c.eps);
  }
  if (!live) return;
  E* n = static_cast<E*>(c.n) + at * c.n_stride;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    if (index(k) >= D) continue;
    float w[VEC], b[VEC], t[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = 1.f, b[e] = 0.f;
    if (c.pre_w) load<WHOLE>(c.pre_w + index(k), D - index(k), w);
    if (c.pre_b) load<WHOLE>(c.pre_b + index(k), D - index(k), b);
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] = fmaf((res[k * VEC + e] - mean) * f, w[e], b[e]);
    store<WHOLE>(n + index(k), D - index(k), t);
  }
}

template <class E, class RE, bool WHOLE, int NV, int TPR, bool GROUPED>
hipError_t launch(const NormCall& c, hipStream_t st) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
  // one axis of a launch takes fewer than 2^32 threads: 2^20 workgroups of it
  const unsigned n = ((unsigned)c.rows + RPB - 1) / RPB, x = n < 1u << 20 ? n : 1u << 20;
  const dim3 grid(x, (n + x - 1) / x), block(TPR < 256 ? 256 : TPR);
  const size_t bytes = GROUPED ? RPB * ((size_t)c.D + 2 * (size_t)c.groups) * sizeof(float) : 0;
  auto kernel = k_norm<E, RE, WHOLE, NV, TPR, GROUPED>;
  if (bytes > 65536 - 1024) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, grid, block, bytes, st, c);
  return hipGetLastError();
}

// A wave holds a row of up to 2048 values, 256 threads one of up to 8192 and
// 1024 threads the longest.  Parts normed on their own meet in LDS, where four
// waves a row are faster from some length on (16384 rows of 2048 in four parts
// 88 us, a wave 105; of 512 a wave 27, four 48).
template <class E, class RE, bool WHOLE>
hipError_t launch_rows(const NormCall& c, hipStream_t st) {
  const bool grouped = c.groups > 1 && c.o && c.post != LCSM_NORM_NONE;
  if (grouped) {
    if (c.D <= 512) return launch<E, RE, WHOLE, 1, 64, true>(c, st);
    if (c.D <= 2048) return launch<E, RE, WHOLE, 1, 256, true>(c, st);
    if (c.D <= 8192) return launch<E, RE, WHOLE, 4, 256, true>(c, st);
    return launch<E, RE, WHOLE, 4, 1024, true>(c, st);
  }
  if (c.D <= 512) return launch<E, RE, WHOLE, 1, 64, false>(c, st);
  if (c.D <= 2048) return launch<E, RE, WHOLE, 4, 64, false>(c, st);
  if (c.D <= 8192) return launch<E, RE, WHOLE, 4, 256, false>(c, st);
  return launch<E, RE, WHOLE, 4, 1024, false>(c, st);
}

bool aligned(const void* p, size_t stride, size_t elem) {
  return !p || (((uintptr_t)p & 15) == 0 && stride * elem % 16 == 0);
}

template <class E, class RE>
hipError_t launch_norm(const NormCall& c, hipStream_t st) {
  const bool whole = c.D % kVec == 0 && aligned(c.o, c.o_stride, sizeof(E)) &&
                   aligned(c.g, c.g_stride, sizeof(E)) && aligned(c.n, c.n_stride, sizeof(E)) &&
                   aligned(c.r, c.r_stride, sizeof(RE)) && aligned(c.r_out, c.r_out_stride, sizeof(RE));
  return whole ? launch_rows<E, RE, true>(c, st) : launch_rows<E, RE, false>(c, st);
}

}  // namespace
}  // namespace lcsm

struct lcsm_norm {
  lcsm_norm_shape s;
  hipStream_t stream;
  float* mem;
  float* w[5];  // post_w, post_b, scale, pre_w, pre_b; NULL where not given
  bool faulted;
  char msg[256];
};

namespace {

int norm_fail(lcsm_norm* c, int code, const char* what, hipError_t e = hipSuccess) {
  if (e != hipSuccess) {
    snprintf(c->msg, sizeof(c->msg), "%s: %s", what, hipGetErrorString(e));
    c->faulted = true;
    return LCSM_EDEVICE;
  }
  snprintf(c->msg, sizeof(c->msg), "%s", what);
  return code;
}

bool norm_shape_ok(const lcsm_norm_shape* s) {
  return s && s->M >= 1 && s->M <= 16384 && s->D >= 1 && s->D <= lcsm::kNormMaxD && s->post >= 0 &&
         s->post <= LCSM_NORM_LAYER && s->pre >= 0 && s->pre <= LCSM_NORM_LAYER && s->act >= 0 &&
         s->act <= LCSM_ACT_SIGMOID && s->groups >= 1 && s->groups <= lcsm::kNormMaxGroups &&
         s->D % s->groups == 0 && lcsm::dtype_ok(s->dtype) &&
         (s->res_dtype == s->dtype || s->res_dtype == LCSM_F32) && isfinite(s->alpha) &&
         isfinite(s->eps) && s->eps >= 0.f && !s->reserved[0] && !s->reserved[1];
}

}  // namespace

extern "C" {

int lcsm_norm_init(lcsm_norm** out, const lcsm_norm_shape* shape, const float* post_w,
                   const float* post_b, const float* scale, const float* pre_w, const float* pre_b,
                   void* stream) {
  if (!out) return LCSM_EINVAL;
  *out = nullptr;
  if (!norm_shape_ok(shape)) return LCSM_EINVAL;
  lcsm_norm* c = new (std::nothrow) lcsm_norm();
  if (!c) return LCSM_ENOMEM;
  c->s = *shape;
  c->stream = (hipStream_t)stream;
  const float* src[5] = {post_w, post_b, scale, pre_w, pre_b};
  const size_t n = (size_t)shape->M * shape->D, room = (n + 63) / 64 * 64;
  size_t given = 0;
  for (const float* p : src) given += p != nullptr;
  if (given) {
    void* mem = nullptr;
    if (hipMalloc(&mem, given * room * sizeof(float)) != hipSuccess) {
      (void)hipGetLastError();
      delete c;
      return LCSM_ENOMEM;
    }
    c->mem = (float*)mem;
    size_t at = 0;
    hipError_t e = hipSuccess;
    for (int k = 0; k < 5 && e == hipSuccess; ++k) {
      if (!src[k]) continue;
      c->w[k] = c->mem + at;
      at += room;
      e = hipMemcpyAsync(c->w[k], src[k], n * sizeof(float), hipMemcpyDeviceToDevice, c->stream);
    }
    if (e != hipSuccess) {
      (void)hipGetLastError();
      (void)hipStreamSynchronize(c->stream);
      (void)hipFree(c->mem);
      delete c;
      return LCSM_EDEVICE;
    }
  }
  *out = c;
  return LCSM_OK;
}

int lcsm_norm_block(lcsm_norm* ctx, int layer, int rows, const lcsm_norm_io* io) {
  if (!ctx) return LCSM_EINVAL;
  const lcsm_norm_shape& s = ctx->s;
  if (layer < 0 || layer >= s.M) return norm_fail(ctx, LCSM_EINVAL, "layer out of range");
  if (rows < 0 || !io) return norm_fail(ctx, LCSM_EINVAL, "rows below zero or null io");
  const size_t D = (size_t)s.D;
  if (rows > 0) {
    if (!io->r || (!io->r_out && !io->n)) return norm_fail(ctx, LCSM_EINVAL, "null residual or no output");
    if ((io->o && s.act != LCSM_ACT_NONE) != (io->g != nullptr))
      return norm_fail(ctx, LCSM_EINVAL, "a gate is needed with act and o, and only then");
    if ((io->o && io->o_stride < D) || (io->g && io->g_stride < D) || io->r_stride < D ||
        (io->r_out && io->r_out_stride < D) || (io->n && io->n_stride < D))
      return norm_fail(ctx, LCSM_EINVAL, "a row stride is shorter than the row");
  }
  if (ctx->faulted) return LCSM_ESTATE;
  if (!rows) return LCSM_OK;
  const float* w[5];
  for (int k = 0; k < 5; ++k) {
    const bool used = k == 2 || (k < 2 ? s.post : s.pre) != LCSM_NORM_NONE;
    w[k] = ctx->w[k] && used ? ctx->w[k] + (size_t)layer * D : nullptr;
  }
  const lcsm::NormCall c{rows, s.D, s.groups, s.post, s.pre, s.act, s.alpha, s.eps,
                         io->o, io->g, io->r, io->r_out, io->n,
                         io->o_stride, io->g_stride, io->r_stride, io->r_out_stride, io->n_stride,
                         w[0], w[1], w[2], w[3], w[4]};
  const hipError_t e = lcsm::with_dtype(s.dtype, [&](auto v) {
    typedef decltype(v) E;
    return s.res_dtype == LCSM_F32 ? lcsm::launch_norm<E, float>(c, ctx->stream)
                                   : lcsm::launch_norm<E, E>(c, ctx->stream);
  });
  return e == hipSuccess ? LCSM_OK : norm_fail(ctx, LCSM_EDEVICE, "norm launch", e);
}

int lcsm_norm_reset(lcsm_norm* ctx) {
  if (!ctx) return LCSM_EINVAL;
  ctx->faulted = false;
  ctx->msg[0] = 0;
  return LCSM_OK;
}

void lcsm_norm_destroy(lcsm_norm* ctx) {
  if (!ctx) return;
  (void)hipStreamSynchronize(ctx->stream);
  if (ctx->mem) (void)hipFree(ctx->mem);
  delete ctx;
}

const char* lcsm_norm_last_error(const lcsm_norm* ctx) { return ctx ? ctx->msg : ""; }

}  // extern "C"
