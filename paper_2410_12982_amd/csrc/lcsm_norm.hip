// Norms around a block with its gate, residual scale and sum (lcsm_norm.h).
//
// A row is held in the registers of TPR threads from its first load to its last
// store, so that it is read and written once; the statistics are sums over
// those registers (the variance a second sum, of the differences from the
// mean).
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

// VEC consecutive elements from p, which VEC = 8 has aligned to 16 bytes.
template <int VEC, class E>
__device__ __forceinline__ void load(const E* p, float (&v)[VEC]) {
  struct alignas(VEC == 1 ? sizeof(E) : 16) Pack {
    E e[VEC];
  };
  const Pack k = *reinterpret_cast<const Pack*>(p);
#pragma unroll
  for (int i = 0; i < VEC; ++i) v[i] = (float)k.e[i];
}
template <int VEC, class E>
__device__ __forceinline__ void store(E* p, const float (&v)[VEC]) {
  struct alignas(VEC == 1 ? sizeof(E) : 16) Pack {
    E e[VEC];
  } k;
#pragma unroll
  for (int i = 0; i < VEC; ++i) k.e[i] = (E)v[i];
  *reinterpret_cast<Pack*>(p) = k;
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

template <class E, class RE, int VEC, int NV, int TPR, bool GROUPED>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void k_norm(NormCall c) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;  // rows a workgroup
  constexpr int FP = VEC * NV;
  __shared__ float part[TPR / 64];
  extern __shared__ float lds[];  // GROUPED: the row, then mean and factor of every group
  const int lane = (int)threadIdx.x % TPR;
  const int row = (int)blockIdx.x * RPB + (int)threadIdx.x / TPR;
  // rows past the last one are computed again by whoever takes them, and not
  // stored: every thread meets every barrier
  const bool live = row < c.rows;
  const size_t at = (size_t)(live ? row : c.rows - 1);
  const int D = c.D;
  auto index = [&](int k) { return (k * TPR + lane) * VEC; };

  float v[FP], res[FP];
  {
    const RE* r = static_cast<const RE*>(c.r) + at * c.r_stride;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float t[VEC] = {};
      if (index(k) < D) load<VEC>(r + index(k), t);
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
        load<VEC>(o + index(k), t);
        if (c.act != LCSM_ACT_NONE) load<VEC>(g + index(k), u);
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
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int e = 0; e < VEC; ++e)
            if (index(k) + e < D) lds[index(k) + e] = v[k * VEC + e];
        __syncthreads();
        for (int q = (int)threadIdx.x / 64; q < c.groups; q += TPR / 64) {
          const float* x = lds + q * per;
          float mean = 0.f, var = 0.f;
          if (c.post == LCSM_NORM_LAYER) {
            for (int i = (int)threadIdx.x % 64; i < per; i += 64) mean += x[i];
            mean = row_sum<64>(mean, nullptr) / per;
          }
          for (int i = (int)threadIdx.x % 64; i < per; i += 64) var += (x[i] - mean) * (x[i] - mean);
          var = row_sum<64>(var, nullptr) / per;
          if (threadIdx.x % 64 == 0) {
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
          for (int i = 0; i < FP; ++i) mean += v[i];
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
      if (c.post_w) load<VEC>(c.post_w + index(k), w);
      if (c.post_b) load<VEC>(c.post_b + index(k), b);
      if (c.scale) load<VEC>(c.scale + index(k), s);
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        res[k * VEC + e] = fmaf(s[e], fmaf(v[k * VEC + e], w[e], b[e]), res[k * VEC + e]);
    }
  }
  if (c.r_out && live) {
    RE* r = static_cast<RE*>(c.r_out) + at * c.r_out_stride;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float t[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) t[e] = res[k * VEC + e];
      if (index(k) < D) store<VEC>(r + index(k), t);
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
    if (c.pre_w) load<VEC>(c.pre_w + index(k), w);
    if (c.pre_b) load<VEC>(c.pre_b + index(k), b);
#pragma unroll
    for (int e = 0; e < VEC; ++e) t[e] = fmaf((res[k * VEC + e] - mean) * f, w[e], b[e]);
    store<VEC>(n + index(k), t);
  }
}

template <class E, class RE, int VEC, int NV, int TPR>
hipError_t launch(const NormCall& c, hipStream_t st) {
  constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
  const dim3 grid((unsigned)((c.rows + RPB - 1) / RPB)), block(TPR < 256 ? 256 : TPR);
  if constexpr (TPR > 64) {
    if (c.groups > 1 && c.o && c.post != LCSM_NORM_NONE) {
      const size_t bytes = ((size_t)c.D + 2 * (size_t)c.groups) * sizeof(float);
      auto kernel = k_norm<E, RE, VEC, NV, TPR, true>;
      if (bytes > 65536 - 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != hipSuccess) return e;
      }
      hipLaunchKernelGGL(kernel, grid, block, bytes, st, c);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((k_norm<E, RE, VEC, NV, TPR, false>), grid, block, 0, st, c);
  return hipGetLastError();
}

// A wave holds a row of up to 2048 values, 256 threads one of up to 8192 and
// 1024 threads the longest; parts normed on their own meet in LDS, which the
// rows of a workgroup do not share.
template <class E, class RE, int VEC>
hipError_t launch_vec(const NormCall& c, hipStream_t st) {
  const bool wave = c.D <= 2048 && (c.groups == 1 || !c.o || c.post == LCSM_NORM_NONE);
  if (wave) {
    if (c.D <= 512) return launch<E, RE, VEC, 8 / VEC, 64>(c, st);
    return launch<E, RE, VEC, 32 / VEC, 64>(c, st);
  }
  if (c.D <= 2048) return launch<E, RE, VEC, 8 / VEC, 256>(c, st);
  if (c.D <= 8192) return launch<E, RE, VEC, 32 / VEC, 256>(c, st);
  return launch<E, RE, VEC, 32 / VEC, 1024>(c, st);
}

bool aligned(const void* p, size_t stride, size_t elem) {
  return !p || (((uintptr_t)p & 15) == 0 && stride * elem % 16 == 0);
}

template <class E, class RE>
hipError_t launch_norm(const NormCall& c, hipStream_t st) {
  const bool vec = c.D % 8 == 0 && aligned(c.o, c.o_stride, sizeof(E)) &&
                   aligned(c.g, c.g_stride, sizeof(E)) && aligned(c.n, c.n_stride, sizeof(E)) &&
                   aligned(c.r, c.r_stride, sizeof(RE)) && aligned(c.r_out, c.r_out_stride, sizeof(RE));
  return vec ? launch_vec<E, RE, 8>(c, st) : launch_vec<E, RE, 1>(c, st);
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
