// Linear attention with a decay for each head: the context, and single tokens.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>

#include "lcsm_internal.h"
#include "lcsm_lin_internal.h"

namespace lcsm {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kLinMaxK = 256;
constexpr int kLinMaxV = 4096;
constexpr int kLinMaxSlots = 32768;

// One token of each sequence: S' = d S + k v^T and y = scale q S'.  A workgroup
// takes 4 VL values of a state, a thread four of them and every 256 / VL'th key, J
// keys in all: the state is read once, changed in registers, and written.  The
// sums over the keys of a head's outputs are taken over the lanes of a wave that
// have the same values, then over the waves in LDS.
//
// Bound by the states: 64 tokens of 32 states of 128 x 128 take 46 us, 5.9 TB/s of
// reads and writes together, part of them in the memory's cache; one token of 16
// states takes 4.4 us, a launch and a round trip.
template <class E, int VL, int J>
__global__ __launch_bounds__(256) void k_lin_step(LinCall c) {
  constexpr int KR = 256 / VL, VB = 4 * VL;
  __shared__ __align__(16) float sq[kLinMaxK], sk[kLinMaxK];
  __shared__ __align__(16) float sy[4][VB];
  const int i = (int)blockIdx.z, g = (int)blockIdx.y, heads = c.H / c.G;
  const int tid = (int)threadIdx.x, vl = tid % VL, kr = tid / VL;
  const int v = (int)blockIdx.x * VB + 4 * vl;
  const int s = lin_slot(c.src, i, c.slots), d = lin_slot(c.dst, i, c.slots);
  const size_t each = (size_t)c.K * c.V;
  const bool quads = c.V % 4 == 0;
  v4f S[J];
#pragma unroll
  for (int j = 0; j < J; ++j) {
    S[j] = v4f{0.f, 0.f, 0.f, 0.f};
    const int k = kr + j * KR;
    if (s < 0 || k >= c.K || v >= c.V) continue;
    // states pass through once a call: not kept in the caches
    const float* at = c.state + ((size_t)s * c.G + g) * each + (size_t)k * c.V + v;
    if (quads) {
      S[j] = __builtin_nontemporal_load(reinterpret_cast<const v4f*>(at));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v + e < c.V) S[j][e] = at[e];
    }
  }
  const E* kp = static_cast<const E*>(c.k) + (size_t)i * c.k_stride + (size_t)g * c.K;
  const E* vp = static_cast<const E*>(c.v) + (size_t)i * c.v_stride + (size_t)g * c.V;
  const E* qp = static_cast<const E*>(c.q) + (size_t)i * c.q_stride + (size_t)g * heads * c.K;
  E* yp = static_cast<E*>(c.y) + (size_t)i * c.y_stride + (size_t)g * heads * c.V;
  if (tid < c.K) sk[tid] = (float)kp[tid], sq[tid] = (float)qp[tid];
  float x[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) x[e] = v + e < c.V ? (float)vp[v + e] : 0.f;
  const LinDecay decay((double)c.decay[g]);
  __syncthreads();
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int k = kr + j * KR;
    if (k >= c.K) continue;
    const float key = sk[k];
#pragma unroll
    for (int e = 0; e < 4; ++e) S[j][e] = fmaf(key, x[e], decay(S[j][e]));
    if (d < 0 || v >= c.V) continue;
    float* at = c.state + ((size_t)d * c.G + g) * each + (size_t)k * c.V + v;
    if (quads) {
      __builtin_nontemporal_store(S[j], reinterpret_cast<v4f*>(at));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (v + e < c.V) at[e] = S[j][e];
    }
  }
  for (int h = 0; h < heads; ++h) {
    if (h > 0) {
      __syncthreads();  // the head before has been summed
      if (tid < c.K) sq[tid] = (float)qp[(size_t)h * c.K + tid];
      __syncthreads();
    }
    v4f y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int k = kr + j * KR;
      if (k >= c.K) continue;
      const float f = sq[k];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fmaf(f, S[j][e], y[e]);
    }
#pragma unroll
    for (int m = VL; m < 64; m *= 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] += __shfl_xor(y[e], m);
    if (tid % 64 < VL) *reinterpret_cast<v4f*>(&sy[tid / 64][4 * vl]) = y;
    __syncthreads();
    const int at = (int)blockIdx.x * VB + tid;
    if (tid < VB && at < c.V)
      yp[(size_t)h * c.V + at] = (E)(c.scale * ((sy[0][tid] + sy[1][tid]) + (sy[2][tid] + sy[3][tid])));
  }
}

template <class E, int VL, int J>
hipError_t launch_step_of(const LinCall& c, hipStream_t st) {
  hipLaunchKernelGGL((k_lin_step<E, VL, J>), dim3((unsigned)((c.V + 4 * VL - 1) / (4 * VL)), (unsigned)c.G, (unsigned)c.n),
                     dim3(256), 0, st, c);
  return hipGetLastError();
}
// Workgroups of 128 values where these are enough for the card, else of 32.  us of
// 128 and 32 by their number, states of 128 x 128, bf16:
//     16  8.2  4.4   256   9.8   7.4    512  11.5  11.1
//   1024 20.3 26.0  2048  46.9  51.7   8192 205   200
template <class E>
hipError_t launch_step(const LinCall& c, hipStream_t st) {
  if (c.V > 32 && (long long)c.n * c.G * ((c.V + 127) / 128) >= 1024)
    return c.K <= 128 ? launch_step_of<E, 32, 16>(c, st) : launch_step_of<E, 32, 32>(c, st);
  return c.K <= 128 ? launch_step_of<E, 8, 4>(c, st) : launch_step_of<E, 8, 8>(c, st);
}

// How a prompt call is cut: segments of `per` chunks so that about as many
// workgroups are on their way as there is room for at once (two or one a compute
// unit; half, one and a half and twice as many are slower at 16384 tokens);
// sequences that are that many by themselves are not cut, however unequal they are: 32
// states of 128 x 128, bf16, one of 16384 tokens beside fourteen of 33 253 to 259 us,
// beside fifteen, which is the limit there, 1515 (sixteen of 1024, uncut, 166 to 184,
// fifteen, cut, 174 to 182).
//
// Calls of up to so many chunks are not cut either, since cutting takes two more
// launches.  us cut and uncut, 32 states of 128 x 128, bf16 (chunks of 64): 96 tokens
// 25.2 and 18.6, 160 27.3 and 24.1, 256 29.5 and 28.4; fp32 (chunks of 32): 48 tokens
// 25.0 and 17.2, 96 27.1 and 22.3, fp16 96 26.0 and 19.9.
constexpr int kLinCutChunks = 4;
int lin_want(int G, int K, int V) {
  const long long wgs = (long long)G * ((V + 32 * kLinWaves - 1) / (32 * kLinWaves));
  return (int)((K > 128 ? 256 : 512) / (wgs < 512 ? wgs : 512));
}

hipError_t launch_prompt(const LinCall& c, int dtype, float* states, hipStream_t st) {
  LinCut w;
  const int blocks = c.T / lin_chunk_of(dtype, c.K) + c.n;  // a sequence's last chunk may be short
  const int want = lin_want(c.G, c.K, c.V);
  const bool cut = want > c.n && c.T > kLinCutChunks * lin_chunk_of(dtype, c.K);
  w.states = states;
  w.per = cut ? (blocks + want - 1) / want : blocks;
  w.segments = cut ? blocks / w.per + c.n : c.n;
  const size_t e = dtype_size(dtype);
  auto aligned = [&](const void* p, size_t stride, int width, int n) {
    return (uintptr_t)p % (n * e) == 0 && stride % n == 0 && width % n == 0;
  };
  w.direct = e == 2 && aligned(c.q, c.q_stride, c.K, 8) && aligned(c.k, c.k_stride, c.K, 8) && aligned(c.v, c.v_stride, c.V, 8);
  w.wide = e == 2 && aligned(c.y, c.y_stride, c.V, 8) ? 8 : aligned(c.y, c.y_stride, c.V, 4) ? 4 : 1;
  return dtype == LCSM_F32 ? lin_prompt_f32(c, w, st) : dtype == LCSM_BF16 ? lin_prompt_bf16(c, w, st) : lin_prompt_f16(c, w, st);
}

}  // namespace
}  // namespace lcsm

struct lcsm_lin {
  lcsm_lin_shape s;
  hipStream_t stream;
  void* owned;
  float *state, *decay, *segments;
  size_t floats;  // of all states
  bool faulted;
  char msg[256];
};

namespace {

struct Plan {
  size_t state, decay, segments, total;
};

bool lin_plan(const lcsm_lin_shape* s, Plan* p) {
  if (!s || s->M < 1 || s->M > 16384 || s->slots < 1 || s->slots > lcsm::kLinMaxSlots || s->H < 1 || s->H > 65535 ||
      s->G < 1 || s->H % s->G || s->K < 1 || s->K > lcsm::kLinMaxK || s->V < 1 || s->V > lcsm::kLinMaxV ||
      !lcsm::dtype_ok(s->dtype) || s->max_tokens < 0 || s->max_tokens > (1 << 26) || !isfinite(s->scale))
    return false;
  for (int r : s->reserved)
    if (r) return false;
  const double ms = (double)s->M * s->slots, each = (double)s->G * s->K * s->V * 4;
  if ((double)s->H * (s->K + s->V) > (1 << 24) || ms * each > 70368744177664.0) return false;
  size_t at = 0;
  auto take = [&](size_t* where, size_t bytes) {
    *where = at;
    at = (at + bytes + 255) / 256 * 256;
  };
  take(&p->state, (size_t)s->M * s->slots * (size_t)each);
  take(&p->decay, (size_t)s->M * s->G * 4);
  p->segments = 0;
  if (s->max_tokens > 0) {
    // fewer than `want` pieces of all chunks and one more for each of fewer than
    // `want` sequences; calls of as many sequences are not cut
    const size_t chunks = (size_t)s->max_tokens / lcsm::lin_chunk_of(s->dtype, s->K) + s->slots;
    size_t most = 2 * (size_t)lcsm::lin_want(s->G, s->K, s->V) + 2;
    if (most > chunks + s->slots) most = chunks + s->slots;
    if ((double)most * each > 70368744177664.0) return false;
    take(&p->segments, most * (size_t)each);
  }
  p->total = at;
  return true;
}

int lin_fail(lcsm_lin* c, int code, const char* what, hipError_t e = hipSuccess) {
  if (e != hipSuccess) {
    snprintf(c->msg, sizeof(c->msg), "%s: %s", what, hipGetErrorString(e));
    c->faulted = true;
    return LCSM_EDEVICE;
  }
  snprintf(c->msg, sizeof(c->msg), "%s", what);
  return code;
}

// Checks the arguments of a call and lays them out for the kernels.
int lin_call(lcsm_lin* c, int layer, int T, int n, const lcsm_lin_io* io, lcsm::LinCall* k) {
  const lcsm_lin_shape& s = c->s;
  if (layer < 0 || layer >= s.M) return lin_fail(c, LCSM_EINVAL, "layer out of range");
  if (n < 0 || n > s.slots) return lin_fail(c, LCSM_EINVAL, "more sequences than slots");
  if (!io) return lin_fail(c, LCSM_EINVAL, "null io");
  if (T > 0 && n > 0) {
    if (!io->q || !io->k || !io->v || !io->y) return lin_fail(c, LCSM_EINVAL, "null input or output pointer");
    if (io->q_stride < (size_t)s.H * s.K || io->k_stride < (size_t)s.G * s.K || io->v_stride < (size_t)s.G * s.V ||
        io->y_stride < (size_t)s.H * s.V)
      return lin_fail(c, LCSM_EINVAL, "a row stride is shorter than the row");
    for (size_t stride : {io->q_stride, io->k_stride, io->v_stride, io->y_stride})
      if (stride > lcsm::kMaxStride) return lin_fail(c, LCSM_EINVAL, "a row stride is above 2^24 elements");
  }
  if (c->faulted) return LCSM_ESTATE;
  const size_t m = (size_t)layer;
  *k = lcsm::LinCall{s.H, s.G, s.K, s.V, s.slots, T, n, s.scale, nullptr, io->src, io->dst, io->q, io->k, io->v, io->y,
                     io->q_stride, io->k_stride, io->v_stride, io->y_stride, c->decay + m * s.G,
                     c->state + m * s.slots * (size_t)s.G * s.K * s.V};
  return LCSM_OK;
}

}  // namespace

extern "C" {

int lcsm_lin_workspace_bytes(const lcsm_lin_shape* shape, size_t* bytes) {
  Plan p;
  if (!bytes || !lin_plan(shape, &p)) return LCSM_EINVAL;
  *bytes = p.total;
  return LCSM_OK;
}

int lcsm_lin_init(lcsm_lin** out, const lcsm_lin_shape* shape, const float* decay, void* stream,
                  void* workspace, size_t workspace_bytes) {
  if (!out) return LCSM_EINVAL;
  *out = nullptr;
  Plan p;
  if (!decay || !lin_plan(shape, &p)) return LCSM_EINVAL;
  if (workspace && ((uintptr_t)workspace & 255)) return LCSM_EINVAL;
  if (workspace && workspace_bytes < p.total) return LCSM_ENOMEM;
  lcsm_lin* c = new (std::nothrow) lcsm_lin();
  if (!c) return LCSM_ENOMEM;
  c->s = *shape;
  c->stream = (hipStream_t)stream;
  if (!workspace) {
    if (hipMalloc(&c->owned, p.total) != hipSuccess) {
      (void)hipGetLastError();
      delete c;
      return LCSM_ENOMEM;
    }
    workspace = c->owned;
  }
  char* mem = (char*)workspace;
  c->state = (float*)(mem + p.state);
  c->decay = (float*)(mem + p.decay);
  c->segments = (float*)(mem + p.segments);
  c->floats = (size_t)shape->M * shape->slots * shape->G * shape->K * shape->V;
  hipError_t e = lcsm::launch_zero(c->state, c->floats, c->stream);
  if (e == hipSuccess)
    e = hipMemcpyAsync(c->decay, decay, (size_t)shape->M * shape->G * 4, hipMemcpyDeviceToDevice, c->stream);
  if (e != hipSuccess) {
    (void)hipGetLastError();
    (void)hipStreamSynchronize(c->stream);
    if (c->owned) (void)hipFree(c->owned);
    delete c;
    return LCSM_EDEVICE;
  }
  *out = c;
  return LCSM_OK;
}

int lcsm_lin_step_layer(lcsm_lin* ctx, int layer, int n, const lcsm_lin_io* io) {
  if (!ctx) return LCSM_EINVAL;
  lcsm::LinCall k;
  int r = lin_call(ctx, layer, n, n, io, &k);
  if (r || !n) return r;
  const hipError_t e =
      lcsm::with_dtype(ctx->s.dtype, [&](auto v) { return lcsm::launch_step<decltype(v)>(k, ctx->stream); });
  return e == hipSuccess ? LCSM_OK : lin_fail(ctx, LCSM_EDEVICE, "step launch", e);
}

int lcsm_lin_prompt_layer(lcsm_lin* ctx, int layer, int T, int n, const int* offsets,
                          const lcsm_lin_io* io) {
  if (!ctx) return LCSM_EINVAL;
  if (T < 0 || T > ctx->s.max_tokens) return lin_fail(ctx, LCSM_EINVAL, "tokens out of range");
  if (!offsets && n != 1) return lin_fail(ctx, LCSM_EINVAL, "offsets are needed for n sequences");
  lcsm::LinCall k;
  int r = lin_call(ctx, layer, T, n, io, &k);
  if (r || !n) return r;
  k.offsets = offsets;
  const hipError_t e = lcsm::launch_prompt(k, ctx->s.dtype, ctx->segments, ctx->stream);
  return e == hipSuccess ? LCSM_OK : lin_fail(ctx, LCSM_EDEVICE, "prompt launch", e);
}

int lcsm_lin_state(lcsm_lin* ctx, int layer, float** state) {
  if (!ctx || !state || layer < 0 || layer >= ctx->s.M) return LCSM_EINVAL;
  *state = ctx->state + (size_t)layer * ctx->s.slots * ctx->s.G * ctx->s.K * ctx->s.V;
  return LCSM_OK;
}

int lcsm_lin_reset(lcsm_lin* ctx) {
  if (!ctx) return LCSM_EINVAL;
  const hipError_t e = lcsm::launch_zero(ctx->state, ctx->floats, ctx->stream);
  if (e != hipSuccess) return lin_fail(ctx, LCSM_EDEVICE, "reset", e);
  ctx->faulted = false;
  ctx->msg[0] = 0;
  return LCSM_OK;
}

void lcsm_lin_destroy(lcsm_lin* ctx) {
  if (!ctx) return;
  (void)hipStreamSynchronize(ctx->stream);
  if (ctx->owned) (void)hipFree(ctx->owned);
  delete ctx;
}

const char* lcsm_lin_last_error(const lcsm_lin* ctx) { return ctx ? ctx->msg : ""; }

}  // extern "C"
