// The selective state space mixer with its short causal convolution: the
// context, and the scan position by position.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>

#include "lcsm_internal.h"
#include "lcsm_ssm_internal.h"

namespace lcsm {
namespace {

constexpr int kSsmMaxN = 256;
constexpr int kSsmMaxW = 4;
constexpr int kScanRows = 16;  // channels of a head a workgroup takes

// The short convolution of channel ch at row t of a sequence that begins at
// row t0: taps before t0 from the window of slot s (s < 0: zeros).
template <class E>
__device__ __forceinline__ float ssm_conv(const SsmCall& c, int ch, int t, int t0, int s) {
  const E* x = static_cast<const E*>(c.xbc);
  const E* w = static_cast<const E*>(c.window);
  float a = c.conv_b[ch];
  for (int k = 0; k < c.W; ++k) {
    const int tt = t - c.W + 1 + k;
    float v = 0.f;
    if (tt >= t0)
      v = (float)x[(size_t)tt * c.xbc_stride + ch];
    else if (s >= 0)
      v = (float)w[((size_t)s * (c.W - 1) + (tt - t0 + c.W - 1)) * c.C + ch];
    a = fmaf(c.conv_w[(size_t)ch * c.W + k], v, a);
  }
  return silu(a);
}

// The recurrence as it is written, one workgroup per sequence, head and
// kScanRows channels.  L lanes hold the states of a channel, four of every 4 L
// of them each.
template <class E, int L>
__global__ __launch_bounds__(256) void k_ssm_scan(SsmCall c) {
  constexpr int RPP = 256 / L;  // channels side by side
  constexpr int R = kScanRows > RPP ? kScanRows / RPP : 1;
  __shared__ float su[2][kScanRows + 2 * kSsmMaxN];
  const int i = (int)blockIdx.x, h = (int)blockIdx.y, p0 = (int)blockIdx.z * kScanRows;
  const int tid = (int)threadIdx.x, n0 = tid % L * 4, r0 = tid / L;
  const int g = h / (c.H / c.G);
  int t0, t1;
  ssm_rows(c, i, t0, t1);
  const int s = ssm_slot(c.src, i, c.slots), d = ssm_slot(c.dst, i, c.slots);
  float S[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int p = p0 + r0 + r * RPP;
      const bool in = r0 + r * RPP < kScanRows && p < c.P && n0 + e < c.N;
      S[r][e] = in && s >= 0 ? c.state[(((size_t)s * c.H + h) * c.P + p) * c.N + n0 + e] : 0.f;
    }
  for (int t = t0; t < t1; ++t) {
    float* u = su[t & 1];
    for (int k = tid; k < kScanRows + 2 * c.N; k += 256) {
      int ch;
      bool in = true;
      if (k < kScanRows) {
        in = p0 + k < c.P;
        ch = h * c.P + p0 + k;
      } else {
        const int j = k - kScanRows;
        ch = c.D + (j < c.N ? g * c.N + j : c.G * c.N + g * c.N + j - c.N);
      }
      u[k] = in ? ssm_conv<E>(c, ch, t, t0, s) : 0.f;
    }
    const float step = softplus((float)static_cast<const E*>(c.dt)[(size_t)t * c.dt_stride + h] +
                                c.dt_bias[h]);
    const float decay = __expf(step * c.A[h]);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int q = r0 + r * RPP, p = p0 + q;
      const float x = q < kScanRows ? u[q] : 0.f;
      float y = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n0 + e < c.N) {
          S[r][e] = fmaf(S[r][e], decay, step * x * u[kScanRows + n0 + e]);
          y = fmaf(S[r][e], u[kScanRows + c.N + n0 + e], y);
        }
#pragma unroll
      for (int m = 1; m < L; m *= 2) y += __shfl_xor(y, m);
      if (tid % L == 0 && q < kScanRows && p < c.P) {
        const int ch = h * c.P + p;
        y = fmaf(c.skip[h], x, y);
        if (c.z) y *= silu((float)static_cast<const E*>(c.z)[(size_t)t * c.z_stride + ch]);
        static_cast<E*>(c.y)[(size_t)t * c.y_stride + ch] = (E)y;
      }
    }
  }
  if (d < 0) return;
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int p = p0 + r0 + r * RPP;
      if (r0 + r * RPP < kScanRows && p < c.P && n0 + e < c.N)
        c.state[(((size_t)d * c.H + h) * c.P + p) * c.N + n0 + e] = S[r][e];
    }
}

// The windows after a call: a thread per sequence and channel.
template <class E>
__global__ __launch_bounds__(256) void k_ssm_window(SsmCall c) {
  const int ch = (int)blockIdx.x * 256 + (int)threadIdx.x, i = (int)blockIdx.y;
  if (ch >= c.C) return;
  int t0, t1;
  ssm_rows(c, i, t0, t1);
  const int s = ssm_slot(c.src, i, c.slots), d = ssm_slot(c.dst, i, c.slots);
  if (d < 0) return;
  const E* x = static_cast<const E*>(c.xbc);
  E* w = static_cast<E*>(c.window);
  E v[kSsmMaxW - 1];
#pragma unroll
  for (int k = 0; k < kSsmMaxW - 1; ++k) {
    v[k] = (E)0.f;
    if (k >= c.W - 1) continue;
    const int tt = t1 - (c.W - 1) + k;
    if (tt >= t0)
      v[k] = x[(size_t)tt * c.xbc_stride + ch];
    else if (s >= 0)
      v[k] = w[((size_t)s * (c.W - 1) + (tt - t0 + c.W - 1)) * c.C + ch];
  }
#pragma unroll
  for (int k = 0; k < kSsmMaxW - 1; ++k)
    if (k < c.W - 1) w[((size_t)d * (c.W - 1) + k) * c.C + ch] = v[k];
}

template <class E>
hipError_t launch_scan(const SsmCall& c, hipStream_t st) {
  const dim3 grid((unsigned)c.n, (unsigned)c.H, (unsigned)((c.P + kScanRows - 1) / kScanRows));
  if (c.N > 128)
    hipLaunchKernelGGL((k_ssm_scan<E, 64>), grid, dim3(256), 0, st, c);
  else if (c.N > 64)
    hipLaunchKernelGGL((k_ssm_scan<E, 32>), grid, dim3(256), 0, st, c);
  else
    hipLaunchKernelGGL((k_ssm_scan<E, 16>), grid, dim3(256), 0, st, c);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || c.W == 1) return e;
  hipLaunchKernelGGL(k_ssm_window<E>, dim3((unsigned)((c.C + 255) / 256), (unsigned)c.n), dim3(256),
                     0, st, c);
  return hipGetLastError();
}

// How a prompt call is cut: segments of `per` chunks so that about one
// workgroup per compute unit is on its way, which is what LDS holds; sequences
// that are that many by themselves are not cut.
constexpr int kSsmWorkgroups = 256;

int head_groups(int H, int G, int P, int N) {
  const int items = H / G * ((P + 31) / 32), nw = items < ssm_waves(N) ? items : ssm_waves(N);
  return G * ((items + nw - 1) / nw);
}
// Upper bound of the segments of a call that is cut: fewer than `want` pieces
// of all chunks and one more for each of fewer than `want` sequences; `cuts`:
// chunks and sequences of the largest call.
size_t most_segments(int H, int G, int P, int N, size_t cuts) {
  const size_t most = 2 * (size_t)kSsmWorkgroups / head_groups(H, G, P, N) + 2;
  return most < cuts ? most : cuts;
}

hipError_t launch_prompt(const SsmCall& c, int dtype, SsmScratch w, hipStream_t st) {
  w.blocks = c.T / kSsmQ + c.n;  // a sequence's last chunk may be short
  const int wgs = head_groups(c.H, c.G, c.P, c.N), want = kSsmWorkgroups / wgs;
  w.per = want > c.n ? (w.blocks + want - 1) / want : w.blocks;
  w.segments = want > c.n ? w.blocks / w.per + c.n : c.n;
  const size_t e = dtype_size(dtype);
  auto two = [&](const void* p, size_t stride) { return !p || ((uintptr_t)p % (2 * e) == 0 && stride % 2 == 0); };
  w.pair = c.P % 2 == 0 && two(c.xbc, c.xbc_stride) && two(c.z, c.z_stride) && two(c.y, c.y_stride);
  w.quads = c.N % 4 == 0;
  if (c.T == 0) w.blocks = 0;
  hipError_t r = dtype == LCSM_F32 ? ssm_prompt_f32(c, w, st)
                 : dtype == LCSM_BF16 ? ssm_prompt_bf16(c, w, st) : ssm_prompt_f16(c, w, st);
  if (r != hipSuccess || c.W == 1) return r;
  const dim3 grid((unsigned)((c.C + 255) / 256), (unsigned)c.n);
  with_dtype(dtype, [&](auto v) {
    hipLaunchKernelGGL(k_ssm_window<decltype(v)>, grid, dim3(256), 0, st, c);
    return 0;
  });
  return hipGetLastError();
}

}  // namespace
}  // namespace lcsm

struct lcsm_ssm {
  lcsm_ssm_shape s;
  int D, C;
  hipStream_t stream;
  char* mem;
  void* owned;
  float *state, *conv_w, *conv_b, *A, *skip, *dt_bias;
  char* window;
  lcsm::SsmScratch scratch;
  size_t zero_floats;  // states and windows, from `state` on
  bool faulted;
  char msg[256];
};

namespace {

size_t align256(size_t v) { return (v + 255) / 256 * 256; }

struct Plan {
  size_t state, window, conv_w, conv_b, A, skip, dt_bias, bc, scal, lq, states, decay, total;
};

bool ssm_plan(const lcsm_ssm_shape* s, Plan* p) {
  if (!s || s->M < 1 || s->slots < 1 || s->H < 1 || s->P < 1 || s->N < 1 || s->G < 1 || s->W < 1)
    return false;
  if (s->P > 4096 || s->N > lcsm::kSsmMaxN || s->W > lcsm::kSsmMaxW || s->H % s->G || !lcsm::dtype_ok(s->dtype))
    return false;
  if (s->M > 16384 || s->slots > 65535 || s->max_tokens < 0 || s->max_tokens > (1 << 26)) return false;
  for (int r : s->reserved)
    if (r) return false;
  const double D = (double)s->H * s->P, C = D + 2.0 * s->G * s->N, ms = (double)s->M * s->slots;
  if (C > (1 << 24) || s->H > 65535 || ms * D * s->N * 4 + ms * C * 16 + s->M * C * 20 > 70368744177664.0)
    return false;
  const size_t M = (size_t)s->M, MS = M * s->slots, c = (size_t)C, H = (size_t)s->H;
  size_t at = 0;
  auto take = [&](size_t* where, size_t bytes) {
    *where = at;
    at = align256(at + bytes);
  };
  take(&p->state, MS * (size_t)D * s->N * 4);
  take(&p->window, MS * (s->W - 1) * c * lcsm::dtype_size(s->dtype));
  take(&p->conv_w, M * c * s->W * 4);
  take(&p->conv_b, M * c * 4);
  take(&p->A, M * H * 4);
  take(&p->skip, M * H * 4);
  take(&p->dt_bias, M * H * 4);
  if (s->max_tokens) {
    const size_t blocks = (size_t)s->max_tokens / lcsm::kSsmQ + s->slots;
    const size_t each = lcsm::ssm_block_bytes(s->N, lcsm::dtype_size(s->dtype));
    const size_t segments = lcsm::most_segments(s->H, s->G, s->P, s->N, blocks + s->slots);
    if ((double)blocks * (s->G * (double)each + H * 2048.0) + (double)segments * D * s->N * 4 > 70368744177664.0)
      return false;
    take(&p->bc, blocks * s->G * each);
    take(&p->scal, blocks * H * 4 * lcsm::kSsmQ * 4);
    take(&p->lq, blocks * H * 16);
    take(&p->states, segments * (size_t)D * s->N * 4);
    take(&p->decay, segments * H * 4);
  }
  p->total = at;
  return true;
}

int ssm_fail(lcsm_ssm* c, int code, const char* what, hipError_t e = hipSuccess) {
  if (e != hipSuccess) {
    snprintf(c->msg, sizeof(c->msg), "%s: %s", what, hipGetErrorString(e));
    c->faulted = true;
    return LCSM_EDEVICE;
  }
  snprintf(c->msg, sizeof(c->msg), "%s", what);
  return code;
}

// Checks the arguments of a call and lays them out for the kernels.
int ssm_call(lcsm_ssm* c, int layer, int T, int n, const lcsm_ssm_io* io, lcsm::SsmCall* k) {
  if (layer < 0 || layer >= c->s.M) return ssm_fail(c, LCSM_EINVAL, "layer out of range");
  if (n < 0 || n > c->s.slots) return ssm_fail(c, LCSM_EINVAL, "more sequences than slots");
  if (!io) return ssm_fail(c, LCSM_EINVAL, "null io");
  if (T > 0 && n > 0) {
    if (!io->xbc || !io->dt || !io->y) return ssm_fail(c, LCSM_EINVAL, "null input or output pointer");
    if (io->xbc_stride < (size_t)c->C || io->dt_stride < (size_t)c->s.H || io->y_stride < (size_t)c->D ||
        (io->z && io->z_stride < (size_t)c->D))
      return ssm_fail(c, LCSM_EINVAL, "a row stride is shorter than the row");
    for (size_t stride : {io->xbc_stride, io->dt_stride, io->y_stride, io->z ? io->z_stride : 0})
      if (stride > lcsm::kSsmMaxStride) return ssm_fail(c, LCSM_EINVAL, "a row stride is above 2^25 elements");
  }
  if (c->faulted) return LCSM_ESTATE;
  const size_t m = (size_t)layer, C = (size_t)c->C, H = (size_t)c->s.H;
  *k = lcsm::SsmCall{c->s.H, c->s.P, c->s.N, c->s.G, c->s.W, c->D, c->C, c->s.slots, T, n,
                     0, nullptr, io->src, io->dst, io->xbc, io->dt, io->z, io->y,
                     io->xbc_stride, io->dt_stride, io->z_stride, io->y_stride,
                     c->conv_w + m * C * c->s.W, c->conv_b + m * C, c->A + m * H, c->skip + m * H,
                     c->dt_bias + m * H, c->state + m * c->s.slots * (size_t)c->D * c->s.N,
                     c->window + m * c->s.slots * (c->s.W - 1) * C * lcsm::dtype_size(c->s.dtype)};
  return LCSM_OK;
}

}  // namespace

extern "C" {

int lcsm_ssm_workspace_bytes(const lcsm_ssm_shape* shape, size_t* bytes) {
  Plan p;
  if (!bytes || !ssm_plan(shape, &p)) return LCSM_EINVAL;
  *bytes = p.total;
  return LCSM_OK;
}

int lcsm_ssm_init(lcsm_ssm** out, const lcsm_ssm_shape* shape, const float* conv_w,
                  const float* conv_b, const float* A, const float* skip, const float* dt_bias,
                  void* stream, void* workspace, size_t workspace_bytes) {
  if (!out) return LCSM_EINVAL;
  *out = nullptr;
  Plan p;
  if (!conv_w || !A || !ssm_plan(shape, &p)) return LCSM_EINVAL;
  if (workspace && ((uintptr_t)workspace & 255)) return LCSM_EINVAL;
  if (workspace && workspace_bytes < p.total) return LCSM_ENOMEM;
  lcsm_ssm* c = new (std::nothrow) lcsm_ssm();
  if (!c) return LCSM_ENOMEM;
  c->s = *shape;
  c->D = shape->H * shape->P;
  c->C = c->D + 2 * shape->G * shape->N;
  c->stream = (hipStream_t)stream;
  if (workspace) {
    c->mem = (char*)workspace;
  } else {
    if (hipMalloc(&c->owned, p.total) != hipSuccess) {
      (void)hipGetLastError();
      delete c;
      return LCSM_ENOMEM;
    }
    c->mem = (char*)c->owned;
  }
  c->state = (float*)(c->mem + p.state);
  c->window = c->mem + p.window;
  c->zero_floats = (p.conv_w - p.state) / 4;
  c->conv_w = (float*)(c->mem + p.conv_w);
  c->conv_b = (float*)(c->mem + p.conv_b);
  c->A = (float*)(c->mem + p.A);
  c->skip = (float*)(c->mem + p.skip);
  c->dt_bias = (float*)(c->mem + p.dt_bias);
  if (shape->max_tokens) {
    c->scratch.bc = c->mem + p.bc;
    c->scratch.scal = (float*)(c->mem + p.scal);
    c->scratch.lq = (double*)(c->mem + p.lq);
    c->scratch.states = (float*)(c->mem + p.states);
    c->scratch.decay = (float*)(c->mem + p.decay);
  }
  const size_t MC = (size_t)shape->M * c->C, MH = (size_t)shape->M * shape->H;
  const struct {
    float* dst;
    const float* src;
    size_t n;
  } copies[] = {{c->conv_w, conv_w, MC * shape->W}, {c->conv_b, conv_b, MC}, {c->A, A, MH},
                {c->skip, skip, MH}, {c->dt_bias, dt_bias, MH}};
  hipError_t e = lcsm::launch_zero(c->state, c->zero_floats, c->stream);
  for (const auto& k : copies) {
    if (e != hipSuccess) break;
    e = k.src ? hipMemcpyAsync(k.dst, k.src, k.n * 4, hipMemcpyDeviceToDevice, c->stream)
              : lcsm::launch_zero(k.dst, k.n, c->stream);
  }
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

int lcsm_ssm_step_layer(lcsm_ssm* ctx, int layer, int n, const lcsm_ssm_io* io) {
  if (!ctx) return LCSM_EINVAL;
  lcsm::SsmCall k;
  int r = ssm_call(ctx, layer, n, n, io, &k);
  if (r || !n) return r;
  k.step = 1;
  hipError_t e = lcsm::with_dtype(ctx->s.dtype, [&](auto v) {
    return lcsm::launch_scan<decltype(v)>(k, ctx->stream);
  });
  return e == hipSuccess ? LCSM_OK : ssm_fail(ctx, LCSM_EDEVICE, "step launch", e);
}

int lcsm_ssm_prompt_layer(lcsm_ssm* ctx, int layer, int T, int n, const int* offsets,
                          const lcsm_ssm_io* io) {
  if (!ctx) return LCSM_EINVAL;
  if (T < 0 || T > ctx->s.max_tokens) return ssm_fail(ctx, LCSM_EINVAL, "tokens out of range");
  if (!offsets && n != 1) return ssm_fail(ctx, LCSM_EINVAL, "offsets are needed for n sequences");
  lcsm::SsmCall k;
  int r = ssm_call(ctx, layer, T, n, io, &k);
  if (r || !n) return r;
  k.offsets = offsets;
  hipError_t e = lcsm::launch_prompt(k, ctx->s.dtype, ctx->scratch, ctx->stream);
  return e == hipSuccess ? LCSM_OK : ssm_fail(ctx, LCSM_EDEVICE, "prompt launch", e);
}

int lcsm_ssm_state(lcsm_ssm* ctx, int layer, float** state) {
  if (!ctx || !state || layer < 0 || layer >= ctx->s.M) return LCSM_EINVAL;
  *state = ctx->state + (size_t)layer * ctx->s.slots * (size_t)ctx->D * ctx->s.N;
  return LCSM_OK;
}

int lcsm_ssm_window(lcsm_ssm* ctx, int layer, void** window) {
  if (!ctx || !window || layer < 0 || layer >= ctx->s.M) return LCSM_EINVAL;
  *window = ctx->window + (size_t)layer * ctx->s.slots * (ctx->s.W - 1) * ctx->C *
                              lcsm::dtype_size(ctx->s.dtype);
  return LCSM_OK;
}

int lcsm_ssm_reset(lcsm_ssm* ctx) {
  if (!ctx) return LCSM_EINVAL;
  hipError_t e = lcsm::launch_zero(ctx->state, ctx->zero_floats, ctx->stream);
  if (e != hipSuccess) return ssm_fail(ctx, LCSM_EDEVICE, "reset", e);
  ctx->faulted = false;
  ctx->msg[0] = 0;
  return LCSM_OK;
}

void lcsm_ssm_destroy(lcsm_ssm* ctx) {
  if (!ctx) return;
  (void)hipStreamSynchronize(ctx->stream);
  if (ctx->owned) (void)hipFree(ctx->owned);
  delete ctx;
}

const char* lcsm_ssm_last_error(const lcsm_ssm* ctx) { return ctx ? ctx->msg : ""; }

}  // extern "C"
