// Products with 8-bit weights and rows quantized to 8 bits (lcsm_q8.h).
//
// Codes of weights and of rows are kept as tiles of 16 rows x 64 inputs, 16
// bytes a lane: lane l has inputs 16 (l / 16) ..+15 of row l % 16, which is its
// share of either operand of a 16x16x64 integer product.  A call quantizes its
// rows into such tiles first, a wave a row.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>

#include "lcsm_elem.h"
#include "lcsm_q8.h"

namespace lcsm {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr int kTileK = 64;   // inputs of a tile, of 16 rows
constexpr int kPadK = 128;   // inputs are padded to whole pairs of tiles
constexpr int kMaxK = 1 << 17;  // 127 * 128 * 2^17 < 2^31

struct Q8Call {
  int rows, N, K, kb;  // kb: tiles along K
  const void* x;
  void* y;
  size_t x_stride, y_stride;
  const char* codes;
  const float *scales, *bias;  // bias NULL: none
  char* row_codes;
  float* row_scales;
};

// ---- quantizing

// The codes of a row whose largest magnitude is `most` (NaN where a value is):
// x / s rounded to the nearest, exactly.  The quotient by the reciprocal may
// land beside it where x is almost between two codes, which the remainder
// shows: x - q s is exact for the integers q next to x / s.
struct Codes {
  float s, sf, f, inv;  // f: a power of two that keeps small scales normal
  __device__ explicit Codes(float most) {
    s = most < INFINITY ? __fdiv_rn(most, 127.f) : __builtin_nanf("");
    f = most < 0x1p-60f ? 0x1p80f : 1.f;
    sf = s * f;
    inv = s > 0.f ? 1.f / sf : 0.f;  // (zero and NaN: codes of zero)
  }
  __device__ int operator()(float x) const {
    const float xf = x * f, q = rintf(xf * inv), r = 2.f * fmaf(-q, sf, xf);
    int c = (int)q;
    if (fabsf(r) > sf || (fabsf(r) == sf && (c & 1))) c += r > 0.f ? 1 : -1;
    return inv > 0.f ? min(max(c, -127), 127) : 0;
  }
};

__device__ __forceinline__ float larger(float a, float b) { return b > a || b != b ? b : a; }

// 16 elements from p, zeros from `have` on; wide accesses of global memory may
// begin at any element.
template <class E>
__device__ __forceinline__ void load16(const E* p, int have, float (&v)[16]) {
  struct __attribute__((packed, aligned(sizeof(E)))) Pack {
    E e[16];
  };
  if (have >= 16) {
    const Pack k = *reinterpret_cast<const Pack*>(p);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = (float)k.e[i];
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = i < have ? (float)p[i] : 0.f;
  }
}

// A wave a row.  TILES: into tiles (padded with zeros to whole tiles), else the
// codes one after another.
template <class E, bool TILES>
__global__ __launch_bounds__(256) void k_q8_rows(const void* x, size_t x_stride, int rows, int K, int kb,
                                                 char* __restrict__ codes, float* __restrict__ scales) {
  const int lane = (int)threadIdx.x & 63;
  const long long row = (long long)blockIdx.x * 4 + threadIdx.x / 64;
  if (row >= rows) return;
  const E* p = static_cast<const E*>(x) + (size_t)row * x_stride;
  float most = 0.f;
  for (int k = 16 * lane; k < K; k += 1024) {
    float v[16];
    load16(p + k, K - k, v);
#pragma unroll
    for (int i = 0; i < 16; ++i) most = larger(most, fabsf(v[i]));
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) most = larger(most, __shfl_xor(most, m));
  const Codes code(most);
  if (lane == 0) scales[row] = code.s;
  const int end = TILES ? kb * kTileK : K;
  for (int k = 16 * lane; k < end; k += 1024) {
    float v[16];
    load16(p + k, K - k, v);
    v4i w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (code(v[4 * i]) & 255) | (code(v[4 * i + 1]) & 255) << 8 | (code(v[4 * i + 2]) & 255) << 16 |
             (int)((unsigned)code(v[4 * i + 3]) << 24);
    if constexpr (TILES) {
      const size_t tile = (size_t)(row / 16) * kb + k / kTileK;
      *reinterpret_cast<v4i*>(codes + tile * 1024 + (k % kTileK / 16 * 16 + row % 16) * 16) = w;
    } else {
      char* to = codes + (size_t)row * K + k;
      for (int i = 0; i < 16 && k + i < K; ++i) to[i] = (char)(w[i / 4] >> (8 * (i % 4)));
    }
  }
}

// Weights [M][N][K] as tiles [M][nts][kb][64][16], zeros past N and K.
__global__ __launch_bounds__(256) void k_q8_codes(const int8_t* __restrict__ src, v4i* __restrict__ dst, int M, int N,
                                                  int K, int nts, int kb) {
  const size_t n = (size_t)M * nts * kb * 64, step = (size_t)gridDim.x * 256;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    const int lane = (int)(i % 64);
    const size_t tile = i / 64, tk = tile % kb, tn = tile / kb % nts, m = tile / kb / nts;
    const size_t out = tn * 16 + lane % 16, k0 = tk * kTileK + 16 * (lane / 16);
    const int8_t* p = src + (m * N + out) * K + k0;
    v4i w = {0, 0, 0, 0};
    if (out < (size_t)N) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (k0 + e < (size_t)K) w[e / 4] |= (int)((unsigned)(uint8_t)p[e] << (8 * (e % 4)));
    }
    dst[i] = w;
  }
}

// ---- products

// A workgroup takes NT tiles of 16 outputs and RT of 16 rows; its waves take
// every so many'th tile along K, and their sums meet in LDS.
constexpr int kAhead = 4;  // tiles along K on their way

template <class E, int RT, int NT>
__global__ __launch_bounds__(1024) void k_q8_few(Q8Call c) {
  extern __shared__ __align__(16) v4i part[];  // [waves][NT][RT][64]
  const int lane = (int)threadIdx.x & 63, nw = (int)blockDim.x >> 6;
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int nts = (c.N + 15) / 16, rts = (c.rows + 15) / 16;
  const int nt0 = (int)blockIdx.x * NT, rt0 = (int)blockIdx.y * RT;
  const v4i *w[NT], *x[RT];
#pragma unroll
  for (int t = 0; t < NT; ++t) w[t] = reinterpret_cast<const v4i*>(c.codes) + (size_t)min(nt0 + t, nts - 1) * c.kb * 64 + lane;
#pragma unroll
  for (int r = 0; r < RT; ++r) x[r] = reinterpret_cast<const v4i*>(c.row_codes) + (size_t)min(rt0 + r, rts - 1) * c.kb * 64 + lane;
  v4i acc[NT][RT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[t][r] = v4i{0, 0, 0, 0};
  for (int k0 = wv; k0 < c.kb; k0 += kAhead * nw) {
    v4i a[kAhead][NT], b[kAhead][RT];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int k = min(k0 + u * nw, c.kb - 1);
#pragma unroll
      for (int t = 0; t < NT; ++t) a[u][t] = w[t][(size_t)k * 64];
#pragma unroll
      for (int r = 0; r < RT; ++r) b[u][r] = x[r][(size_t)k * 64];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (k0 + u * nw >= c.kb) break;
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < RT; ++r) acc[t][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[u][t], b[u][r], acc[t][r], 0, 0, 0);
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) part[((wv * NT + t) * RT + r) * 64 + lane] = acc[t][r];
  __syncthreads();
  const int* sum = reinterpret_cast<const int*>(part);
  for (int o = (int)threadIdx.x; o < NT * RT * 256; o += (int)blockDim.x) {
    const int t = o / 16 % NT, n = (nt0 + t) * 16 + o % 16, r = o / (16 * NT);
    const int at = rt0 * 16 + r;
    if (n >= c.N || at >= c.rows) continue;
    const int i = (t * RT + r / 16) * 256 + (o % 16 / 4 * 16 + r % 16) * 4 + o % 4;
    int v = 0;
    for (int k = 0; k < nw; ++k) v += sum[k * NT * RT * 256 + i];
    const float y = (float)v * c.scales[n] * c.row_scales[at];
    static_cast<E*>(c.y)[(size_t)at * c.y_stride + n] = (E)(c.bias ? y + c.bias[n] : y);
  }
}

template <class E, int RT, int NT>
hipError_t launch_few(const Q8Call& c, hipStream_t st) {
  const int waves = c.kb < 8 ? c.kb : 8;
  const dim3 grid((unsigned)(((c.N + 15) / 16 + NT - 1) / NT), (unsigned)((c.rows + 16 * RT - 1) / (16 * RT)));
  hipLaunchKernelGGL((k_q8_few<E, RT, NT>), grid, dim3(64 * waves), (size_t)waves * NT * RT * 1024, st, c);
  return hipGetLastError();
}

// Many rows.  A workgroup of WN x WX waves takes WN NT tiles of outputs and WX RT
// of rows, a wave NT x RT of them, in registers.  The tiles of 64 inputs go from
// memory straight into one of four stages in LDS, three stages ahead of the one
// that is multiplied.
constexpr int kStages = 4;

// All waves past their LDS reads; transfers into LDS stay on their way, which
// __syncthreads would wait for.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <class E, int WN, int WX, int NT, int RT>
__global__ __launch_bounds__(64 * WN * WX, 2) void k_q8_many(Q8Call c) {
  constexpr int WAVES = WN * WX, TN = WN * NT, TX = WX * RT, EACH = (TN + TX) / WAVES;  // tiles a wave fetches
  constexpr int STAGE = (TN + TX) * 1024;
  static_assert((TN + TX) % WAVES == 0 && EACH == 4, "the waits below count four transfers a stage");
  extern __shared__ __align__(16) char lds[];
  const int lane = (int)threadIdx.x & 63, q = lane >> 4, l = lane & 15;
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wn = wv / WX, wx = wv % WX;
  const int nts = (c.N + 15) / 16, rts = (c.rows + 15) / 16;
  const int gn = (nts + TN - 1) / TN, gx = (rts + TX - 1) / TX;
  // Workgroup b runs on XCD b % 8: each XCD (and its L2) takes a contiguous range
  // of the tiles, ordered so that those at work together share rows and outputs.
  constexpr int GROUP = 4;  // row pieces that go through the outputs together
  const int total = gn * gx, per = total / 8, rest = total % 8, xcd = (int)blockIdx.x % 8;
  const int id = xcd * per + min(xcd, rest) + (int)blockIdx.x / 8;
  const int group = id / (GROUP * gn), first = group * GROUP, have = min(GROUP, gx - first);
  const int pn = (id - first * gn) / have, px = first + (id - first * gn) % have;
  // what this wave fetches: tiles of outputs first, then of rows (past the last
  // one the last one again: what is made of it is not stored)
  __amdgpu_buffer_rsrc_t from[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int t = wv * EACH + i;
    const char* p = t < TN ? c.codes + (size_t)min(pn * TN + t, nts - 1) * c.kb * 1024
                           : c.row_codes + (size_t)min(px * TX + t - TN, rts - 1) * c.kb * 1024;
    from[i] = uniform_buffer(p, (unsigned)c.kb * 1024u);
  }
  auto fetch = [&](int k) {
#pragma unroll
    for (int i = 0; i < EACH; ++i)
      fetch_to_lds(from[i], lane * 16u, k * 1024u, lds + k % kStages * STAGE + (wv * EACH + i) * 1024);
  };
  v4i acc[NT][RT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[t][r] = v4i{0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k)
    if (k < c.kb) fetch(k);
  for (int k = 0; k < c.kb; ++k) {
    // this wave's transfers of stage k have arrived, those of the next two may be on
    // their way; then all waves' have, and stage k - 1 has been read
    if (k + kStages - 1 <= c.kb)
      asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    lds_barrier();
    if (k + kStages - 1 < c.kb) fetch(k + kStages - 1);
    const v4i* at = reinterpret_cast<const v4i*>(lds + k % kStages * STAGE) + lane;
    v4i a[NT], b[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) b[r] = at[(TN + wx * RT + r) * 64];
#pragma unroll
    for (int t = 0; t < NT; ++t) a[t] = at[(wn * NT + t) * 64];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < RT; ++r) acc[t][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[t], b[r], acc[t][r], 0, 0, 0);
  }
  // outputs 4 q ..+3 of tile t, row l of tile r
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    const int row = (px * TX + wx * RT + r) * 16 + l;
    if (row >= c.rows) continue;
    const float s = c.row_scales[row];
    E* y = static_cast<E*>(c.y) + (size_t)row * c.y_stride;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int n = (pn * TN + wn * NT + t) * 16 + 4 * q;
      struct __attribute__((packed, aligned(sizeof(E)))) Pack {
        E e[4];
      } out;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = min(n + i, c.N - 1);
        const float v = (float)acc[t][r][i] * c.scales[at] * s;
        out.e[i] = (E)(c.bias ? v + c.bias[at] : v);
      }
      if (n + 4 <= c.N) {
        *reinterpret_cast<Pack*>(y + n) = out;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < c.N) y[n + i] = out.e[i];
      }
    }
  }
}

template <class E, int WN, int WX, int NT, int RT>
hipError_t launch_many(const Q8Call& c, hipStream_t st) {
  constexpr int TN = WN * NT, TX = WX * RT, LDS = kStages * (TN + TX) * 1024;
  const long long gn = ((c.N + 15) / 16 + TN - 1) / TN, gx = ((c.rows + 15) / 16 + TX - 1) / TX;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_q8_many<E, WN, WX, NT, RT>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_q8_many<E, WN, WX, NT, RT>), dim3((unsigned)(gn * gx)), dim3(64 * WN * WX), LDS, st, c);
  return hipGetLastError();
}

template <class E>
hipError_t launch_q8(const Q8Call& c, hipStream_t st) {
  hipLaunchKernelGGL((k_q8_rows<E, true>), dim3((unsigned)((c.rows + 3) / 4)), dim3(256), 0, st, c.x, c.x_stride, c.rows,
                     c.K, c.kb, c.row_codes, c.row_scales);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (c.rows <= 16) return launch_few<E, 1, 1>(c, st);
  if (c.rows <= 64) return launch_few<E, 2, 2>(c, st);
  const long long n = c.N, r = c.rows;
  if (((n + 255) / 256) * ((r + 255) / 256) >= 192) return launch_many<E, 2, 4, 8, 4>(c, st);
  return launch_many<E, 2, 2, 4, 4>(c, st);
}

unsigned blocks(size_t n) {
  const size_t b = (n + 255) / 256;
  return (unsigned)(b < 16384 ? b : 16384);
}

}  // namespace
}  // namespace lcsm

struct lcsm_q8 {
  lcsm_q8_shape s;
  int nts, kb;
  hipStream_t stream;
  void* owned;
  char *codes, *row_codes;
  float *scales, *bias, *row_scales;
  bool faulted;
  char msg[256];
};

namespace {

struct Plan {
  int nts, kb;
  size_t codes, scales, bias, row_codes, row_scales, total;
};

bool q8_plan(const lcsm_q8_shape* s, Plan* p) {
  if (!s || s->M < 1 || s->M > 16384 || s->N < 1 || s->K < 1 || s->N > (1 << 24) || s->K > lcsm::kMaxK ||
      s->max_rows < 1 || s->max_rows > (1 << 24) || (double)s->N * s->K > 1099511627776.0)
    return false;
  for (int r : s->reserved)
    if (r) return false;
  p->nts = (s->N + 15) / 16;
  p->kb = (s->K + lcsm::kPadK - 1) / lcsm::kPadK * (lcsm::kPadK / lcsm::kTileK);
  const size_t M = (size_t)s->M, rts = ((size_t)s->max_rows + 15) / 16;
  size_t at = 0;
  auto take = [&](size_t* where, size_t bytes) {
    *where = at;
    at = (at + bytes + 255) / 256 * 256;
  };
  take(&p->codes, M * p->nts * p->kb * 1024);
  take(&p->scales, M * s->N * sizeof(float));
  take(&p->bias, M * s->N * sizeof(float));
  take(&p->row_codes, rts * p->kb * 1024);
  take(&p->row_scales, rts * 16 * sizeof(float));
  p->total = at;
  return true;
}

int q8_fail(lcsm_q8* c, int code, const char* what, hipError_t e = hipSuccess) {
  if (e != hipSuccess) {
    snprintf(c->msg, sizeof(c->msg), "%s: %s", what, hipGetErrorString(e));
    c->faulted = true;
    return LCSM_EDEVICE;
  }
  snprintf(c->msg, sizeof(c->msg), "%s", what);
  return code;
}

}  // namespace

extern "C" {

int lcsm_q8_workspace_bytes(const lcsm_q8_shape* shape, size_t* bytes) {
  Plan p;
  if (!bytes || !q8_plan(shape, &p)) return LCSM_EINVAL;
  *bytes = p.total;
  return LCSM_OK;
}

int lcsm_q8_init(lcsm_q8** out, const lcsm_q8_shape* shape, const void* codes, const float* scales,
                 const float* bias, void* stream, void* workspace, size_t workspace_bytes) {
  if (!out) return LCSM_EINVAL;
  *out = nullptr;
  Plan p;
  if (!codes || !scales || !q8_plan(shape, &p)) return LCSM_EINVAL;
  if (workspace && ((uintptr_t)workspace & 255)) return LCSM_EINVAL;
  if (workspace && workspace_bytes < p.total) return LCSM_ENOMEM;
  lcsm_q8* c = new (std::nothrow) lcsm_q8();
  if (!c) return LCSM_ENOMEM;
  c->s = *shape;
  c->nts = p.nts;
  c->kb = p.kb;
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
  c->codes = mem + p.codes;
  c->scales = (float*)(mem + p.scales);
  c->bias = bias ? (float*)(mem + p.bias) : nullptr;
  c->row_codes = mem + p.row_codes;
  c->row_scales = (float*)(mem + p.row_scales);
  const size_t lanes = (size_t)shape->M * p.nts * p.kb * 64, each = (size_t)shape->M * shape->N * sizeof(float);
  hipLaunchKernelGGL(lcsm::k_q8_codes, dim3(lcsm::blocks(lanes)), dim3(256), 0, c->stream, (const int8_t*)codes,
                     (lcsm::v4i*)c->codes, shape->M, shape->N, shape->K, p.nts, p.kb);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) e = hipMemcpyAsync(c->scales, scales, each, hipMemcpyDeviceToDevice, c->stream);
  if (e == hipSuccess && bias) e = hipMemcpyAsync(c->bias, bias, each, hipMemcpyDeviceToDevice, c->stream);
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

int lcsm_q8_matmul(lcsm_q8* ctx, int layer, int rows, int dtype, const void* x, size_t x_stride,
                   void* y, size_t y_stride) {
  if (!ctx) return LCSM_EINVAL;
  const lcsm_q8_shape& s = ctx->s;
  if (layer < 0 || layer >= s.M) return q8_fail(ctx, LCSM_EINVAL, "layer out of range");
  if (rows < 0 || rows > s.max_rows) return q8_fail(ctx, LCSM_EINVAL, "rows below zero or above max_rows");
  if (!lcsm::dtype_ok(dtype)) return q8_fail(ctx, LCSM_EINVAL, "unknown type");
  if (rows > 0) {
    if (!x || !y) return q8_fail(ctx, LCSM_EINVAL, "null input or output pointer");
    if (x_stride < (size_t)s.K || y_stride < (size_t)s.N)
      return q8_fail(ctx, LCSM_EINVAL, "a row stride is shorter than the row");
  }
  if (ctx->faulted) return LCSM_ESTATE;
  if (!rows) return LCSM_OK;
  const size_t m = (size_t)layer;
  const lcsm::Q8Call c{rows, s.N, s.K, ctx->kb, x, y, x_stride, y_stride, ctx->codes + m * ctx->nts * ctx->kb * 1024,
                       ctx->scales + m * s.N, ctx->bias ? ctx->bias + m * s.N : nullptr, ctx->row_codes,
                       ctx->row_scales};
  const hipError_t e = lcsm::with_dtype(dtype, [&](auto v) { return lcsm::launch_q8<decltype(v)>(c, ctx->stream); });
  return e == hipSuccess ? LCSM_OK : q8_fail(ctx, LCSM_EDEVICE, "product launch", e);
}

int lcsm_q8_quantize(const float* w, int rows, int K, void* codes, float* scales, void* stream) {
  if (rows < 0 || K < 1 || K > (1 << 24)) return LCSM_EINVAL;
  if (!rows) return LCSM_OK;
  if (!w || !codes || !scales) return LCSM_EINVAL;
  hipLaunchKernelGGL((lcsm::k_q8_rows<float, false>), dim3((unsigned)(((long long)rows + 3) / 4)), dim3(256), 0,
                     (hipStream_t)stream, w, (size_t)K, rows, K, 0, (char*)codes, scales);
  return hipGetLastError() == hipSuccess ? LCSM_OK : LCSM_EDEVICE;
}

int lcsm_q8_reset(lcsm_q8* ctx) {
  if (!ctx) return LCSM_EINVAL;
  ctx->faulted = false;
  ctx->msg[0] = 0;
  return LCSM_OK;
}

void lcsm_q8_destroy(lcsm_q8* ctx) {
  if (!ctx) return;
  (void)hipStreamSynchronize(ctx->stream);
  if (ctx->owned) (void)hipFree(ctx->owned);
  delete ctx;
}

const char* lcsm_q8_last_error(const lcsm_q8* ctx) { return ctx ? ctx->msg : ""; }

}  // extern "C"
