// Norms of queries and keys for each head with the rotation by their positions
// (lcsm_rot.h).
//
// A team of lanes has a head of a token in registers from its load to its
// store, both values of a pair in one lane: the norm is a sum over the team, the
// rotation needs nothing from outside.  A team goes through several heads of its
// token, so that the sines and cosines of the lane's pairs are made once for
// them: made for each head they would take longer than the bytes do.
//
// Bound by those: 16384 rows of 32 heads of 128 of queries and of keys, bf16, take
// 115 us, 4.7 TB/s, what a large copy reaches; a few rows take the time of a launch.
// The angle is made in 64 bits up to its share of a turn, whatever the type.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>
#include <type_traits>

#include "lcsm_elem.h"
#include "lcsm_rot.h"

namespace lcsm {
namespace {

constexpr int kRotMaxP = 512;
constexpr int kRotMaxHeads = 65536;

struct RotCall {
  int rows, P, q_heads, k_heads, rotary, norm;
  int team, teams, q_teams;  // lanes a head; teams a row, and how many of them have queries
  float eps;
  const void *q, *k;
  void *q_out, *k_out;
  size_t q_stride, k_stride, q_out_stride, k_out_stride;
  const int* positions;
  const double* turns;       // turns a position, [rotary / 2]
  const float *q_w, *k_w;    // of the layer, NULL: ones
};

// V elements side by side, at any element's address: wide accesses of global
// memory allow that.
template <class E, int V>
struct __attribute__((packed, aligned(sizeof(E)))) Pack {
  E e[V];
};

// Sum over the L lanes of a team (a power of two), in a fixed order; every lane
// gets it.  Once quads have their sums, lanes that lie mirrored in a row of 8 or 16
// have the other half's.
__device__ __forceinline__ float team_sum(float v, int L) {
  auto add = [&](auto dpp) {
    const int x = __builtin_bit_cast(int, v);
    v += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, x, decltype(dpp)::value, 0xf, 0xf, false));
  };
  if (L > 1) add(std::integral_constant<int, 0xB1>());   // quad_perm 1 0 3 2
  if (L > 2) add(std::integral_constant<int, 0x4E>());   // quad_perm 2 3 0 1
  if (L > 4) add(std::integral_constant<int, 0x141>());  // row_half_mirror
  if (L > 8) add(std::integral_constant<int, 0x140>());  // row_mirror
  if (L > 16) v += __shfl_xor(v, 16);
  if (L > 32) v += __shfl_xor(v, 32);
  return v;
}

// A lane has up to CNT items of a head: V pairs, or V values that are not
// turned; pairs first.  A team takes `each` heads of queries, or of keys.
template <class E, int V, bool HALF, int CNT>
__global__ __launch_bounds__(256) void k_rot(RotCall c) {
  const int L = c.team, lane = (int)threadIdx.x % L;
  const size_t unit = ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * (256 / L) + threadIdx.x / L;
  const size_t row = unit / c.teams;
  if (row >= (size_t)c.rows) return;  // whole teams: no lane waits for them
  const int mine = (int)(unit % c.teams), half = c.rotary / 2;
  const int pairs = half / V, items = pairs + (c.P - c.rotary) / V;
  const bool key = mine >= c.q_teams;
  const int first = key ? mine - c.q_teams : mine, step = key ? c.teams - c.q_teams : c.q_teams;
  const int heads = key ? c.k_heads : c.q_heads;
  const E* x = key ? static_cast<const E*>(c.k) + row * c.k_stride : static_cast<const E*>(c.q) + row * c.q_stride;
  E* y = key ? static_cast<E*>(c.k_out) + row * c.k_out_stride : static_cast<E*>(c.q_out) + row * c.q_out_stride;
  const float* w = key ? c.k_w : c.q_w;

  auto item = [&](int i) { return i * L + lane; };
  auto at_a = [&](int j) { return j < pairs ? (HALF ? j * V : 2 * j * V) : c.rotary + (j - pairs) * V; };
  Pack<E, V> a[CNT], b[CNT];
  auto load = [&](int h) {
#pragma unroll
    for (int i = 0; i < CNT; ++i) {
      const int j = item(i);
      if (j >= items) continue;
      const E* p = x + (size_t)h * c.P + at_a(j);
      if (HALF || j >= pairs) {
        a[i] = *reinterpret_cast<const Pack<E, V>*>(p);
        if (j < pairs) b[i] = *reinterpret_cast<const Pack<E, V>*>(p + half);
      } else {
        const Pack<E, 2 * V> both = *reinterpret_cast<const Pack<E, 2 * V>*>(p);
#pragma unroll
        for (int e = 0; e < V; ++e) a[i].e[e] = both.e[2 * e], b[i].e[e] = both.e[2 * e + 1];
      }
    }
  };
  load(first);

  float wa[CNT][V], wb[CNT][V], cs[CNT][V], sn[CNT][V];
  const double t = pairs > 0 ? (double)c.positions[row] : 0.0;
#pragma unroll
  for (int i = 0; i < CNT; ++i) {
    const int j = item(i);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      wa[i][e] = w && j < items ? w[at_a(j) + (HALF || j >= pairs ? e : 2 * e)] : 1.f;
      wb[i][e] = w && j < pairs ? w[at_a(j) + (HALF ? half + e : 2 * e + 1)] : 1.f;
      cs[i][e] = 1.f;
      sn[i][e] = 0.f;
      if (j >= pairs) continue;
      const double r = t * c.turns[j * V + e];
      sincospif((float)(2.0 * (r - rint(r))), &sn[i][e], &cs[i][e]);
    }
  }
  const float inv = 1.f / (float)c.P;
  for (int h = first; h < heads; h += step) {
    float va[CNT][V], vb[CNT][V];
#pragma unroll
    for (int i = 0; i < CNT; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        va[i][e] = item(i) < items ? (float)a[i].e[e] : 0.f;
        vb[i][e] = item(i) < pairs ? (float)b[i].e[e] : 0.f;
      }
    if (h + step < heads) load(h + step);
    if (c.norm != LCSM_NORM_NONE) {
      if (c.norm == LCSM_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < CNT; ++i)
#pragma unroll
          for (int e = 0; e < V; ++e) s += va[i][e] + vb[i][e];
        const float mean = team_sum(s, L) * inv;
#pragma unroll
        for (int i = 0; i < CNT; ++i)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            va[i][e] = item(i) < items ? va[i][e] - mean : 0.f;
            vb[i][e] = item(i) < pairs ? vb[i][e] - mean : 0.f;
          }
      }
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < CNT; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) s = fmaf(va[i][e], va[i][e], fmaf(vb[i][e], vb[i][e], s));
      const float f = 1.f / sqrtf(fmaf(team_sum(s, L), inv, c.eps));
#pragma unroll
      for (int i = 0; i < CNT; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) va[i][e] *= f * wa[i][e], vb[i][e] *= f * wb[i][e];
    }
    E* to = y + (size_t)h * c.P;
#pragma unroll
    for (int i = 0; i < CNT; ++i) {
      const int j = item(i);
      if (j >= items) continue;
      E* p = to + at_a(j);
      Pack<E, V> ra, rb;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        // (a value that is not turned is not made of products: 0 * inf)
        ra.e[e] = (E)(j < pairs ? va[i][e] * cs[i][e] - vb[i][e] * sn[i][e] : va[i][e]);
        rb.e[e] = (E)(j < pairs ? vb[i][e] * cs[i][e] + va[i][e] * sn[i][e] : 0.f);
      }
      if (HALF || j >= pairs) {
        *reinterpret_cast<Pack<E, V>*>(p) = ra;
        if (j < pairs) *reinterpret_cast<Pack<E, V>*>(p + half) = rb;
      } else {
        Pack<E, 2 * V> both;
#pragma unroll
        for (int e = 0; e < V; ++e) both.e[2 * e] = ra.e[e], both.e[2 * e + 1] = rb.e[e];
        *reinterpret_cast<Pack<E, 2 * V>*>(p) = both;
      }
    }
  }
}

// Heads that a team goes through at most, and the waves that have to be left: the
// lanes' weights, sines and cosines are made once for them.  us of bf16 rows with 32
// heads of 128 of queries and of keys, for at most 4, 8, 16 heads with 2048 waves left,
// for 16 with 8192, and for single heads:
//     512 rows   7.7   7.7   7.8   9.8  10.1      4096 rows  29.7  27.0  28.5  29.7  62.2
//    2048 rows  16.6  15.5  15.5  21.8  33.3     16384 rows 126.7 114.5 116.3 116.6 253.9
constexpr int kRotHeads = 8;
constexpr long long kRotWaves = 2048;

template <class E, int V, bool HALF, int CNT>
hipError_t launch_rot_of(RotCall c, hipStream_t st) {
  const int items = c.rotary / 2 / V + (c.P - c.rotary) / V;
  c.team = 1;
  while (c.team < items && c.team < 64) c.team *= 2;
  const long long waves = (long long)c.rows * (c.q_heads + c.k_heads) * c.team / 64;
  const int each = waves < 2 * kRotWaves ? 1 : waves >= kRotHeads * kRotWaves ? kRotHeads : (int)(waves / kRotWaves);
  c.q_teams = (c.q_heads + each - 1) / each;
  c.teams = c.q_teams + (c.k_heads + each - 1) / each;
  const long long per = 256 / c.team, groups = ((long long)c.rows * c.teams + per - 1) / per;
  const long long x = groups < (1 << 20) ? groups : 1 << 20;
  hipLaunchKernelGGL((k_rot<E, V, HALF, CNT>), dim3((unsigned)x, (unsigned)((groups + x - 1) / x)), dim3(256), 0, st, c);
  return hipGetLastError();
}

// The widest accesses that both kinds of items divide into.
template <class E, bool HALF>
hipError_t launch_rot_pairs(const RotCall& c, hipStream_t st) {
  const int half = c.rotary / 2, rest = c.P - c.rotary;
  constexpr int W = 16 / (int)sizeof(E);
  if (half % W == 0 && rest % W == 0) return launch_rot_of<E, W, HALF, kRotMaxP / W / 64>(c, st);
  if (half % 2 == 0 && rest % 2 == 0) return launch_rot_of<E, 2, HALF, kRotMaxP / 2 / 64>(c, st);
  if (half + rest <= 64) return launch_rot_of<E, 1, HALF, 1>(c, st);
  return launch_rot_of<E, 1, HALF, kRotMaxP / 64>(c, st);
}
template <class E>
hipError_t launch_rot(const RotCall& c, int pairs, hipStream_t st) {
  return pairs == LCSM_PAIRS_HALF ? launch_rot_pairs<E, true>(c, st) : launch_rot_pairs<E, false>(c, st);
}

__global__ __launch_bounds__(256) void k_rot_turns(const double* f, double* turns, int n) {
  const int i = (int)(blockIdx.x * 256 + threadIdx.x);
  if (i < n) turns[i] = f[i] * 0.15915494309189533577;  // 1 / (2 pi)
}

}  // namespace
}  // namespace lcsm

struct lcsm_rot {
  lcsm_rot_shape s;
  hipStream_t stream;
  void* owned;
  double* turns;
  float* w[2];  // of queries and keys; NULL where not given
  bool faulted;
  char msg[256];
};

namespace {

int rot_fail(lcsm_rot* c, int code, const char* what, hipError_t e = hipSuccess) {
  if (e != hipSuccess) {
    snprintf(c->msg, sizeof(c->msg), "%s: %s", what, hipGetErrorString(e));
    c->faulted = true;
    return LCSM_EDEVICE;
  }
  snprintf(c->msg, sizeof(c->msg), "%s", what);
  return code;
}

bool rot_shape_ok(const lcsm_rot_shape* s) {
  if (!s || s->M < 1 || s->M > 16384 || s->P < 1 || s->P > lcsm::kRotMaxP || s->q_heads < 1 ||
      s->q_heads > lcsm::kRotMaxHeads || s->k_heads < 0 || s->k_heads > lcsm::kRotMaxHeads)
    return false;
  for (int r : s->reserved)
    if (r) return false;
  return s->rotary >= 0 && s->rotary <= s->P && s->rotary % 2 == 0 && s->pairs >= LCSM_PAIRS_HALF &&
         s->pairs <= LCSM_PAIRS_ADJACENT && s->norm >= LCSM_NORM_NONE && s->norm <= LCSM_NORM_LAYER &&
         lcsm::dtype_ok(s->dtype) && isfinite(s->eps) && s->eps >= 0.f;
}

struct Plan {
  size_t turns, w[2], total;
};

bool rot_plan(const lcsm_rot_shape* s, Plan* p) {
  if (!rot_shape_ok(s)) return false;
  size_t at = 0;
  auto take = [&](size_t* where, size_t bytes) {
    *where = at;
    at = (at + bytes + 255) / 256 * 256;
  };
  take(&p->turns, (size_t)(s->rotary / 2) * sizeof(double));
  for (size_t& w : p->w) take(&w, (size_t)s->M * s->P * sizeof(float));
  p->total = at;
  return true;
}

}  // namespace

extern "C" {

int lcsm_rot_workspace_bytes(const lcsm_rot_shape* shape, size_t* bytes) {
  Plan p;
  if (!bytes || !rot_plan(shape, &p)) return LCSM_EINVAL;
  *bytes = p.total;
  return LCSM_OK;
}

int lcsm_rot_init(lcsm_rot** out, const lcsm_rot_shape* shape, const double* freqs, const float* q_w,
                  const float* k_w, void* stream, void* workspace, size_t workspace_bytes) {
  if (!out) return LCSM_EINVAL;
  *out = nullptr;
  Plan p;
  if (!rot_plan(shape, &p) || (shape->rotary > 0 && !freqs)) return LCSM_EINVAL;
  if (workspace && ((uintptr_t)workspace & 255)) return LCSM_EINVAL;
  if (workspace && workspace_bytes < p.total) return LCSM_ENOMEM;
  lcsm_rot* c = new (std::nothrow) lcsm_rot();
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
  c->turns = (double*)((char*)workspace + p.turns);
  const int half = shape->rotary / 2;
  hipError_t e = hipSuccess;
  if (half) {
    hipLaunchKernelGGL(lcsm::k_rot_turns, dim3((unsigned)((half + 255) / 256)), dim3(256), 0, c->stream, freqs, c->turns,
                       half);
    e = hipGetLastError();
  }
  const float* src[2] = {q_w, k_w};
  for (int k = 0; k < 2 && e == hipSuccess; ++k) {
    if (!src[k]) continue;
    c->w[k] = (float*)((char*)workspace + p.w[k]);
    e = hipMemcpyAsync(c->w[k], src[k], (size_t)shape->M * shape->P * sizeof(float), hipMemcpyDeviceToDevice, c->stream);
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

int lcsm_rot_apply(lcsm_rot* ctx, int layer, int rows, const lcsm_rot_io* io) {
  if (!ctx) return LCSM_EINVAL;
  const lcsm_rot_shape& s = ctx->s;
  if (layer < 0 || layer >= s.M) return rot_fail(ctx, LCSM_EINVAL, "layer out of range");
  if (rows < 0 || !io) return rot_fail(ctx, LCSM_EINVAL, "rows below zero or null io");
  const size_t qw = (size_t)s.q_heads * s.P, kw = (size_t)s.k_heads * s.P;
  if (rows > 0) {
    if (!io->q || !io->q_out || (kw && (!io->k || !io->k_out)))
      return rot_fail(ctx, LCSM_EINVAL, "null input or output pointer");
    if (s.rotary && !io->positions) return rot_fail(ctx, LCSM_EINVAL, "null positions");
    if (io->q_stride < qw || io->q_out_stride < qw || (kw && (io->k_stride < kw || io->k_out_stride < kw)))
      return rot_fail(ctx, LCSM_EINVAL, "a row stride is shorter than the row");
  }
  if (ctx->faulted) return LCSM_ESTATE;
  if (!rows) return LCSM_OK;
  const size_t at = (size_t)layer * s.P;
  lcsm::RotCall c{};
  c.rows = rows, c.P = s.P, c.q_heads = s.q_heads, c.k_heads = s.k_heads;
  c.rotary = s.rotary, c.norm = s.norm, c.eps = s.eps;
  c.q = io->q, c.k = io->k, c.q_out = io->q_out, c.k_out = io->k_out;
  c.q_stride = io->q_stride, c.k_stride = io->k_stride, c.q_out_stride = io->q_out_stride, c.k_out_stride = io->k_out_stride;
  c.positions = io->positions, c.turns = ctx->turns;
  c.q_w = ctx->w[0] ? ctx->w[0] + at : nullptr;
  c.k_w = ctx->w[1] ? ctx->w[1] + at : nullptr;
  const hipError_t e =
      lcsm::with_dtype(s.dtype, [&](auto v) { return lcsm::launch_rot<decltype(v)>(c, s.pairs, ctx->stream); });
  return e == hipSuccess ? LCSM_OK : rot_fail(ctx, LCSM_EDEVICE, "rotation launch", e);
}

int lcsm_rot_reset(lcsm_rot* ctx) {
  if (!ctx) return LCSM_EINVAL;
  ctx->faulted = false;
  ctx->msg[0] = 0;
  return LCSM_OK;
}

void lcsm_rot_destroy(lcsm_rot* ctx) {
  if (!ctx) return;
  (void)hipStreamSynchronize(ctx->stream);
  if (ctx->owned) (void)hipFree(ctx->owned);
  delete ctx;
}

const char* lcsm_rot_last_error(const lcsm_rot* ctx) { return ctx ? ctx->msg : ""; }

}  // extern "C"
