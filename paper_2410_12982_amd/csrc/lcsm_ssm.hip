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

typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kSsmMaxN = 256;
constexpr int kSsmMaxW = 4;
// The value of the lane whose number differs in bit M.
template <int M>
__device__ __forceinline__ float xor_lane(float v) {
  const int x = __builtin_bit_cast(int, v);
  int r;
  if constexpr (M == 1)
    r = __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xf, 0xf, false);  // quad_perm 1 0 3 2
  else if constexpr (M == 2)
    r = __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xf, 0xf, false);  // quad_perm 2 3 0 1
  else if constexpr (M == 8)
    r = __builtin_amdgcn_update_dpp(0, x, 0x128, 0xf, 0xf, false);  // row_ror 8
  else if constexpr (M < 32)
    r = __builtin_amdgcn_ds_swizzle(x, M << 10 | 0x1f);
  else
    r = __shfl_xor(x, M);
  return __builtin_bit_cast(float, r);
}
// Of 2 HALF sums, lanes with bit M keep the upper ones and lanes without the
// lower ones, both with the other's share added.
template <int M, int HALF>
__device__ __forceinline__ void halve(float* y, int lane) {
  const bool up = lane & M;
#pragma unroll
  for (int j = 0; j < HALF; ++j) {
    const float mine = up ? y[j + HALF] : y[j], theirs = up ? y[j] : y[j + HALF];
    y[j] = mine + xor_lane<M>(theirs);
  }
}

// The recurrence as it is written, for single tokens and short prompts.  A
// workgroup takes ROWS channels of a head of one sequence and keeps their states
// in registers (L lanes a channel, four states each); TB positions at a time it
// convolves their x and its group's B and C into LDS, side by side, and then
// goes through them one by one.  What a position costs is then a dozen FMAs a
// lane: the sums over the states' lanes are taken for eight positions at once,
// halving the lanes' shares of them instead of repeating the sum in all.
//
// The window of x is read and written by the workgroup that has its channels;
// that of B and C is read by all heads of the group, and written by whichever
// of them is the last to have read it (a count in `tickets`, back at zero
// afterwards), so that a sequence can be continued in its own slot by this one
// launch.
// Single tokens: the states, read and written once, bound it where there are
// many (64 tokens of 64 heads x 64 x 128: 273 MB in 75 us, 3.6 TB/s); one token of
// 32 heads takes 7.6 us, two dependent round trips to memory and the launch.
// Prompts: the chain of positions, 0.24 us each (29 tokens 14 us).
template <class E, int L, int R, int TB>
__global__ __launch_bounds__(256) void k_ssm_scan(SsmCall c) {
  constexpr int RPP = 256 / L, ROWS = R * RPP, NP = 4 * L, NC = ROWS + 2 * NP;
  __shared__ __align__(16) float su[TB][NC];  // x, B, C
  __shared__ float sy[TB][ROWS];
  __shared__ float sstep[TB], sdecay[TB];
  __shared__ int slast;
  const int i = (int)blockIdx.z, h = (int)blockIdx.y, p0 = (int)blockIdx.x * ROWS;
  const int tid = (int)threadIdx.x, n0 = tid % L * 4, r0 = tid / L;
  const int g = h / (c.H / c.G), W1 = c.W - 1;
  int t0, t1;
  ssm_rows(c, i, t0, t1);
  const int s = ssm_slot(c.src, i, c.slots), d = ssm_slot(c.dst, i, c.slots);
  const size_t head = (size_t)c.P * c.N;
  const bool quads = c.N % 4 == 0;
  // a single token's gate is on its way from the start
  E zt = (E)0.f;
  if (TB == 1 && c.z && tid < ROWS && p0 + tid < c.P)
    zt = static_cast<const E*>(c.z)[(size_t)i * c.z_stride + h * c.P + p0 + tid];
  float S[R][4];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int p = p0 + r0 + r * RPP;
#pragma unroll
    for (int e = 0; e < 4; ++e) S[r][e] = 0.f;
    if (s < 0 || p >= c.P || n0 >= c.N) continue;
    // states pass through once a call: not kept in the caches (64 tokens of 64 heads
    // x 64 x 128 89 -> 75 us)
    const float* at = c.state + ((size_t)s * c.H + h) * head + (size_t)p * c.N + n0;
    if (quads) {
      const v4f v = __builtin_nontemporal_load(reinterpret_cast<const v4f*>(at));
#pragma unroll
      for (int e = 0; e < 4; ++e) S[r][e] = v[e];
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n0 + e < c.N) S[r][e] = at[e];
    }
  }
  // channel of a row that column k of su is, -1: none
  auto channel = [&](int k) {
    if (k < ROWS) return p0 + k < c.P ? h * c.P + p0 + k : -1;
    const int j = (k - ROWS) % NP;
    return j < c.N ? c.D + (k < ROWS + NP ? 0 : c.G * c.N) + g * c.N + j : -1;
  };
  const E* x = static_cast<const E*>(c.xbc);
  E* win = static_cast<E*>(c.window);
  // rows before t0 from the window of slot s
  auto raw = [&](int t, int ch) {
    if (t >= t0) return x[(size_t)t * c.xbc_stride + ch];
    return s >= 0 ? win[((size_t)s * W1 + (t - t0 + W1)) * c.C + ch] : (E)0.f;
  };
  const float skip = c.skip[h];
  int ticket = 0;

  for (int b = t0; b < t1; b += TB) {
    const int nt = min(TB, t1 - b);
    if (TB > 1 && b > t0) __syncthreads();  // the positions before have been read
    // a thread convolves a channel along RUN positions; the rows of all that it
    // takes of them are on their way before the first is used
    constexpr int RUN = TB < 8 ? TB : 8, ITEMS = NC * (TB / RUN), EACH = (ITEMS + 255) / 256;
    constexpr int AT = TB == 1 ? 1 : EACH < 5 ? EACH : 5;  // (one token: registers count for more)
    const int up = b == t0 ? 0 : 3;  // rows between the base and row b; those before t0 are the window's
    const auto rows = row_buffer<E>(c.xbc, (size_t)(b - up), c.xbc_stride, nt + up, c.C);
    const unsigned xs = (unsigned)c.xbc_stride * (unsigned)sizeof(E);
#pragma unroll 1
    for (int e0 = 0; e0 < EACH; e0 += AT) {
      float v[AT][RUN + 3];
#pragma unroll
      for (int e = 0; e < AT; ++e) {
        const int it = (e0 + e) * 256 + tid, run = it / NC * RUN, ch = max(channel(it % NC), 0);
        const unsigned at = (unsigned)ch * (unsigned)sizeof(E) + (unsigned)(run - 3 + up) * xs;
#pragma unroll
        for (int j = 0; j < RUN + 3; ++j) v[e][j] = load_one<E>(rows, at + (unsigned)j * xs);
        if (up == 0 && run == 0 && s >= 0) {
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (3 - j < c.W) v[e][j] = (float)win[((size_t)s * W1 + j - 3 + W1) * c.C + ch];
        }
      }
#pragma unroll
      for (int e = 0; e < AT; ++e) {
        const int it = (e0 + e) * 256 + tid, k = it % NC, run = it / NC * RUN, ch = channel(k);
        float tap[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) tap[j] = 3 - j < c.W ? c.conv_w[(size_t)max(ch, 0) * c.W + c.W - 4 + j] : 0.f;
        const float bias = c.conv_b[max(ch, 0)];
        if (it >= ITEMS) continue;
#pragma unroll
        for (int t = 0; t < RUN; ++t) {
          float a = bias;
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (3 - j < c.W) a = fmaf(tap[j], v[e][t + j], a);
          if (run + t < TB) su[run + t][k] = ch < 0 || run + t >= nt ? 0.f : silu(a);
        }
      }
    }
    if (tid < TB) {  // positions past the last one leave the states as they are
      float step = 0.f;
      if (tid < nt)
        step = softplus((float)static_cast<const E*>(c.dt)[(size_t)(b + tid) * c.dt_stride + h] + c.dt_bias[h]);
      sstep[tid] = step;
      sdecay[tid] = tid < nt ? __expf(step * c.A[h]) : 1.f;
    }
    __syncthreads();
    if constexpr (TB == 1) {
      const float step = sstep[0], decay = sdecay[0];
      const float4 B = *reinterpret_cast<const float4*>(&su[0][ROWS + n0]);
      const float4 C = *reinterpret_cast<const float4*>(&su[0][ROWS + NP + n0]);
      float y[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float dx = step * su[0][r0 + r * RPP];
        S[r][0] = fmaf(S[r][0], decay, dx * B.x);
        S[r][1] = fmaf(S[r][1], decay, dx * B.y);
        S[r][2] = fmaf(S[r][2], decay, dx * B.z);
        S[r][3] = fmaf(S[r][3], decay, dx * B.w);
        y[r] = fmaf(C.x, S[r][0], fmaf(C.y, S[r][1], fmaf(C.z, S[r][2], C.w * S[r][3])));
      }
#pragma unroll
      for (int r = 0; r < R; ++r) {
        y[r] += xor_lane<1>(y[r]);
        y[r] += xor_lane<2>(y[r]);
        if constexpr (L >= 8) y[r] += xor_lane<4>(y[r]);
        if constexpr (L >= 16) y[r] += xor_lane<8>(y[r]);
        if constexpr (L >= 32) y[r] += xor_lane<16>(y[r]);
        if constexpr (L >= 64) y[r] += xor_lane<32>(y[r]);
      }
      if (tid % L == 0)
#pragma unroll
        for (int r = 0; r < R; ++r) sy[0][r0 + r * RPP] = y[r];
    } else {
      constexpr int U = 8;
      for (int u0 = 0; u0 < nt; u0 += U) {
        float y[R][U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int t = u0 + u;
          const float step = sstep[t], decay = sdecay[t];
          const float4 B = *reinterpret_cast<const float4*>(&su[t][ROWS + n0]);
          const float4 C = *reinterpret_cast<const float4*>(&su[t][ROWS + NP + n0]);
#pragma unroll
          for (int r = 0; r < R; ++r) {
            const float dx = step * su[t][r0 + r * RPP];
            S[r][0] = fmaf(S[r][0], decay, dx * B.x);
            S[r][1] = fmaf(S[r][1], decay, dx * B.y);
            S[r][2] = fmaf(S[r][2], decay, dx * B.z);
            S[r][3] = fmaf(S[r][3], decay, dx * B.w);
            y[r][u] = fmaf(C.x, S[r][0], fmaf(C.y, S[r][1], fmaf(C.z, S[r][2], C.w * S[r][3])));
          }
        }
        // lanes that differ in bit 0, 1, 3 (2 where there is none) share the eight
        // sums among them
        const int lane = tid % L;
        constexpr int M2 = L >= 16 ? 8 : 4, HALVE = L >= 8 ? 3 : 2, HAVE = U >> HALVE;
#pragma unroll
        for (int r = 0; r < R; ++r) {
          halve<1, 4>(y[r], lane);
          halve<2, 2>(y[r], lane);
          if constexpr (L >= 8) halve<M2, 1>(y[r], lane);
#pragma unroll
          for (int j = 0; j < HAVE; ++j) {
            if constexpr (L >= 16) y[r][j] += xor_lane<4>(y[r][j]);
            if constexpr (L >= 32) y[r][j] += xor_lane<16>(y[r][j]);
            if constexpr (L >= 64) y[r][j] += xor_lane<32>(y[r][j]);
          }
        }
        const int u = (lane & 1 ? 4 : 0) + (lane & 2 ? 2 : 0) + (L >= 8 && lane & M2 ? 1 : 0);
        if ((lane & ~(3 | (L >= 8 ? M2 : 0))) == 0) {
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < HAVE; ++j) sy[u0 + u + j][r0 + r * RPP] = y[r][j];
        }
      }
    }
    // All of this workgroup's reads of the window lie before the barrier above, their
    // values used; relaxed, since nothing else is handed over (a release would
    // write the whole L2 back), and looked at only at the end.
    if (b == t0 && tid == 0 && W1 > 0 && d >= 0)
      ticket = __hip_atomic_fetch_add(c.tickets + (size_t)i * c.G + g, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    for (int k = tid; k < nt * ROWS; k += 256) {
      const int t = TB > 1 ? k / ROWS : 0, r = k % ROWS;
      if (p0 + r >= c.P) continue;
      const int ch = h * c.P + p0 + r;
      float y = fmaf(skip, su[t][r], sy[t][r]);
      if (c.z) y *= silu((float)(TB == 1 ? zt : static_cast<const E*>(c.z)[(size_t)(b + t) * c.z_stride + ch]));
      static_cast<E*>(c.y)[(size_t)(b + t) * c.y_stride + ch] = (E)y;
    }
  }
  if (d < 0) return;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int p = p0 + r0 + r * RPP;
    if (p >= c.P || n0 >= c.N) continue;
    float* at = c.state + ((size_t)d * c.H + h) * head + (size_t)p * c.N + n0;
    if (quads) {
      __builtin_nontemporal_store((v4f){S[r][0], S[r][1], S[r][2], S[r][3]}, reinterpret_cast<v4f*>(at));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n0 + e < c.N) at[e] = S[r][e];
    }
  }
  // the window: x's by this workgroup, B's and C's by the last of the group; a
  // sequence without tokens has read nothing, and copies its own
  if (W1 == 0) return;
  const bool none = t0 == t1;
  if (none && s == d) return;
  if (tid == 0) {
    slast = none ? h % (c.H / c.G) == 0 && blockIdx.x == 0 : ticket == c.H / c.G * (int)gridDim.x - 1;
    if (slast && !none)
      __hip_atomic_store(c.tickets + (size_t)i * c.G + g, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  const bool shared = slast;
  for (int k = tid; k < NC; k += 256) {
    const int ch = channel(k);
    if (ch < 0 || (k >= ROWS && !shared)) continue;
    E v[3];
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (j < W1) v[j] = raw(t1 - W1 + j, ch);
#pragma unroll
    for (int j = 0; j < 3; ++j)
      if (j < W1) win[((size_t)d * W1 + j) * c.C + ch] = v[j];
  }
}

template <class E, int L, int R, int TB>
hipError_t launch_scan_of(const SsmCall& c, hipStream_t st) {
  constexpr int ROWS = R * 256 / L;
  hipLaunchKernelGGL((k_ssm_scan<E, L, R, TB>), dim3((unsigned)((c.P + ROWS - 1) / ROWS), (unsigned)c.H, (unsigned)c.n),
                     dim3(256), 0, st, c);
  return hipGetLastError();
}
constexpr int kScanBlock = 32;  // positions of a prompt in LDS

// 16 channels a workgroup while that is what fills the card, 64 where there are
// heads and sequences enough: B and C are then convolved for four times as many.
template <class E, int L, int R, int R4>
hipError_t launch_scan_rows(const SsmCall& c, hipStream_t st) {
  if (!c.step) return launch_scan_of<E, L, R, kScanBlock>(c, st);
  if ((long long)c.n * c.H * ((c.P + 63) / 64) >= 1024) return launch_scan_of<E, L, R4, 1>(c, st);
  return launch_scan_of<E, L, R, 1>(c, st);
}
template <class E>
hipError_t launch_scan(const SsmCall& c, hipStream_t st) {
  if (c.N <= 16) return launch_scan_rows<E, 4, 1, 1>(c, st);
  if (c.N <= 32) return launch_scan_rows<E, 8, 1, 2>(c, st);
  if (c.N <= 64) return launch_scan_rows<E, 16, 1, 4>(c, st);
  if (c.N <= 128) return launch_scan_rows<E, 32, 2, 8>(c, st);
  return launch_scan_rows<E, 64, 4, 16>(c, st);
}

// Up to so many tokens a prompt call goes through k_ssm_scan: one prompt of 32
// heads x 64 x 128 in bf16 takes 14 us for 29 tokens, 37 for 128 and 52 for 192
// with it (a quarter of a microsecond a token), in chunks 61 for 193 and 65 for
// 512; one of 24 heads x 64 x 64 in fp32 26 for 128 and 36 for 192, in chunks 36
// for 193 and 37 for 512.  The tokens of all sequences count, since each of many
// takes a share of the card: 24 of 8 tokens 38 us position by position, 32 of 8 42
// in chunks.
constexpr int kSsmScanTokens = 192;

// How a prompt call is cut: segments of `per` chunks so that about as many
// workgroups are on their way as there is room for at once (two or one a compute
// unit); sequences that are that many by themselves are not cut.
constexpr int ssm_workgroups(int N) { return N <= 64 ? 512 : 256; }

int head_groups(int H, int G, int P, int N) {
  const int items = H / G * ((P + 31) / 32), nw = items < ssm_waves(N) ? items : ssm_waves(N);
  return G * ((items + nw - 1) / nw);
}
// Upper bound of the segments of a call that is cut: fewer than `want` pieces
// of all chunks and one more for each of fewer than `want` sequences; `cuts`:
// chunks and sequences of the largest call.
size_t most_segments(int H, int G, int P, int N, size_t cuts) {
  const size_t most = 2 * (size_t)ssm_workgroups(N) / head_groups(H, G, P, N) + 2;
  return most < cuts ? most : cuts;
}

hipError_t launch_prompt(const SsmCall& c, int dtype, SsmScratch w, hipStream_t st) {
  w.blocks = c.T / kSsmQ + c.n;  // a sequence's last chunk may be short
  const int wgs = head_groups(c.H, c.G, c.P, c.N), want = ssm_workgroups(c.N) / wgs;
  w.per = want > c.n ? (w.blocks + want - 1) / want : w.blocks;
  w.segments = want > c.n ? w.blocks / w.per + c.n : c.n;
  const size_t e = dtype_size(dtype);
  auto two = [&](const void* p, size_t stride) { return !p || ((uintptr_t)p % (2 * e) == 0 && stride % 2 == 0); };
  w.pair = c.P % 2 == 0 && two(c.xbc, c.xbc_stride) && two(c.z, c.z_stride) && two(c.y, c.y_stride);
  w.quads = c.N % 4 == 0;
  return dtype == LCSM_F32 ? ssm_prompt_f32(c, w, st) : dtype == LCSM_BF16 ? ssm_prompt_bf16(c, w, st) : ssm_prompt_f16(c, w, st);
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
  int* tickets;
  lcsm::SsmScratch scratch;
  size_t zero_floats;  // states, windows and tickets, from `state` on
  bool faulted;
  char msg[256];
};

namespace {

size_t align256(size_t v) { return (v + 255) / 256 * 256; }

struct Plan {
  size_t state, window, tickets, conv_w, conv_b, A, skip, dt_bias, windows, bc, scal, lq, states, decay, total;
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
  take(&p->tickets, (size_t)s->slots * s->G * 4);
  take(&p->conv_w, M * c * s->W * 4);
  take(&p->conv_b, M * c * 4);
  take(&p->A, M * H * 4);
  take(&p->skip, M * H * 4);
  take(&p->dt_bias, M * H * 4);
  if (s->max_tokens > lcsm::kSsmScanTokens) {
    if (s->G + (s->H + 31) / 32 > 65534) return false;  // rows of k_ssm_bc's launch
    const size_t blocks = (size_t)s->max_tokens / lcsm::kSsmQ + s->slots;
    const size_t each = lcsm::ssm_block_bytes(s->N);
    const size_t segments = lcsm::most_segments(s->H, s->G, s->P, s->N, blocks + s->slots);
    if ((double)blocks * (s->G * (double)each + H * 2048.0) + (double)segments * D * s->N * 4 > 70368744177664.0)
      return false;
    take(&p->windows, (size_t)s->slots * (s->W - 1) * c * lcsm::dtype_size(s->dtype));
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
      if (stride > lcsm::kSsmMaxStride) return ssm_fail(c, LCSM_EINVAL, "a row stride is above 2^24 elements");
  }
  if (c->faulted) return LCSM_ESTATE;
  const size_t m = (size_t)layer, C = (size_t)c->C, H = (size_t)c->s.H;
  *k = lcsm::SsmCall{c->s.H, c->s.P, c->s.N, c->s.G, c->s.W, c->D, c->C, c->s.slots, T, n,
                     0, nullptr, io->src, io->dst, io->xbc, io->dt, io->z, io->y,
                     io->xbc_stride, io->dt_stride, io->z_stride, io->y_stride,
                     c->conv_w + m * C * c->s.W, c->conv_b + m * C, c->A + m * H, c->skip + m * H,
                     c->dt_bias + m * H, c->state + m * c->s.slots * (size_t)c->D * c->s.N,
                     c->window + m * c->s.slots * (c->s.W - 1) * C * lcsm::dtype_size(c->s.dtype), c->tickets};
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
  c->tickets = (int*)(c->mem + p.tickets);
  c->zero_floats = (p.conv_w - p.state) / 4;
  c->conv_w = (float*)(c->mem + p.conv_w);
  c->conv_b = (float*)(c->mem + p.conv_b);
  c->A = (float*)(c->mem + p.A);
  c->skip = (float*)(c->mem + p.skip);
  c->dt_bias = (float*)(c->mem + p.dt_bias);
  if (shape->max_tokens > lcsm::kSsmScanTokens) {
    c->scratch.windows = c->mem + p.windows;
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
  hipError_t e;
  if (T <= lcsm::kSsmScanTokens)
    e = lcsm::with_dtype(ctx->s.dtype, [&](auto v) { return lcsm::launch_scan<decltype(v)>(k, ctx->stream); });
  else
    e = lcsm::launch_prompt(k, ctx->s.dtype, ctx->scratch, ctx->stream);
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
