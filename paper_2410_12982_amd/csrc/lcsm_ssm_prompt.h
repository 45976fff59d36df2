// Prompts of the state space mixer in chunks of 64 positions on the matrix
// units; included by one source per element type.
//
// Within a chunk let l_t be the sum of the steps' log2-decays up to t, e the last
// position of t's half (32 positions) of the chunk, w_t = step_t 2^(l_e - l_t)
// and E_t = 2^(l_t - l_e).  The recurrence unrolled over a half is, per head,
//
//   y_t  = E_t [ C (2^l_e S)^T + tril(C B^T) (w o x) ]_t,
//   S'   = 2^l_e S + (w o x)^T B,
//
// and over the chunk the same with the first half's share of the second one's
// rows, and of S, multiplied by the second one's decay in between:
//
// three matrix products in which only w o x, S and the row factor E belong to
// the head: B, C and tril(C B^T) are made once per chunk and group, by
// k_ssm_bc, already as matrix operands, and staged in LDS for the heads of a
// workgroup.  A wave has 32 channels of a head (lane: two neighbouring ones)
// and keeps their states in registers as the products' accumulators; with the
// K index of a product ordered as below, an accumulator of S is the right
// operand of C S^T as it stands, and the lane that convolves x at a position
// is the one that gets y there, so nothing of a head goes through LDS.
//
// E and w stay within 2^64 of each other while the halves' decays do; where they
// do not (steps that forget everything), the factor 2^(l_t - l_s) <= 1 is put
// into the elements of tril(C B^T) one by one instead (`fast` false).
//
// Values go into the products as sums of three bf16 parts, which hold fp32's range
// (fp16 would not) and all of its bits; the six products above 2^-24 make sums as
// good as fp32's.  Two parts and three products would be good to 2^-16 of the
// terms: enough for outputs of 16 bits as long as the terms do not cancel (16384
// tokens of 64 heads x 64 x 128 in bf16 388 us in all, 462 now).
//
// A call is four launches: k_ssm_bc; where sequences are cut into segments, what
// each segment adds (k_ssm_chunks without OUT) and the states before them
// (k_ssm_join); and the outputs.
//
// A product with a value that is not finite reaches positions before it as 0 *
// inf; where the state shows such a value, the affected channels' products are
// made without it and their rows from it on set to NaN.
#pragma once

#include "lcsm_ssm_internal.h"

namespace lcsm {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef bf16_t v8bf __attribute__((ext_vector_type(8)));
typedef bf16_t v2bf __attribute__((ext_vector_type(2)));

// K slots of a 16x16x32 product: lane quarter q holds, in this order, 4q .. 4q+3
// and 16 + 4q .. 16 + 4q+3 of the block's 32, which are the rows that it holds
// of two 16x16 accumulators.
//
// c[e] += a b[e] with both in parts, the small products first.
template <int P, int Q>
__device__ __forceinline__ void mul(const v8bf (&a)[P], const v8bf (&b)[2][Q], v4f (&c)[2]) {
#pragma unroll
  for (int sum = P - 1; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i <= sum; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) c[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[e][sum - i], c[e], 0, 0, 0);
}

// Eight values as an operand's parts: each the bf16 nearest to what the parts
// before it leave.
template <int P>
__device__ __forceinline__ void split(float (&v)[8], v8bf (&to)[P]) {
#pragma unroll
  for (int p = 0; p < P; ++p) {
    v4u w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const v2bf two = {(bf16_t)v[2 * k], (bf16_t)v[2 * k + 1]};
      w[k] = __builtin_bit_cast(unsigned, two);
      if (p + 1 < P) {
        v[2 * k] -= __builtin_bit_cast(float, w[k] << 16);
        v[2 * k + 1] -= __builtin_bit_cast(float, w[k] & 0xffff0000u);
      }
    }
    to[p] = __builtin_bit_cast(v8bf, w);
  }
}

// The piece [*k0, *k1) of `per` chunks (and its sequence, its number in it and
// the sequence's chunks) that has number `want` when the pieces of all
// sequences are counted one after another, every sequence having at least
// `least`; false past the last one.  All lanes of a wave together.
__device__ __forceinline__ bool ssm_piece(const SsmCall& c, int want, int per, int least, int& seq, int& num,
                                          int& chunks) {
  const int lane = (int)threadIdx.x & 63;
  int base = 0;
  for (int i0 = 0; i0 < c.n; i0 += 64) {
    int mine = 0, ch = 0;
    if (i0 + lane < c.n) {
      int t0, t1;
      ssm_rows(c, i0 + lane, t0, t1);
      ch = (t1 - t0 + kSsmQ - 1) / kSsmQ;
      mine = max((ch + per - 1) / per, least);
    }
    int sum = mine;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
      const int v = __shfl_up(sum, m);
      if (lane >= m) sum += v;
    }
    const int total = __shfl(sum, 63);
    if (want < base + total) {
      const unsigned long long past = __ballot(base + sum > want);
      const int who = __ffsll(past) - 1;
      seq = __builtin_amdgcn_readfirstlane(i0 + who);
      num = __builtin_amdgcn_readfirstlane(want - base - __shfl(sum - mine, who));
      chunks = __builtin_amdgcn_readfirstlane(__shfl(ch, who));
      return true;
    }
    base += total;
  }
  return false;
}

// Two neighbouring channels as they come.
template <class E>
struct Two {
  unsigned v;
  __device__ float lo() const { return (float)__builtin_bit_cast(E, (unsigned short)v); }
  __device__ float hi() const { return (float)__builtin_bit_cast(E, (unsigned short)(v >> 16)); }
  __device__ void set(float a, float b) {
    v = __builtin_bit_cast(unsigned short, (E)a) | (unsigned)__builtin_bit_cast(unsigned short, (E)b) << 16;
  }
};
template <>
struct Two<float> {
  unsigned a, b;
  __device__ float lo() const { return __builtin_bit_cast(float, a); }
  __device__ float hi() const { return __builtin_bit_cast(float, b); }
  __device__ void set(float x, float y) {
    a = __builtin_bit_cast(unsigned, x);
    b = __builtin_bit_cast(unsigned, y);
  }
};

template <class E, bool PAIR>
__device__ __forceinline__ Two<E> load_two(__amdgpu_buffer_rsrc_t r, unsigned at) {
  Two<E> t;
  if constexpr (sizeof(E) == 4) {
    if constexpr (PAIR) {
      const auto v = __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0);
      t.a = v[0];
      t.b = v[1];
    } else {
      t.a = __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
      t.b = __builtin_amdgcn_raw_buffer_load_b32(r, at + 4, 0, 0);
    }
  } else if constexpr (PAIR) {
    t.v = __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0);
  } else {
    const unsigned a = __builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0);
    const unsigned b = __builtin_amdgcn_raw_buffer_load_b16(r, at + 2, 0, 0);
    t.v = a | b << 16;
  }
  return t;
}
// `second`: where the second channel goes by itself.
template <class E, bool PAIR>
__device__ __forceinline__ void store_two(Two<E> t, __amdgpu_buffer_rsrc_t r, unsigned at, unsigned second) {
  if constexpr (sizeof(E) == 4) {
    if constexpr (PAIR) {
      typedef unsigned v2u __attribute__((ext_vector_type(2)));
      __builtin_amdgcn_raw_buffer_store_b64((v2u){t.a, t.b}, r, at, 0, 0);
    } else {
      __builtin_amdgcn_raw_buffer_store_b32(t.a, r, at, 0, 0);
      __builtin_amdgcn_raw_buffer_store_b32(t.b, r, second, 0, 0);
    }
  } else if constexpr (PAIR) {
    __builtin_amdgcn_raw_buffer_store_b32(t.v, r, at, 0, 0);
  } else {
    __builtin_amdgcn_raw_buffer_store_b16((unsigned short)t.v, r, at, 0, 0);
    __builtin_amdgcn_raw_buffer_store_b16((unsigned short)(t.v >> 16), r, second, 0, 0);
  }
}

// What a chunk's positions have of a head, a position a lane: w, then E where
// the chunk is `fast`, else step and l in two parts.
__device__ __forceinline__ bool ssm_fast(double l0, double l1) { return fabs(l0) < 64.0 && fabs(l1) < 64.0; }

constexpr int kSsmHeads = 4;  // heads a wave, at once
constexpr int kSsmWaves = 8;  // waves of a workgroup of k_ssm_bc

template <class E>
__device__ __forceinline__ void ssm_decays(const SsmCall& c, const SsmScratch& w, int block, int r0, int rows, int h0) {
  const int lane = (int)threadIdx.x & 63;
  float step[kSsmHeads];
  double l[kSsmHeads];  // fp64: l reaches thousands where steps are long, and its differences count
#pragma unroll
  for (int j = 0; j < kSsmHeads; ++j)
    step[j] = (float)static_cast<const E*>(c.dt)[(size_t)(r0 + min(lane, rows - 1)) * c.dt_stride + min(h0 + j, c.H - 1)];
#pragma unroll
  for (int j = 0; j < kSsmHeads; ++j) {
    const int h = min(h0 + j, c.H - 1);
    step[j] = lane < rows ? softplus(step[j] + c.dt_bias[h]) : 0.f;
    l[j] = (double)(step[j] * c.A[h]) * 1.4426950408889634;
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2)
#pragma unroll
    for (int j = 0; j < kSsmHeads; ++j) {
      const double v = __shfl_up(l[j], m);
      if (lane >= m) l[j] += v;
    }
#pragma unroll
  for (int j = 0; j < kSsmHeads; ++j) {
    if (h0 + j >= c.H) break;
    const double l0 = __shfl(l[j], 31), lq = __shfl(l[j], 63), le = lane < 32 ? l0 : lq;
    const size_t at = (size_t)block * c.H + h0 + j;
    float* to = w.scal + at * 4 * kSsmQ + lane;
    to[0] = step[j] * exp2_hw((float)(le - l[j]));
    const float hi = (float)l[j];
    to[kSsmQ] = ssm_fast(l0, lq - l0) ? exp2_hw((float)(l[j] - le)) : step[j];
    to[2 * kSsmQ] = hi;
    to[3 * kSsmQ] = (float)(l[j] - (double)hi);
    if (lane < 2) w.lq[2 * at + lane] = lane ? lq - l0 : l0;
  }
}

// The windows that the call begins from, put where no sequence of the call
// writes (zeros for a new one): a workgroup a sequence.
template <class E>
__device__ __forceinline__ void ssm_keep_window(const SsmCall& c, const SsmScratch& w, int seq) {
  const int s = ssm_slot(c.src, seq, c.slots);
  const size_t each = (size_t)(c.W - 1) * c.C;
  const E* from = static_cast<const E*>(c.window) + (s >= 0 ? s * each : 0);
  E* to = static_cast<E*>(w.windows) + seq * each;
  for (size_t k = threadIdx.x; k < each; k += 64 * kSsmWaves) to[k] = s >= 0 ? from[k] : (E)0.f;
}

// The windows after a call: channels `first`, `first` + `step` .. of a sequence.
template <class E>
__device__ __forceinline__ void ssm_window(const SsmCall& c, const SsmScratch& w, int seq, int first, int step) {
  int t0, t1;
  ssm_rows(c, seq, t0, t1);
  const int d = ssm_slot(c.dst, seq, c.slots), W1 = c.W - 1;
  if (d < 0) return;
  const E* x = static_cast<const E*>(c.xbc);
  const E* before = static_cast<const E*>(w.windows) + (size_t)seq * W1 * c.C;
  E* to = static_cast<E*>(c.window) + (size_t)d * W1 * c.C;
  for (int ch = first; ch < c.C; ch += step)
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      if (k >= W1) continue;
      const int t = t1 - W1 + k;
      to[(size_t)k * c.C + ch] = t >= t0 ? x[(size_t)t * c.xbc_stride + ch] : before[(size_t)(t - t0 + W1) * c.C + ch];
    }
}
template <class E>
__global__ __launch_bounds__(256) void k_ssm_window(SsmCall c, SsmScratch w) {
  ssm_window<E>(c, w, (int)blockIdx.y, (int)(blockIdx.x * 256 + threadIdx.x), (int)gridDim.x * 256);
}

// B, C and tril(C B^T) of one chunk and group as operands (SsmBlock); and in
// workgroups of their own, at the same time, what the chunk's positions have of
// the heads, and the windows (two launches less: 62 -> 56 us for 4198 tokens of 15
// heads x 48 x 40 with two parts a value).  Bound by the latency of a chunk's three
// steps, so by eight waves: 16384 tokens of 64 heads x 64 x 128 20 us, 26 with four;
// 11 and 13 for the former.
template <class E, int NT>
__global__ __launch_bounds__(64 * kSsmWaves) void k_ssm_bc(SsmCall c, SsmScratch w) {
  constexpr int NP = 32 * NT, LD = NP + 4;
  typedef SsmBlock<NT> Blk;
  __shared__ __align__(16) float lb[kSsmQ * LD];
  __shared__ __align__(16) float lc[kSsmQ * LD];
  const int g = (int)blockIdx.y, tid = (int)threadIdx.x;
  if ((int)blockIdx.y == (int)gridDim.y - 1) {
    if ((int)blockIdx.x < c.n) ssm_keep_window<E>(c, w, (int)blockIdx.x);
    return;
  }
  int seq, num, chunks;
  if ((int)blockIdx.x >= w.blocks || !ssm_piece(c, (int)blockIdx.x, 1, 0, seq, num, chunks)) return;
  int t0, t1;
  ssm_rows(c, seq, t0, t1);
  const int s = ssm_slot(c.src, seq, c.slots), r0 = t0 + num * kSsmQ, rows = min(kSsmQ, t1 - r0);
  if (g >= c.G) {
    const int h = ((g - c.G) * kSsmWaves + __builtin_amdgcn_readfirstlane(tid / 64)) * kSsmHeads;
    if (h < c.H) ssm_decays<E>(c, w, (int)blockIdx.x, r0, rows, h);
    return;
  }
  // a thread convolves one channel along a quarter of the chunk's rows, all of
  // which are loaded at once (zeros before the sequence and past it)
  constexpr int RUN = kSsmQ / 4;
  for (int k = tid; k < 2 * NP * 4; k += 64 * kSsmWaves) {
    // (whole waves have the same rows: 64 divides 2 NP, or they are padding)
    const int col = k % (2 * NP), run = __builtin_amdgcn_readfirstlane(k / (2 * NP)) * RUN;
    const int n = col % NP;
    const int ch = c.D + (col < NP ? 0 : c.G * c.N) + g * c.N + min(n, c.N - 1);
    const int up = num == 0 && run == 0 ? 0 : 3, base = r0 + run - up;
    const auto r = row_buffer<E>(c.xbc, base, c.xbc_stride, min(t1 - base, RUN + 3), c.C);
    const unsigned xs = (unsigned)c.xbc_stride * (unsigned)sizeof(E), at = (unsigned)ch * (unsigned)sizeof(E);
    float x[RUN + 3];
#pragma unroll
    for (int j = 0; j < RUN + 3; ++j) x[j] = load_one<E>(r, at + (unsigned)(j - 3 + up) * xs);
    if (up == 0 && s >= 0) {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (3 - j < c.W)
          x[j] = (float)static_cast<const E*>(c.window)[((size_t)s * (c.W - 1) + j - 3 + c.W - 1) * c.C + ch];
    }
    float tap[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) tap[j] = 3 - j < c.W ? c.conv_w[(size_t)ch * c.W + c.W - 4 + j] : 0.f;
    const float bias = c.conv_b[ch];
    float* to = (col < NP ? lb : lc) + run * LD + n;
    float v[RUN];
#pragma unroll
    for (int t = 0; t < RUN; ++t) v[t] = bias;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (3 - j >= c.W) continue;
#pragma unroll
      for (int t = 0; t < RUN; ++t) v[t] = fmaf(tap[j], x[t + j], v[t]);
    }
#pragma unroll
    for (int t = 0; t < RUN; ++t) to[t * LD] = run + t < rows && n < c.N ? silu(v[t]) : 0.f;
  }
  __syncthreads();
  char* out = w.bc + ((size_t)blockIdx.x * c.G + g) * Blk::BYTES;
  const int lane = tid & 63, wv = tid >> 6, q = lane >> 4, l = lane & 15;
  auto put = [&](int at, int step, float (&v)[8]) {
    v8bf w[kSsmParts];
    split(v, w);
#pragma unroll
    for (int k = 0; k < kSsmParts; ++k) reinterpret_cast<v8bf*>(out + at + k * step)[lane] = w[k];
  };
  for (int f = wv; f < 4 * NT; f += kSsmWaves) {
    const int tt = f / NT, cc = f % NT;
    const float* p = lc + (16 * tt + l) * LD + 32 * cc + 4 * q;
    float v[8] = {p[0], p[1], p[2], p[3], p[16], p[17], p[18], p[19]};
    put(Blk::c_at(tt, cc), Blk::PART, v);
  }
  for (int f = wv; f < 4 * NT; f += kSsmWaves) {
    const int a = f / 2, b = f % 2;
    const float* p = lb + (32 * b + 4 * q) * LD + 16 * a + l;
    float v[8] = {p[0], p[LD], p[2 * LD], p[3 * LD], p[16 * LD], p[17 * LD], p[18 * LD], p[19 * LD]};
    put(Blk::b_at(a, b), Blk::PART, v);
  }
  // (C B^T)[t][s] with t a lane's column of the accumulator: rows 4q + i of it
  // are the lane's slots
  for (int f = wv; f < 6; f += kSsmWaves) {
    const int tt = f < 2 ? f : 2 + (f - 2) / 2, cc = f < 2 ? 0 : (f - 2) % 2;
    float v[8];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int st = 2 * cc + half;
      v4f acc = {0.f, 0.f, 0.f, 0.f};
      if (st <= tt) {
        const float* pb = lb + (16 * st + l) * LD + q;
        const float* pc = lc + (16 * tt + l) * LD + q;
#pragma unroll 8
        for (int k = 0; k < NP / 4; ++k)
          acc = __builtin_amdgcn_mfma_f32_16x16x4f32(pb[4 * k], pc[4 * k], acc, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) v[4 * half + i] = 16 * st + 4 * q + i <= 16 * tt + l ? acc[i] : 0.f;
    }
    put(Blk::g_at(f), Blk::GPART, v);
  }
}

// v, with what is made of it made here: sums of it and of what is the same in
// every turn of a loop are not kept in registers from one turn to the next.
__device__ __forceinline__ unsigned here(unsigned v) {
  asm volatile("" : "+v"(v));
  return v;
}

// All waves past their LDS accesses; loads and stores of global memory stay on
// their way, which __syncthreads would wait for.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// One segment (w.per chunks) of a sequence: OUT, with its outputs and from the
// state before it; else its own contribution to the state after it.
//
// 16384 tokens of 64 heads x 64 x 128 in bf16: OUT 360 us, the contributions 121
// (join 14, operands 21; so traced, one launch at a time.  Passes after one another
// take 443).  What bounds it is issue: 1960 vector instructions (the convolution,
// two SiLUs, parts of states and operands, decays) and 456 matrix instructions of
// 16 cycles a wave and chunk keep a SIMD's vector unit 53 % and its matrix unit 38 %
// of the time, and the two hardly overlap.  All 256 registers are taken: OUT spills
// 27 for 65 to 128 states (59 in fp32) and 17 for 33 to 64 (33).  Of a chunk's transfers only the next chunk's first stage is on its way
// under products: the waits for the chunk's rows and for the decays of its halves,
// which the compiler cannot count apart from transfers of unknown number, wait for
// the second stage and G before the first product.  Tried, with two parts a value:
// half of the waves a stage behind the others, 412 against 383 us in all; 128
// states at once without a second copy, 447; wave priorities, nothing.  4198 tokens
// of 15 heads x 48 x 40 take 27 and 15 us, which is two chunks' latency.
template <class E, int NT, bool OUT, bool PAIR>
__global__ __launch_bounds__(NT == 4 ? 512 : 256, NT > 4 ? 1 : 2) void k_ssm_chunks(SsmCall c, SsmScratch w) {
  constexpr int PS = kSsmParts;
  typedef SsmBlock<NT> Blk;
  typedef SsmLds<NT, OUT> Lds;
  constexpr int NA = 2 * NT, NB = Blk::NB, STAGES = Blk::STAGES;
  extern __shared__ __align__(16) char lds[];
  const int lane = (int)threadIdx.x & 63, q = lane >> 4, l = lane & 15;
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), nw = (int)blockDim.x >> 6;
  // workgroups of one segment share its operands: every eighth one, as an XCD
  // (and its L2) gets them
  const int hg = c.H / c.G, parts = (c.P + 31) / 32, items = hg * parts;
  const int wgs = (items + nw - 1) / nw;
  const int wg = (int)blockIdx.x / 8, segment = (int)blockIdx.y * 8 + (int)blockIdx.x % 8;
  if (segment >= w.segments) return;
  int seq, num, chunks;
  if (!ssm_piece(c, segment, w.per, 1, seq, num, chunks)) return;
  const bool last = (num + 1) * w.per >= chunks;
  if (!OUT && last) return;
  int t0, t1;
  ssm_rows(c, seq, t0, t1);
  t0 = __builtin_amdgcn_readfirstlane(t0);
  t1 = __builtin_amdgcn_readfirstlane(t1);
  const int src = __builtin_amdgcn_readfirstlane(ssm_slot(c.src, seq, c.slots));
  const int dst = __builtin_amdgcn_readfirstlane(ssm_slot(c.dst, seq, c.slots));
  // the first block of this sequence, counted as k_ssm_bc does
  int block0 = 0;
  for (int i = lane; i < seq; i += 64) {
    int a, b;
    ssm_rows(c, i, a, b);
    block0 = min(block0 + (b - a + kSsmQ - 1) / kSsmQ, w.blocks);  // (wrong offsets do not overflow it)
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) block0 += __shfl_xor(block0, m);
  block0 = __builtin_amdgcn_readfirstlane(block0);
  // (offsets that do not rise could count more blocks than there are)
  const int k0 = num * w.per, k1 = min(min(k0 + w.per, chunks), w.blocks - block0);

  // head and channels of this wave; a wave past the last one works on the last
  // one's data and stores nothing
  const int g = wg / wgs, item = wg % wgs * nw + wv;
  const bool live = item < items;
  const int it = live ? item : items - 1;
  const int h = g * hg + it / parts, p = (it % parts) * 32 + 2 * l;
  const int have = min(max(c.P - p, 0), 2);  // channels this lane has
  const int ch = h * c.P + p;                // x, z, y
  float tap[2][4], bias[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int cc = min(ch + e, c.D - 1);
    bias[e] = c.conv_b[cc];
#pragma unroll
    for (int j = 0; j < 4; ++j) tap[e][j] = 3 - j < c.W ? c.conv_w[(size_t)cc * c.W + c.W - 4 + j] : 0.f;
  }
  const float skip = c.skip[h];

  constexpr unsigned kNowhere = 0xC0000000u;  // past every buffer here
  v4f S[NA][2];  // n = 16 a + 4 q + i, channel p + e
  // a head's states as a buffer; quads: four states are aligned as one
  const unsigned sq = ((unsigned)p * c.N + 4 * q) * 4;
  auto state_buffer = [&](const float* head) {
    return uniform_buffer(head, (unsigned)c.P * c.N * 4);
  };
  auto state_at = [&](int a, int e, int i) {
    return e < have && 16 * a + 4 * q + i < c.N ? sq + (unsigned)(e * c.N + 16 * a + i) * 4 : kNowhere;
  };
  auto get_state = [&](__amdgpu_buffer_rsrc_t r, int a, int e) {
    if (w.quads) return __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(r, state_at(a, e, 0), 0, 0));
    v4f v;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, state_at(a, e, i), 0, 0));
    return v;
  };
  auto put_state = [&](float* head) {
    if (!live) return;
    const auto r = state_buffer(head);
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (w.quads) {
          __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, S[a][e]), r, state_at(a, e, 0), 0, 0);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = S[a][e][i];  // (a bit cast of the element itself takes the first one)
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), r, state_at(a, e, i), 0, 0);
          }
        }
      }
  };
  const size_t per_head = (size_t)c.P * c.N;
#pragma unroll
  for (int a = 0; a < NA; ++a)
#pragma unroll
    for (int e = 0; e < 2; ++e) S[a][e] = v4f{0.f, 0.f, 0.f, 0.f};
  // A sequence in one segment begins from its slot.  Of one in several the last
  // may be done, and dst may be src, before another has begun: k_ssm_join has put
  // the state before each segment where the segment's contribution was.
  const float* from_state = nullptr;
  if (OUT && chunks > w.per)
    from_state = w.states + ((size_t)segment * c.H + h) * per_head;
  else if (OUT && src >= 0)
    from_state = c.state + ((size_t)src * c.H + h) * per_head;
  if (from_state) {
    const auto r = state_buffer(from_state);
#pragma unroll
    for (int a = 0; a < NA; ++a)
#pragma unroll
      for (int e = 0; e < 2; ++e) S[a][e] = get_state(r, a, e);
  }

  constexpr unsigned ES = sizeof(E);
  const unsigned xs = (unsigned)c.xbc_stride * ES, xq = 4 * q * xs + (unsigned)ch * ES;
  const unsigned zs = (unsigned)c.z_stride * ES, zq = 4 * q * zs + (unsigned)ch * ES;
  const unsigned ys = (unsigned)c.y_stride * ES, yq = live && have > 0 ? 4 * q * ys + (unsigned)ch * ES : kNowhere;
  const unsigned yq2 = live && have > 1 ? yq + ES : kNowhere;
  // rows 16 m + 4 q - 3 .. + 3 of chunk k, zeros before the sequence and past it
  Two<E> raw[4][7];
  auto load_rows = [&](int k) {
    const int r0 = t0 + k * kSsmQ;
    const unsigned from = here(xq);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int up = k == 0 && m == 0 ? 0 : 3;  // rows between the base and row 16 m
      const int base = r0 + 16 * m - up;
      const auto r = row_buffer<E>(c.xbc, base, c.xbc_stride, min(t1 - base, 22), c.C);
#pragma unroll
      for (int j = 0; j < 7; ++j) raw[m][j] = load_two<E, PAIR>(r, from + (unsigned)(j - 3 + up) * xs);
    }
  };

  // the next chunk's rows are loaded under this one's products, where there are
  // registers for them (16384 tokens of 64 heads x 64 x 64 in bf16: with OUT 388 us
  // in all, 357 without)
  constexpr bool AHEAD = sizeof(E) == 2 && !OUT;
  // 1024 bytes at `at` of a buffer into LDS, 16 a lane.  The compiler does not wait
  // for these where LDS is read: every read comes after an arrived() of the wave
  // that fetched it, and after a barrier where that is another wave.
  auto fetch = [&](__amdgpu_buffer_rsrc_t r, int at, int to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds + to), 16, lane * 16, at, 0, 0);
  };
  auto fetch_part = [&](__amdgpu_buffer_rsrc_t r, int at, int to, int bytes) {
    for (int i = wv * 1024; i < bytes; i += nw * 1024) fetch(r, at + i, to + i);
  };
  auto operands_of = [&](int k) {
    return uniform_buffer(w.bc + ((size_t)(block0 + k) * c.G + g) * Blk::BYTES, Blk::BYTES);
  };
  auto stage_at = [&](int k, int stage) { return Lds::TWICE ? (k * STAGES + stage) % 2 * Lds::STAGE : 0; };
  auto scal_at = [&](int k) { return Lds::WAVES + ((Lds::TWICE ? k % 2 * nw : 0) + wv) * Lds::SCAL; };
  // stage `stage` of chunk k; with the first one what the positions have, with
  // the last one G
  auto fetch_stage = [&](int k, int stage) {
    fetch_part(operands_of(k), stage * Blk::STAGE + (OUT ? 0 : PS * Blk::PART), stage_at(k, stage), Lds::STAGE);
    if (stage == 0) fetch(uniform_buffer(w.scal + ((size_t)(block0 + k) * c.H + h) * 4 * kSsmQ, Lds::SCAL), 0, scal_at(k));
  };
  auto arrived = [&]() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };
  if (k0 < k1) {
    const int k = OUT ? k0 : k1 - 1;
    if (AHEAD) load_rows(k);
    if (Lds::TWICE) {
      fetch_stage(k, 0);
      arrived();
    }
  }

  double total = 0.0;  // log2 of the segment's decay
  // A segment's own contribution is taken from its end: with the decay from there
  // in w, its chunks only add up.
  for (int turn = k0; turn < k1; ++turn) {
    // (kept in a vector register otherwise)
    const int k = __builtin_amdgcn_readfirstlane(OUT ? turn : k0 + k1 - 1 - turn);
    const int next = OUT ? k + 1 : k - 1;
    const bool more = turn + 1 < k1;
    const int r0 = t0 + k * kSsmQ, rows = min(kSsmQ, t1 - r0);
    if (!AHEAD) load_rows(k);
    lds_barrier();  // the stage before has been read (TWICE: this one is there)
    fetch_stage(k, Lds::TWICE ? 1 : 0);
    if (OUT) fetch_part(operands_of(k), Blk::G, Lds::G, Blk::GBYTES);
    const double* lq = w.lq + 2 * ((size_t)(block0 + k) * c.H + h);
    const double l0 = lq[0], l1 = lq[1];
    const float f1 = OUT ? 1.f : exp2_hw((float)total), f0 = OUT ? 1.f : exp2_hw((float)(total + l1));
    total += l0 + l1;
    const bool fast = ssm_fast(l0, l1);
    const float dq0 = exp2_hw((float)l0), dq1 = exp2_hw((float)l1);
    const float* pw = reinterpret_cast<const float*>(lds + scal_at(k));
    const float *pe = pw + kSsmQ, *plh = pw + 2 * kSsmQ, *pll = pw + 3 * kSsmQ;
    Two<E> z[4][4];

    // x convolved: positions 16 m + 4 q + i, zeros past the sequence
    if (k == 0 && src >= 0 && q == 0) {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (3 - j < c.W) {
          const E* at = static_cast<const E*>(w.windows) + ((size_t)seq * (c.W - 1) + (j - 3 + c.W - 1)) * c.C + ch;
          raw[0][j].set(have > 0 ? (float)at[0] : 0.f, have > 1 ? (float)at[1] : 0.f);
        }
    }
    float u[4][4][2];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) u[m][i][0] = bias[0], u[m][i][1] = bias[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (3 - j >= c.W) continue;  // a tap that is not there multiplies nothing, were it inf
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          u[m][i][0] = fmaf(tap[0][j], raw[m][i + j].lo(), u[m][i][0]);
          u[m][i][1] = fmaf(tap[1][j], raw[m][i + j].hi(), u[m][i][1]);
        }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) u[m][i][0] = silu(u[m][i][0]), u[m][i][1] = silu(u[m][i][1]);
    if (rows < kSsmQ) {
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * m + 4 * q + i >= rows) u[m][i][0] = u[m][i][1] = 0.f;
    }
    // u by a factor for every position, as the right operand of position block b
    auto operand = [&](const float* by, int b, int e, auto& to) {
      v4f w0 = *reinterpret_cast<const v4f*>(by + 32 * b + 4 * q);
      v4f w1 = *reinterpret_cast<const v4f*>(by + 32 * b + 16 + 4 * q);
      if (!OUT) {
        w0 *= b ? f1 : f0;
        w1 *= b ? f1 : f0;
      }
      float v[8];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = u[2 * b][i][e] * w0[i];
        v[4 + i] = u[2 * b + 1][i][e] * w1[i];
      }
      split(v, to);
    };
    auto frag = [&](int at, int step, auto& to) {
#pragma unroll
      for (int k = 0; k < (int)(sizeof(to) / sizeof(to[0])); ++k)
        to[k] = *reinterpret_cast<const v8bf*>(lds + at + k * step + lane * 16);
    };
    v8bf xs[2][2][PS];  // w o x, made once where there are registers to keep it
    if (!OUT) {
      if (!Lds::TWICE) arrived();  // w, which this wave has fetched for itself (TWICE: in the turn before)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e) operand(pw, b, e, xs[b][e]);
    }
    v4f y[4][2];
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
      for (int e = 0; e < 2; ++e) y[tt][e] = v4f{0.f, 0.f, 0.f, 0.f};
    int bad[2] = {kSsmQ, kSsmQ};
#pragma unroll
    for (int stage = 0; stage < STAGES; ++stage) {
      constexpr int NF = 4 * NB;  // fragments of C
      const int a0 = 2 * stage * NB, a1 = a0 + 2 * NB, lds_c = stage_at(k, stage), lds_b = lds_c + Lds::C;
      const bool final = stage == STAGES - 1;
      if (!Lds::TWICE) {
        arrived();
        lds_barrier();
      } else if (stage > 0) {
        arrived();
        lds_barrier();  // the stage before has been read, this one is there
        if (!final)
          fetch_stage(k, stage + 1);
        else if (more)
          fetch_stage(next, 0);
      }
      if (final) {
        // under the products: this chunk's gates, or the next one's rows
        if (OUT && c.z) {
          const unsigned from = here(zq);
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const auto r = row_buffer<E>(c.z, r0 + 16 * m, c.z_stride, min(rows - 16 * m, 16), c.D);
#pragma unroll
            for (int i = 0; i < 4; ++i) z[m][i] = load_two<E, PAIR>(r, from + i * zs);
          }
        }
        if (AHEAD) load_rows(max(next, k0));  // (once more than is needed: nothing depends on them then)
      }
      if (OUT) {
        if (fast) {
#pragma unroll
          for (int a = a0; a < a1; ++a)
#pragma unroll
            for (int e = 0; e < 2; ++e) S[a][e] *= dq0;
        }
        // fragments are read one ahead of their products
        v8bf cp[2][PS], sp[2][PS];
        frag(lds_c, Blk::PART, cp[0]);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
          const int cc = stage * NB + f / 4, tt = f % 4;
          if (f + 1 < NF) frag(lds_c + ((f + 1) % 4 * NB + (f + 1) / 4) * 1024, Blk::PART, cp[(f + 1) & 1]);
          if (tt == 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float v[8];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                v[i] = S[2 * cc][e][i];
                v[4 + i] = S[2 * cc + 1][e][i];
              }
              split(v, sp[e]);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          mul(cp[f & 1], sp, y[tt]);
        }
        if (!fast && final) {
          // rows by 2^l_t; the products below have the elements' own decays
#pragma unroll
          for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int t = 16 * tt + 4 * q + i;
              const float f = exp2_hw(plh[t] + pll[t]);
#pragma unroll
              for (int e = 0; e < 2; ++e) y[tt][e][i] *= f;
            }
        }
      }
      if (OUT && !fast) {
#pragma unroll
        for (int a = a0; a < a1; ++a)
#pragma unroll
          for (int e = 0; e < 2; ++e) S[a][e] *= dq0;
      }
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        v8bf xp[2][PS], bp[2][PS];  // w o x; B
        frag(lds_b + b * 1024, Blk::PART, bp[0]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (OUT) {
            operand(pw, b, e, xp[e]);
          } else {
#pragma unroll
            for (int p = 0; p < PS; ++p) xp[e][p] = xs[b][e][p];
          }
        }
        if (OUT && b) {
#pragma unroll
          for (int a = a0; a < a1; ++a)
#pragma unroll
            for (int e = 0; e < 2; ++e) S[a][e] *= dq1;
        }
#pragma unroll
        for (int f = 0; f < 2 * NB; ++f) {
          if (f + 1 < 2 * NB) frag(lds_b + (2 * f + 2 + b) * 1024, Blk::PART, bp[(f + 1) & 1]);
          __builtin_amdgcn_sched_barrier(0);
          mul(bp[f & 1], xp, S[a0 + f]);
        }
        if (!OUT || !final) continue;
        if (b && fast) {
#pragma unroll
          for (int tt = 2; tt < 4; ++tt)
#pragma unroll
            for (int e = 0; e < 2; ++e) y[tt][e] *= dq1;
        }
        v8bf yp[2][PS];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (fast) {
#pragma unroll
            for (int k = 0; k < PS; ++k) yp[e][k] = xp[e][k];
          } else {
            operand(pe, b, e, yp[e]);
          }
        }
        // a value of w o x that is not finite shows in every state of its channel
        const bool odd = !(fabsf(S[0][0][0]) < INFINITY) || !(fabsf(S[0][1][0]) < INFINITY);
        if (__ballot(odd)) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            v4u part[PS];
#pragma unroll
            for (int k = 0; k < PS; ++k) part[k] = __builtin_bit_cast(v4u, yp[e][k]);
#pragma unroll
            for (int j = 7; j >= 0; --j) {
              const unsigned half = j & 1 ? 0xffff0000u : 0xffffu, top = half & 0x7f807f80u;
              if ((part[0][j / 2] & top) != top) continue;
#pragma unroll
              for (int k = 0; k < PS; ++k) part[k][j / 2] &= ~half;
              bad[e] = min(bad[e], 32 * b + (j < 4 ? 4 * q + j : 12 + 4 * q + j));
            }
#pragma unroll
            for (int k = 0; k < PS; ++k) yp[e][k] = __builtin_bit_cast(v8bf, part[k]);
          }
        }
        // the blocks of G that have positions of b as columns: 0, 1, 2, 4 or 3, 5
        v8bf gp[2][PS];
        auto g_at = [&](int tt) { return Lds::G + (tt < 2 ? tt : 2 * tt - 2 + b) * 1024; };
        frag(g_at(2 * b), Blk::GPART, gp[0]);
#pragma unroll
        for (int tt = 2 * b; tt < 4; ++tt) {
          if (tt < 3) frag(g_at(tt + 1), Blk::GPART, gp[(tt + 1) & 1]);
          if (!fast) {
            const int t = 16 * tt + l;
            const float lt = plh[t], rt = pll[t];
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int s = 32 * b + (j < 4 ? 4 * q + j : 12 + 4 * q + j);
              const float d = exp2_hw((lt - plh[s]) + (rt - pll[s]));
              float sum = (float)gp[tt & 1][PS - 1][j];
#pragma unroll
              for (int k = PS - 2; k >= 0; --k) sum += (float)gp[tt & 1][k][j];
              v[j] = s <= t ? sum * d : 0.f;
            }
            split(v, gp[tt & 1]);
          }
          mul(gp[tt & 1], yp, y[tt]);
        }
      }
    }
    if (Lds::TWICE) arrived();  // the next chunk's first stage, before the stores are on their way
    if (!OUT) continue;
    if (__ballot(bad[0] < kSsmQ || bad[1] < kSsmQ)) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        bad[e] = min(bad[e], __shfl_xor(bad[e], 16));
        bad[e] = min(bad[e], __shfl_xor(bad[e], 32));
#pragma unroll
        for (int m = 0; m < 4; ++m)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (16 * m + 4 * q + i >= bad[e]) y[m][e][i] = __builtin_nanf("");
      }
    }
    if (fast) {
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const v4f f = *reinterpret_cast<const v4f*>(pe + 16 * m + 4 * q);
#pragma unroll
        for (int e = 0; e < 2; ++e) y[m][e] *= f;
      }
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        y[m][0][i] = fmaf(skip, u[m][i][0], y[m][0][i]);
        y[m][1][i] = fmaf(skip, u[m][i][1], y[m][1][i]);
      }
    if (c.z) {
#pragma unroll
      for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[m][0][i] *= silu(z[m][i].lo());
          y[m][1][i] *= silu(z[m][i].hi());
        }
    }
    const unsigned to = here(yq), to2 = here(yq2);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const auto r = row_buffer<E>(c.y, r0 + 16 * m, c.y_stride, min(rows - 16 * m, 16), c.D);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        Two<E> out;
        out.set(y[m][0][i], y[m][1][i]);
        store_two<E, PAIR>(out, r, to + i * ys, to2 + i * ys);
      }
    }
  }
  if (!OUT) {
    const size_t sg = (size_t)segment * c.H + h;
    put_state(w.states + sg * per_head);
    if (live && lane == 0 && it % parts == 0) w.decay[sg] = (float)exp2(total);
  } else if (last && dst >= 0) {
    put_state(c.state + ((size_t)dst * c.H + h) * per_head);
  }
}

// The states before the segments of a cut sequence, in place of the segments'
// contributions: a thread per state of a head (grid: states, heads, sequences;
// one row of heads more moves the windows).
constexpr int kSsmJoin = 8;  // contributions on their way

__device__ __forceinline__ void ssm_join(const SsmCall& c, const SsmScratch& w) {
  const int seq = (int)blockIdx.z, h = (int)blockIdx.y;
  // the segments before this sequence's
  int base = 0;
  for (int i = (int)threadIdx.x & 63; i < seq; i += 64) {
    int a, b;
    ssm_rows(c, i, a, b);
    base = min(base + max(((b - a + kSsmQ - 1) / kSsmQ + w.per - 1) / w.per, 1), w.segments);
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) base += __shfl_xor(base, m);
  base = __builtin_amdgcn_readfirstlane(base);
  int t0, t1;
  ssm_rows(c, seq, t0, t1);
  const int segments = min(((t1 - t0 + kSsmQ - 1) / kSsmQ + w.per - 1) / w.per, w.segments - base);
  if (segments < 2) return;
  const int each = c.P * c.N, at = (int)blockIdx.x * 256 + (int)threadIdx.x;
  if (at >= each) return;
  const int src = ssm_slot(c.src, seq, c.slots);
  float s = src >= 0 ? c.state[((size_t)src * c.H + h) * each + at] : 0.f;
  const size_t step = (size_t)c.H * each;
  float* p = w.states + ((size_t)base * c.H + h) * each + at;
  const float* f = w.decay + (size_t)base * c.H + h;
  for (int k = 0; k < segments; k += kSsmJoin) {
    float v[kSsmJoin], d[kSsmJoin];
#pragma unroll
    for (int j = 0; j < kSsmJoin; ++j) {
      const bool in = k + j < segments - 1;
      v[j] = in ? p[(k + j) * step] : 0.f;
      d[j] = in ? f[(size_t)(k + j) * c.H] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kSsmJoin; ++j) {
      if (k + j >= segments) break;
      p[(k + j) * step] = s;
      s = fmaf(s, d[j], v[j]);
    }
  }
}
template <class E>  // one for each source that has this header
__global__ __launch_bounds__(256) void k_ssm_join(SsmCall c, SsmScratch w) {
  if ((int)blockIdx.y == c.H)
    ssm_window<E>(c, w, (int)blockIdx.z, (int)(blockIdx.x * 256 + threadIdx.x), (int)gridDim.x * 256);
  else
    ssm_join(c, w);
}

template <class E, int NT>
hipError_t ssm_prompt_nt(const SsmCall& c, const SsmScratch& w, hipStream_t st) {
  const int items = c.H / c.G * ((c.P + 31) / 32);
  const int nw = items < ssm_waves(c.N) ? items : ssm_waves(c.N);
  const dim3 grid(8 * (unsigned)(c.G * ((items + nw - 1) / nw)), ((unsigned)w.segments + 7) / 8);
  const int lds_out = SsmLds<NT, true>::bytes(nw), lds_sum = SsmLds<NT, false>::bytes(nw);
  auto out = w.pair ? k_ssm_chunks<E, NT, true, true> : k_ssm_chunks<E, NT, true, false>;
  auto sum = w.pair ? k_ssm_chunks<E, NT, false, true> : k_ssm_chunks<E, NT, false, false>;
  const int decays = (c.H + kSsmWaves * kSsmHeads - 1) / (kSsmWaves * kSsmHeads);
  hipLaunchKernelGGL((k_ssm_bc<E, NT>), dim3((unsigned)w.blocks, (unsigned)(c.G + decays + 1)), dim3(64 * kSsmWaves), 0, st,
                     c, w);
  hipError_t e = hipGetLastError();
  auto allow = [&](const void* f, int bytes) {
    if (e == hipSuccess) e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  };
  allow(reinterpret_cast<const void*>(out), lds_out);
  if (w.segments > c.n) allow(reinterpret_cast<const void*>(sum), lds_sum);
  if (e == hipSuccess && w.segments > c.n) {
    hipLaunchKernelGGL(sum, grid, dim3(64 * nw), lds_sum, st, c, w);
    hipLaunchKernelGGL(k_ssm_join<E>, dim3((unsigned)((c.P * c.N + 255) / 256), (unsigned)(c.H + 1), (unsigned)c.n),
                       dim3(256), 0, st, c, w);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(out, grid, dim3(64 * nw), lds_out, st, c, w);
  if (w.segments == c.n)  // (no join that moves them)
    hipLaunchKernelGGL(k_ssm_window<E>, dim3((unsigned)((c.C + 255) / 256), (unsigned)c.n), dim3(256), 0, st, c, w);
  return hipGetLastError();
}

template <class E>
hipError_t ssm_prompt(const SsmCall& c, const SsmScratch& w, hipStream_t st) {
  if (c.N <= 32) return ssm_prompt_nt<E, 1>(c, w, st);
  if (c.N <= 64) return ssm_prompt_nt<E, 2>(c, w, st);
  if (c.N <= 128) return ssm_prompt_nt<E, 4>(c, w, st);
  return ssm_prompt_nt<E, 8>(c, w, st);
}

}  // namespace lcsm
