// Prompts of linear attention in chunks on the matrix units; included by one
// source per element type.
//
// Unrolled over a chunk of C positions, with S the state before it, d the decay
// and rows counted from 0,
//
//   y_t = scale (d^(t+1) q_t S + sum_{j<=t} d^(t-j) (q_t k_j) v_j),
//   S'  = d^C S + sum_j k_j (d^(C-1-j) v_j)^T,
//
// four matrix products.  A workgroup has a state and up to 128 of its values, a
// wave 32 of them, whose part of the state it keeps in registers as the
// products' accumulators.  Queries, keys and values of a chunk are in LDS as
// they are in memory, rows of positions; what a product sums over positions is
// read from there transposed.  The accumulators of one product are an operand
// of the next as they stand: the order of a product's K slots is free as long as
// both operands have it, so that keys are taken in the order that makes S an
// operand of q S.  The scores, which all waves need, are made by all of them, a
// tile of 16 x 16 positions at a time, and handed on through LDS as operands:
// made transposed, a lane's accumulators are its share of them.  Outputs come out
// as four values of a position a lane.
//
// Chunks are counted from a sequence's end, so that the one that is not full is
// its first, and begins with rows of zeros that are nowhere in memory: what the
// factors depend on is then the same for all chunks.
//
// d^(t-j) is put into the scores and into the values as a factor of its own,
// never as a quotient: no decay overflows or vanishes before its time.
//
// What is not a bf16 value goes into the products as a sum of bf16 parts (which
// have fp32's range): queries, keys and values of fp16 are two, of fp32 three,
// exactly.  The scores and S are rounded to two parts (2^-16) where outputs are
// rounded to 16 bits after it, and to three for fp32; the decayed values are
// three parts always, since they are what the states are made of.  Of a product of
// parts those are made whose numbers add up to less than two (fp32, and what states
// are made of: three): of fp16, the product of both lower parts, 2^-16, is left out
// of q k, q S and the scores' products with values.  One q S of 128 keys is off by
// 2.4e-6 of its norm for bf16 and 3.7e-6 for fp16, where fp32 is by 2e-7; outputs of
// 16 bits are rounded by up to 2^-8 and 2^-11, a hundred times as much.
//
// Long calls are cut into segments of chunks: what each adds to the state after it, the
// states between them, then the outputs, three launches.  Bound by memory and by
// instructions, which do not quite hide under each other: 16384 rows of 32 states of
// 128 x 128, bf16, take 231 to 242 us, outputs 175 us (3.0 TB/s; the vector units are
// busy 40 % of it and the matrix units 26 %), contributions 74 us (3.6 TB/s), the join
// 14.  Two workgroups a compute unit fill its registers (of 128 keys, bf16 and fp32,
// outputs spill 16 to 24 a lane), so that a chunk's loads are started a chunk ahead,
// into the LDS of the keys before them, or of queries and values once these have been
// read.  Four stages of 32 rows in place of two of 64 for the contributions: 79 us
// against 74.  More than 128 keys take 432 to 472 registers and spill 20: one workgroup
// a unit, and 256 x 128 in bf16 518 to 550 us, fp16 1130, fp32 1040.
//
// A product with a value v_j that is not finite reaches positions before j as 0 *
// inf; where there is one, the products of the scores are made without it, and
// the outputs from j on set to NaN.
#pragma once

#include "lcsm_lin_internal.h"

namespace lcsm {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef bf16_t v8bf __attribute__((ext_vector_type(8)));
typedef bf16_t v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef short v4s __attribute__((ext_vector_type(4)));

template <class E>
struct LinParts {
  static constexpr int IN = 2;   // of queries, keys and values
  static constexpr int MID = 2;  // of scores and states
};
template <>
struct LinParts<bf16_t> {
  static constexpr int IN = 1, MID = 2;
};
template <>
struct LinParts<float> {
  static constexpr int IN = 3, MID = 3;
};

// Positions of a chunk: 64 where keys and values are one bf16 part and the chunk's
// rows leave room for two workgroups a compute unit, else 32 (fp16, 32 heads of 128
// x 128 and 16384 tokens: 449 us in chunks of 32, 705 us in those of 64; of 64 x 128,
// 311 and 317 us; later steps brought the first to 427).
template <class E>
constexpr int lin_chunk(int KT) {
  return LinParts<E>::IN == 1 && KT <= 4 ? 64 : 32;
}

// c[e] += a b[e] (or a[e] b), both in parts: those products whose parts' numbers add
// up to at most LAST, the small ones first.  The two sums take turns: a product
// that waits for the one before it takes twice as long.
template <int LAST, int P, int Q>
__device__ __forceinline__ void lin_mul(const v8bf (&a)[P], const v8bf (&b)[2][Q], v4f (&c)[2]) {
#pragma unroll
  for (int sum = LAST; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (sum - i >= 0 && sum - i < Q) {
#pragma unroll
        for (int e = 0; e < 2; ++e) c[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i], b[e][sum - i], c[e], 0, 0, 0);
      }
}
template <int LAST, int P, int Q>
__device__ __forceinline__ void lin_mul(const v8bf (&a)[2][P], const v8bf (&b)[Q], v4f (&c)[2]) {
#pragma unroll
  for (int sum = LAST; sum >= 0; --sum)
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (sum - i >= 0 && sum - i < Q) {
#pragma unroll
        for (int e = 0; e < 2; ++e) c[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[e][i], b[sum - i], c[e], 0, 0, 0);
      }
}

// Values as parts: each the bf16 nearest to what the parts before it leave.
template <int P, int N>
__device__ __forceinline__ void lin_parts(float (&v)[N], unsigned (&to)[P][N / 2]) {
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
      // (one conversion of two: as two conversions they are three instructions)
      const v2bf two = __builtin_convertvector((v2f){v[2 * k], v[2 * k + 1]}, v2bf);
      to[p][k] = __builtin_bit_cast(unsigned, two);
      if (p + 1 < P) {
        v[2 * k] -= __builtin_bit_cast(float, to[p][k] << 16);
        v[2 * k + 1] -= __builtin_bit_cast(float, to[p][k] & 0xffff0000u);
      }
    }
}
// Eight values as an operand's.
template <int P>
__device__ __forceinline__ void lin_split(float (&v)[8], v8bf (&to)[P]) {
  unsigned w[P][4];
  lin_parts(v, w);
#pragma unroll
  for (int p = 0; p < P; ++p) to[p] = __builtin_bit_cast(v8bf, (v4u){w[p][0], w[p][1], w[p][2], w[p][3]});
}

// Rows of bf16 in LDS, `chunks` (a power of two) of eight values a row, placed so
// that eight rows' chunks of one column lie in different banks.
__device__ __forceinline__ int lin_at(int row, int chunk, int chunks) {
  const int turn = chunks >= 8 ? row & 7 : chunks == 4 ? row >> 1 & 3 : 0;
  return (row * chunks + (chunk ^ turn)) * 16;
}
// Where rows that are the same modulo 8 have the chunks 4 m + low: two places of
// a lane and what is the same for all lanes.
struct LinPlace {
  int at[2];
  __device__ LinPlace(int row, int low, int chunks) {
    at[0] = lin_at(row, low, chunks);
    at[1] = chunks >= 8 ? at[0] ^ 64 : at[0];
  }
  __device__ int operator()(int rows, int m, int chunks) const { return at[m & 1] + rows * chunks * 16 + (m >> 1) * 128; }
};
__device__ __forceinline__ v8bf lin_read(const char* lds, int at) { return *reinterpret_cast<const v8bf*>(lds + at); }
// Each of 16 lanes names four values of one of four rows (of row lane / 4); it
// gets the four rows' values of column lane % 16 of the sixteen that they name.
__device__ __forceinline__ v4s lin_read_turned(const char* lds, int at) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(lds + at));
}
__device__ __forceinline__ v8bf lin_join(v4s a, v4s b) {
  struct {
    v4s a, b;
  } two = {a, b};
  return __builtin_bit_cast(v8bf, two);
}

constexpr unsigned kLinNowhere = 0xC0000000u;  // past every buffer here

// v, with what is made of it made here: sums of it and of what is the same in
// every turn of a loop are not kept in registers from one turn to the next.
__device__ __forceinline__ unsigned lin_here(unsigned v) {
  asm volatile("" : "+v"(v));
  return v;
}

// The piece [*k0, *k1) of `per` chunks (and its sequence, its number in it and
// the sequence's chunks) that has number `want` when the pieces of all sequences
// are counted one after another, every sequence having at least one; false past
// the last one.  All lanes of a wave together.
template <int C>
__device__ __forceinline__ bool lin_piece(const LinCall& c, int want, int per, int& seq, int& num, int& chunks) {
  const int lane = (int)threadIdx.x & 63;
  int base = 0;
  for (int i0 = 0; i0 < c.n; i0 += 64) {
    int mine = 0, ch = 0;
    if (i0 + lane < c.n) {
      int t0, t1;
      lin_rows(c, i0 + lane, t0, t1);
      ch = (t1 - t0 + C - 1) / C;
      mine = max((ch + per - 1) / per, 1);
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
      seq = i0 + who;
      num = want - base - __shfl(sum - mine, who);
      chunks = __shfl(ch, who);
      return true;
    }
    base += total;  // (offsets that do not rise: at most 64 T / C and `want` at a time)
  }
  return false;
}

// What a thread loads of a chunk's rows, eight elements at a time: all loads are on
// their way before the first is used.
template <class E, int C, int CHUNKS>
struct LinRaw {
  static constexpr int P = LinParts<E>::IN, THREADS = 64 * kLinWaves, N = (C * CHUNKS + THREADS - 1) / THREADS;
  struct Eight {
    E e[8];
  } v[N];
  // Rows of `from` after `pad` rows of zeros, `width` values of each; wide accesses
  // of global memory may begin at any element.
  __device__ __forceinline__ void load(const E* from, size_t stride, int pad, int width) {
    struct __attribute__((packed, aligned(sizeof(E)))) Pack {
      E e[8];
    };
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int at = n * THREADS + (int)threadIdx.x, row = at / CHUNKS, chunk = at % CHUNKS;
      const int have = row >= pad && row < C ? width - 8 * chunk : 0;
      const E* p = from + (size_t)max(row - pad, 0) * stride + 8 * chunk;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[n].e[i] = (E)0.f;
      if (have >= 8) {
        const Pack k = *reinterpret_cast<const Pack*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[n].e[i] = k.e[i];
      } else if (have > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i < have) v[n].e[i] = p[i];
      }
    }
  }
  // As parts into LDS.
  __device__ __forceinline__ void put(char* lds) const {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int at = n * THREADS + (int)threadIdx.x, row = at / CHUNKS, chunk = at % CHUNKS;
      if (at >= C * CHUNKS) break;
      v8bf w[P];
      if constexpr (P == 1) {
        w[0] = __builtin_bit_cast(v8bf, v[n]);
      } else {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)v[n].e[i];
        lin_split(f, w);
      }
#pragma unroll
      for (int p = 0; p < P; ++p) *reinterpret_cast<v8bf*>(lds + p * C * CHUNKS * 16 + lin_at(row, chunk, CHUNKS)) = w[p];
    }
  }
};

// What a lane fetches of a chunk's rows: 16 bytes of every STEP'th row.
template <int CHUNKS>
struct LinLane {
  static constexpr int STEP = 64 * kLinWaves / CHUNKS;
  static_assert(STEP % 8 == 0, "a lane has one chunk of all its rows");
  unsigned at;  // of the first row
  bool have;
  __device__ LinLane(size_t stride, int width) {
    const int row = (int)threadIdx.x / CHUNKS, chunk = lin_at(row, (int)threadIdx.x % CHUNKS, CHUNKS) / 16 - row * CHUNKS;
    at = (unsigned)row * (unsigned)stride * 2u + 16u * (unsigned)chunk;
    have = 8 * chunk < width;
  }
};

// A chunk's rows straight from memory into LDS (bf16 rows of whole and aligned
// eights): `pad` rows of zeros, then those of `from`, `width` values of each and
// zeros past them.  The caller waits for them.
template <class E, int C, int CHUNKS>
__device__ __forceinline__ void lin_fetch(char* lds, const LinLane<CHUNKS>& lane, const E* from, size_t stride, int pad, int width) {
  constexpr int THREADS = 64 * kLinWaves, STEP = LinLane<CHUNKS>::STEP;
  const auto r = row_buffer<E>(from, 0, stride, C - pad, width);
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  // (rows before the first wrap around to past the buffer's end)
  const unsigned each = (unsigned)stride * 2u;
#pragma unroll
  for (int i = 0; i < C / STEP; ++i)
    fetch_to_lds(r, lane.have ? lane.at + (unsigned)(i * STEP - pad) * each : kLinNowhere, 0, lds + (i * THREADS + 64 * wv) * 16);
}

// Outputs of a row that begins at `row` of a buffer: `width` values, of which a lane
// has four from column `at` on and four 16 behind those.  wide: so many are whole and
// aligned as one (8 of 16 bits, 4 or 1).
template <class E>
__device__ __forceinline__ void lin_store(__amdgpu_buffer_rsrc_t r, unsigned row, int at, int width, const v4f (&v)[2], int wide) {
  typedef E v4e __attribute__((ext_vector_type(4)));
  const v4e out[2] = {__builtin_convertvector(v[0], v4e), __builtin_convertvector(v[1], v4e)};
  typedef unsigned v2u __attribute__((ext_vector_type(2)));
  if (wide == 8) {
    if constexpr (sizeof(E) == 2) {
      // lanes 16 apart exchange halves, so that each has eight values: 64 bytes of a row
      // a store in place of 32
      const v2u a = __builtin_bit_cast(v2u, out[0]), b = __builtin_bit_cast(v2u, out[1]);
      const auto lo = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
      const auto hi = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
      const int odd = (int)threadIdx.x >> 4 & 1, first = at + 12 * odd;
      __builtin_amdgcn_raw_buffer_store_b128(v4u{lo[0], hi[0], lo[1], hi[1]}, r,
                                             (int)(first < width ? row + (unsigned)first * 2u : kLinNowhere), 0, 0);
    }
  } else if (wide == 4) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const unsigned to = at + 16 * e < width ? row + (unsigned)(at + 16 * e) * (unsigned)sizeof(E) : kLinNowhere;
      if constexpr (sizeof(E) == 4)
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, out[e]), r, (int)to, 0, 0);
      else
        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(v2u, out[e]), r, (int)to, 0, 0);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = at + 16 * e + i;
        const unsigned to = n < width ? row + (unsigned)n * (unsigned)sizeof(E) : kLinNowhere;
        if constexpr (sizeof(E) == 4)
          __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, (float)out[e][i]), r, (int)to, 0, 0);
        else
          __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (E)out[e][i]), r, (int)to, 0, 0);
      }
  }
}

// What a workgroup has in LDS: keys (DIRECT: this chunk's and the next one's),
// values (the same where there are no outputs), queries, and the scores of the
// tiles of 16 x 32 positions that are not above the diagonal.
template <class E, int KT, bool OUT, bool DIRECT>
struct LinLds {
  static constexpr int C = lin_chunk<E>(KT), IN = LinParts<E>::IN;
  static constexpr int KEYS = IN * C * KT * 64, VALUES = IN * C * kLinWaves * 64;
  static constexpr int V = (DIRECT ? 2 : 1) * KEYS, Q = V + (DIRECT && !OUT ? 2 : 1) * VALUES;
  static constexpr int FRAGS = C == 64 ? 6 : 2, P = Q + (OUT ? KEYS : 0);
  static constexpr int BYTES = P + (OUT ? LinParts<E>::MID * FRAGS * 1024 : 0);
};

// One segment (w.per chunks) of a sequence: OUT, with its outputs and from the
// state before it; else its own contribution to the state after it.
template <class E, int KT, bool OUT, bool DIRECT>
__global__ __launch_bounds__(64 * kLinWaves, KT > 4 ? 1 : 2) void k_lin_chunks(LinCall c, LinCut w) {
  constexpr int C = lin_chunk<E>(KT), TT = C / 16, PB = C / 32;  // tiles and blocks of positions
  constexpr int IN = LinParts<E>::IN, MID = LinParts<E>::MID;
  constexpr int KC = 4 * KT, VC = 4 * kLinWaves;  // chunks of eight a row
  constexpr int KPART = C * KC * 16, VPART = C * VC * 16;
  typedef LinLds<E, KT, OUT, DIRECT> Lds;
  extern __shared__ __align__(16) char lds[];
  char *const lv = lds + Lds::V, *const lq = lds + Lds::Q, *const lp = lds + Lds::P;
  const int lane = (int)threadIdx.x & 63, q = lane >> 4, l = lane & 15;
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int vblocks = (c.V + 32 * kLinWaves - 1) / (32 * kLinWaves);
  const int g = (int)blockIdx.x / vblocks, v0 = (int)blockIdx.x % vblocks * 32 * kLinWaves;
  const int segment = (int)blockIdx.y, heads = c.H / c.G;
  int seq, num, chunks;
  if (!lin_piece<C>(c, segment, w.per, seq, num, chunks)) return;
  // (the same for all lanes, which the compiler does not see past that loop: all that
  // follows from these would be vector work)
  seq = __builtin_amdgcn_readfirstlane(seq);
  num = __builtin_amdgcn_readfirstlane(num);
  chunks = __builtin_amdgcn_readfirstlane(chunks);
  // (at most 2^26 / 32 chunks and as many again)
  const int k0 = num * w.per;
  const bool last = k0 + w.per >= chunks;
  if (!OUT && last) return;
  int t0, t1;
  lin_rows(c, seq, t0, t1);
  t0 = __builtin_amdgcn_readfirstlane(t0);
  t1 = __builtin_amdgcn_readfirstlane(t1);
  const int src = __builtin_amdgcn_readfirstlane(lin_slot(c.src, seq, c.slots));
  const int dst = __builtin_amdgcn_readfirstlane(lin_slot(c.dst, seq, c.slots));
  const int k1 = min(k0 + w.per, chunks);
  const double decay = (double)c.decay[g];
  float g2 = (float)(decay * 1.4426950408889634);
  if (g2 < -1e30f) g2 = -1e30f;  // (d = 0: finite, so that d^0 is 1; NaN stays)
  // d^n, 1 for n <= 0
  auto power = [&](int n) { return exp2_hw(g2 * (float)max(n, 0)); };
  // the same of distances 16 m + n as d^(16 m) d^n: m is the same for all lanes
  float tile[TT], near[4], far[4], back[4];
#pragma unroll
  for (int m = 0; m < TT; ++m) tile[m] = power(16 * m);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    near[i] = c.scale * power(l - 4 * q - i);      // in a tile (where it is not negative)
    far[i] = c.scale * power(16 + l - 4 * q - i);  // from the tile before
    back[i] = power(15 - 4 * q - i);               // to the end of the tile
  }

  // the state: S[a][e][i] is key 32 (a / 2) + 8 q + 4 (a % 2) + i, value vc + 16 e + l
  v4f S[2 * KT][2];
  const int vc = v0 + 32 * wv;  // this wave's first value
  const size_t each = (size_t)c.K * c.V;
  // a state as a buffer: keys past the last one are past its end
  unsigned column[2];
#pragma unroll
  for (int e = 0; e < 2; ++e)
    column[e] = vc + 16 * e + l < c.V ? (unsigned)(8 * q * c.V + vc + 16 * e + l) * 4u : kLinNowhere;
  auto state_at = [&](unsigned from, int a, int i) { return from + (unsigned)((a / 2 * 32 + a % 2 * 4 + i) * c.V) * 4u; };
  const float* from = nullptr;
  if (OUT && chunks > w.per)
    from = w.states + ((size_t)segment * c.G + g) * each;
  else if (OUT && src >= 0)
    from = c.state + ((size_t)src * c.G + g) * each;
  const auto before = uniform_buffer(from, from ? (unsigned)(each * 4) : 0u);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const unsigned at = lin_here(column[e]);
#pragma unroll
    for (int a = 0; a < 2 * KT; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        S[a][e][i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(before, state_at(at, a, i), 0, 0));
  }

  // keys and queries as they are, rows 16 n + l, eights 4 m + q; keys turned, rows
  // 16 n + 4 q ..+3, eights 4 m + 0 ..+3; values turned, eights 4 wv + 2 e + 0 ..+1
  const LinPlace plain(l, q, KC), turned(4 * q + l / 4, l % 4, KC);
  const int value_at[2] = {lin_at(4 * q + l / 4, 4 * wv + l % 4 / 2, VC) + l % 2 * 8,
                           lin_at(4 * q + l / 4, 4 * wv + 2 + l % 4 / 2, VC) + l % 2 * 8};

  LinDecay whole(decay * C);
  const unsigned out_row = (unsigned)c.y_stride * (unsigned)sizeof(E);
  const LinLane<KC> keys_lane(c.k_stride, c.K), queries_lane(c.q_stride, c.K);
  const LinLane<VC> values_lane(c.v_stride, c.V - v0);
  // rows of chunk k, counted from the sequence's end
  int r0 = 0, pad = 0;
  auto locate = [&](int k) {
    const int end = t1 - (chunks - 1 - k) * C;
    r0 = max(end - C, t0);
    pad = C - (end - r0);
  };
  auto keys_of = [&]() { return static_cast<const E*>(c.k) + (size_t)r0 * c.k_stride + (size_t)g * c.K; };
  auto values_of = [&]() { return static_cast<const E*>(c.v) + (size_t)r0 * c.v_stride + (size_t)g * c.V + v0; };
  auto queries_of = [&](int h) { return static_cast<const E*>(c.q) + (size_t)r0 * c.q_stride + ((size_t)g * heads + h) * c.K; };
  auto fetch_keys = [&](int k) {
    locate(k);
    if constexpr (DIRECT) lin_fetch<E, C, KC>(lds + k % 2 * Lds::KEYS, keys_lane, keys_of(), c.k_stride, pad, c.K);
  };
  auto fetch_values = [&](int k) {
    locate(k);
    if constexpr (DIRECT) lin_fetch<E, C, VC>(lv + (OUT ? 0 : k % 2 * Lds::VALUES), values_lane, values_of(), c.v_stride, pad, c.V - v0);
  };
  auto fetch_queries = [&](int k, int h) {
    locate(k);
    if constexpr (DIRECT) lin_fetch<E, C, KC>(lq, queries_lane, queries_of(h), c.q_stride, pad, c.K);
  };
  // (the compiler does not wait for transfers straight into LDS)
  auto arrived = [&]() {
    if (DIRECT) wait_memory_but<0>();
    barrier_for_lds();
  };
  if (OUT) {  // halves of scores above the diagonal stay zero
    for (int i = (int)threadIdx.x; i < MID * Lds::FRAGS * 64; i += 64 * kLinWaves)
      reinterpret_cast<v4u*>(lp)[i] = v4u{0, 0, 0, 0};
  }
  // a segment's own contribution is summed from its end, so that what was read last is
  // what the outputs' kernel reads first, and as one product, not decayed by the chunk
  constexpr int AHEAD = OUT ? 1 : -1;
  const int first = OUT ? k0 : k1 - 1, end = OUT ? k1 : k0 - 1;
  if (DIRECT && k0 < k1) {
    fetch_keys(first);
    fetch_values(first);
    if (OUT) fetch_queries(first, 0);
  }
  for (int k = first; k != end; k += AHEAD) {
    const char* lk = lds + (DIRECT ? k % 2 * Lds::KEYS : 0);
    const char* values = lv + (DIRECT && !OUT ? k % 2 * Lds::VALUES : 0);
    if constexpr (!DIRECT) {
      locate(k);
      LinRaw<E, C, KC> rk, rq;
      LinRaw<E, C, VC> rv;
      rk.load(keys_of(), c.k_stride, pad, c.K);
      rv.load(values_of(), c.v_stride, pad, c.V - v0);
      if (OUT) rq.load(queries_of(0), c.q_stride, pad, c.K);
      barrier_for_lds();  // the chunk before has been read
      rk.put(lds);
      rv.put(lv);
      if (OUT) rq.put(lq);
    }
    arrived();
    // DIRECT: the next chunk's keys (and values) go where those before these were,
    // which all waves have passed
    if (DIRECT && k + AHEAD != end) {
      fetch_keys(k + AHEAD);
      if (!OUT) fetch_values(k + AHEAD);
    }
    locate(k);
    // values as an operand: 32 positions a block, slots 4 q ..+3 and 16 + 4 q ..+3
    v8bf vf[PB][2][IN];
#pragma unroll
    for (int b = 0; b < PB; ++b)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int p = 0; p < IN; ++p) {
          const int at = value_at[e] + p * VPART + 32 * b * VC * 16;
          vf[b][e][p] = lin_join(lin_read_turned(values, at), lin_read_turned(values, at + 16 * VC * 16));
        }
    if constexpr (OUT) {
      // a value that is not finite: the first such position of this lane's value is `bad`
      typedef unsigned short v2h __attribute__((ext_vector_type(2)));
      v2h most = {0, 0};
#pragma unroll
      for (int b = 0; b < PB; ++b)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const v4u w0 = __builtin_bit_cast(v4u, vf[b][e][0]);
#pragma unroll
          for (int j = 0; j < 4; ++j) most = __builtin_elementwise_max(most, __builtin_bit_cast(v2h, w0[j] & 0x7fff7fffu));
        }
      const bool any = __ballot(most[0] >= 0x7f80 || most[1] >= 0x7f80) != 0;
      for (int h = 0; h < heads; ++h) {
        if (h > 0) {
          if constexpr (!DIRECT) {
            LinRaw<E, C, KC> rq;
            rq.load(queries_of(h), c.q_stride, pad, c.K);
            barrier_for_lds();
            rq.put(lq);
          }
          arrived();
        }
        // scores, transposed: positions 16 jt + 4 q + i of the keys for 16 tt + l
#pragma unroll 1
        for (int n = wv; n < TT * (TT + 1) / 2; n += kLinWaves) {
          const int tt = n < 1 ? 0 : n < 3 ? 1 : n < 6 ? 2 : 3, jt = n - tt * (tt + 1) / 2, apart = tt - jt;
          v4f two[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
          for (int kb = 0; kb < KT; ++kb) {
            v8bf qf[IN], kf[IN];
#pragma unroll
            for (int p = 0; p < IN; ++p) {
              qf[p] = lin_read(lq, p * KPART + plain(16 * tt, kb, KC));
              kf[p] = lin_read(lk, p * KPART + plain(16 * jt, kb, KC));
            }
            int turn = kb;
#pragma unroll
            for (int sum = MID - 1; sum >= 0; --sum)
#pragma unroll
              for (int i = 0; i < IN; ++i)
                if (sum - i >= 0 && sum - i < IN) {
                  two[turn & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i], qf[sum - i], two[turn & 1], 0, 0, 0);
                  ++turn;
                }
          }
          const v4f s = two[0] + two[1];
          const float between = apart < 2 ? 1.f : apart == 2 ? tile[1] : tile[TT - 2];
          float v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i)
            v[i] = apart ? s[i] * far[i] * between : l >= 4 * q + i ? s[i] * near[i] : 0.f;
          unsigned parts[MID][2];
          lin_parts(v, parts);
          typedef unsigned v2u __attribute__((ext_vector_type(2)));
          const int at = (tt < 2 ? tt : 2 * tt - 2 + jt / 2) * 1024 + lane * 16 + jt % 2 * 8;
#pragma unroll
          for (int p = 0; p < MID; ++p)
            *reinterpret_cast<v2u*>(lp + p * Lds::FRAGS * 1024 + at) = v2u{parts[p][0], parts[p][1]};
        }
        // y[tt][e]: values 16 e + 4 q + i of position 16 tt + l
        v4f y[TT][2];
#pragma unroll
        for (int tt = 0; tt < TT; ++tt)
#pragma unroll
          for (int e = 0; e < 2; ++e) y[tt][e] = v4f{0.f, 0.f, 0.f, 0.f};
        // (fragments are read from LDS one ahead of their products, the state's parts made
        // meanwhile)
        v8bf qf[2][IN], sp[2][MID];
        auto read_queries = [&](int f) {
#pragma unroll
          for (int p = 0; p < IN; ++p) qf[f % 2][p] = lin_read(lq, p * KPART + plain(f % TT * 16, f / TT, KC));
        };
        read_queries(0);
#pragma unroll
        for (int f = 0; f < KT * TT; ++f) {
          const int kb = f / TT, tt = f % TT;
          if (f + 1 < KT * TT) read_queries(f + 1);
          if (tt == 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float v[8];
              // (the parts of all states, made before the loop over the heads, would take
              // more registers than there are)
              asm volatile("" : "+v"(S[2 * kb][e]), "+v"(S[2 * kb + 1][e]));
#pragma unroll
              for (int i = 0; i < 4; ++i) v[i] = S[2 * kb][e][i], v[4 + i] = S[2 * kb + 1][e][i];
              lin_split(v, sp[e]);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
          lin_mul<MID - 1>(sp, qf[f % 2], y[tt]);
        }
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) {
          const float f = c.scale * power((int)lin_here((unsigned)(16 * tt + l + 1 - pad)));
#pragma unroll
          for (int e = 0; e < 2; ++e) y[tt][e] *= f;
        }
        barrier_for_lds();  // the scores are there; queries and values have been read
        if (DIRECT) {
          if (h + 1 < heads)
            fetch_queries(k, h + 1);
          else if (k + 1 < k1)
            fetch_queries(k + 1, 0);
          if (h == 0 && k + 1 < k1) fetch_values(k + 1);
          locate(k);
        }
        auto scores_times = [&](const v8bf (&x)[2][IN], int b) {
#pragma unroll
          for (int tt = 2 * b; tt < TT; ++tt) {
            __builtin_amdgcn_sched_barrier(0);
            v8bf pf[MID];
#pragma unroll
            for (int p = 0; p < MID; ++p)
              pf[p] = *reinterpret_cast<const v8bf*>(lp + (p * Lds::FRAGS + (tt < 2 ? tt : 2 * tt - 2 + b)) * 1024 + lane * 16);
            lin_mul<MID - 1>(x, pf, y[tt]);
          }
        };
        if (!any) {
#pragma unroll
          for (int b = 0; b < PB; ++b) scores_times(vf[b], b);
        } else {
          // without the values that are not finite, and from the first of them on NaN
          unsigned bad[2] = {0, 0};  // slots 8 b + 0 ..+7 that have such a value
#pragma unroll
          for (int b = 0; b < PB; ++b) {
            v8bf fine[2][IN];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              v4u part[IN];
#pragma unroll
              for (int p = 0; p < IN; ++p) {
                part[p] = __builtin_bit_cast(v4u, vf[b][e][p]);
                asm volatile("" : "+v"(part[p]));  // (made here, not before the loop over the heads)
              }
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                // of each half one where it is finite, and so the half's mask
                const v2h one = __builtin_elementwise_min(__builtin_bit_cast(v2h, (part[0][j] & 0x7f807f80u) ^ 0x7f807f80u), (v2h){1, 1});
                const unsigned mask = __builtin_bit_cast(unsigned, (v2h){0, 0} - one), none = ~mask;
                bad[e] |= ((none & 1) | (none >> 30 & 2)) << (8 * b + 2 * j);
#pragma unroll
                for (int p = 0; p < IN; ++p) part[p][j] &= mask;
              }
#pragma unroll
              for (int p = 0; p < IN; ++p) fine[e][p] = __builtin_bit_cast(v8bf, part[p]);
            }
            scores_times(fine, b);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int slot = __ffs(bad[e]) - 1;
            int at = slot < 0 ? C : slot / 8 * 32 + 4 * q + slot % 8 + (slot % 8 < 4 ? 0 : 12);
            at = min(at, __shfl_xor(at, 16));
            at = min(at, __shfl_xor(at, 32));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int first = __shfl(at, 4 * q + i);
#pragma unroll
              for (int tt = 0; tt < TT; ++tt)
                if (16 * tt + l >= first) y[tt][e][i] = __builtin_nanf("");
            }
          }
        }
        const auto r = row_buffer<E>(static_cast<E*>(c.y) + ((size_t)g * heads + h) * c.V, (size_t)r0, c.y_stride, C - pad, c.V);
        const unsigned to = lin_here((unsigned)(l - pad) * out_row);
        const int column = (int)lin_here((unsigned)(vc + 4 * q));
#pragma unroll
        for (int tt = 0; tt < TT; ++tt) lin_store<E>(r, to + 16 * tt * out_row, column, c.V, y[tt], w.wide);
      }
    }
    if (OUT && k + 1 == k1 && !(last && dst >= 0)) break;  // nothing asks for the state after it
    // the state after the chunk, or what the chunk adds to that after the segment
    float later = 1.f;  // from the chunk's end to the segment's
    if constexpr (OUT) {
      const LinDecay d = pad == 0 ? whole : LinDecay(decay * (C - pad));
      if (d.keep != 0.f) {
#pragma unroll
        for (int a = 0; a < 2 * KT; ++a)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) S[a][e][i] = fmaf(S[a][e][i], d.by, S[a][e][i]);
      } else {
#pragma unroll
        for (int a = 0; a < 2 * KT; ++a)
#pragma unroll
          for (int e = 0; e < 2; ++e) S[a][e] *= d.by;
      }
    } else if (k + 1 < k1) {
      later = (float)exp(decay * ((k1 - 1 - k) * C));
    }
    v8bf kf[2][IN], xf[2][3];
    auto read_keys = [&](int f) {
#pragma unroll
      for (int p = 0; p < IN; ++p) {
        const int a = f % (2 * KT), at = p * KPART + turned(f / (2 * KT) * 32, a / 2, KC) + a % 2 * 8;
        kf[f % 2][p] = lin_join(lin_read_turned(lk, at), lin_read_turned(lk, at + 16 * KC * 16));
      }
    };
    read_keys(0);
#pragma unroll
    for (int f = 0; f < PB * 2 * KT; ++f) {
      const int b = f / (2 * KT), a = f % (2 * KT);
      if (f + 1 < PB * 2 * KT) read_keys(f + 1);
      if (a == 0) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float x = (float)vf[b][e][IN - 1][j];
#pragma unroll
            for (int p = IN - 2; p >= 0; --p) x += (float)vf[b][e][p][j];
            const float far_back = tile[TT - 1 - 2 * b - j / 4];
            v[j] = OUT ? x * back[j % 4] * far_back : x * (back[j % 4] * (far_back * later));
          }
          lin_split(v, xf[e]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      lin_mul<2>(kf[f % 2], xf, S[a]);
    }
  }
  float* to = nullptr;
  if (!OUT)
    to = w.states + ((size_t)segment * c.G + g) * each;
  else if (last && dst >= 0)
    to = c.state + ((size_t)dst * c.G + g) * each;
  if (!to) return;
  const auto after = uniform_buffer(to, (unsigned)(each * 4));
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const unsigned at = lin_here(column[e]);
#pragma unroll
    for (int a = 0; a < 2 * KT; ++a)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float v = S[a][e][i];  // (a bit cast of the element itself takes the first one)
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, v), after, (int)state_at(at, a, i), 0, 0);
      }
  }
}

// The states before the segments of a cut sequence, in place of the segments'
// contributions: a thread a value of a state (grid: values, states, sequences).
constexpr int kLinJoin = 8;  // contributions on their way

template <class E, int KT>
__global__ __launch_bounds__(256) void k_lin_join(LinCall c, LinCut w) {
  constexpr int C = lin_chunk<E>(KT);
  const int seq = (int)blockIdx.z, g = (int)blockIdx.y;
  // the segments before this sequence's
  int base = 0;
  for (int i = (int)threadIdx.x & 63; i < seq; i += 64) {
    int a, b;
    lin_rows(c, i, a, b);
    base = min(base + max(((b - a + C - 1) / C + w.per - 1) / w.per, 1), w.segments);
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) base = min(base + __shfl_xor(base, m), w.segments);
  int t0, t1;
  lin_rows(c, seq, t0, t1);
  const int segments = min(((t1 - t0 + C - 1) / C + w.per - 1) / w.per, w.segments - base);
  if (segments < 2) return;
  const size_t each = (size_t)c.K * c.V, at = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= each) return;
  const int src = lin_slot(c.src, seq, c.slots);
  float s = src >= 0 ? c.state[((size_t)src * c.G + g) * each + at] : 0.f;
  // (the first segment's first chunk may not be full)
  const double decay = (double)c.decay[g], whole = (double)C * w.per;
  const LinDecay first(decay * (whole - ((t1 - t0 + C - 1) / C * C - (t1 - t0)))), d(decay * whole);
  const size_t step = (size_t)c.G * each;
  float* p = w.states + ((size_t)base * c.G + g) * each + at;
  for (int k = 0; k < segments; k += kLinJoin) {
    float v[kLinJoin];
#pragma unroll
    for (int j = 0; j < kLinJoin; ++j) v[j] = k + j < segments - 1 ? p[(k + j) * step] : 0.f;
#pragma unroll
    for (int j = 0; j < kLinJoin; ++j) {
      if (k + j >= segments) break;
      p[(k + j) * step] = s;
      s = (k + j == 0 ? first(s) : d(s)) + v[j];
    }
  }
}

template <class E, int KT>
hipError_t lin_prompt_kt(const LinCall& c, const LinCut& w, hipStream_t st) {
  constexpr bool CAN = LinParts<E>::IN == 1;
  const bool direct = CAN && w.direct;
  const int lds_out = direct ? LinLds<E, KT, true, CAN>::BYTES : LinLds<E, KT, true, false>::BYTES;
  const int lds_sum = direct ? LinLds<E, KT, false, CAN>::BYTES : LinLds<E, KT, false, false>::BYTES;
  const unsigned vblocks = (unsigned)((c.V + 32 * kLinWaves - 1) / (32 * kLinWaves));
  const dim3 grid((unsigned)c.G * vblocks, (unsigned)w.segments), threads(64 * kLinWaves);
  auto out = direct ? k_lin_chunks<E, KT, true, CAN> : k_lin_chunks<E, KT, true, false>;
  auto sum = direct ? k_lin_chunks<E, KT, false, CAN> : k_lin_chunks<E, KT, false, false>;
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(out), hipFuncAttributeMaxDynamicSharedMemorySize, lds_out);
  if (e == hipSuccess && w.segments > c.n) {
    e = hipFuncSetAttribute(reinterpret_cast<const void*>(sum), hipFuncAttributeMaxDynamicSharedMemorySize, lds_sum);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(sum, grid, threads, lds_sum, st, c, w);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_lin_join<E, KT>), dim3((unsigned)(((size_t)c.K * c.V + 255) / 256), (unsigned)c.G, (unsigned)c.n),
                       dim3(256), 0, st, c, w);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(out, grid, threads, lds_out, st, c, w);
  return hipGetLastError();
}

template <class E>
hipError_t lin_prompt(const LinCall& c, const LinCut& w, hipStream_t st) {
  switch (lin_blocks_of(c.K)) {
    case 1: return lin_prompt_kt<E, 1>(c, w, st);
    case 2: return lin_prompt_kt<E, 2>(c, w, st);
    case 4: return lin_prompt_kt<E, 4>(c, w, st);
    default: return lin_prompt_kt<E, 8>(c, w, st);
  }
}

}  // namespace lcsm
