// Products with 8-bit weights and rows quantized to 8 bits (lcsm_q8.h).
//
// Codes of weights and of rows are kept as tiles of 16 rows x 64 inputs, 16
// bytes a lane: lane l has inputs 16 (l / 16) ..+15 of row l % 16, which is its
// share of either operand of a 16x16x64 integer product.  A call quantizes its
// rows into such tiles first, in a launch of its own, or with few rows in the
// product's.  A codes' sum is exact in 32 bits, so that it may be taken in any
// order; what is rounded is its float, twice times a scale, the bias and the output.
//
// Few rows are bound by the weights' bytes and by launches, many by the matrix
// units: 16384 rows of 2048 inputs to 8192 outputs, bf16, take 278 us, some 28 of
// them for the rows' codes (241 us at the rate that a large library product of 8-bit
// integers reaches, 509 us at that of 16-bit floats); a row of 2048 to 8192 outputs
// takes 4.7 us, 3.7 us of it to read the weights at the rate of a large copy.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>

#include "lcsm_elem.h"
#include "lcsm_q8.h"

namespace lcsm {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

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
  int wide;  // 16 bytes of outputs are aligned as one, 16 rows of them reach less than 2^32 bytes
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
  // Four codes a word.  x inv is within 2^-17 of x / s, so that its nearest integer
  // is the code where it is not that close to a border; where one value of a wave
  // is, all are made as above (a quarter of the instructions without).
  template <int N>
  __device__ void words(const float (&x)[N], int (&to)[N / 4]) const {
    constexpr float M = 12582912.f;  // 1.5 2^23: an integer added to it is in its low bits
    float b[N], worst = f == 1.f && inv > 0.f ? 0.f : 1.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      b[i] = fmaf(x[i], inv, M);
      worst = fmaxf(worst, fabsf(fmaf(x[i], inv, M - b[i])));
    }
    if (__any(!(worst < 0.4999f))) {
#pragma unroll
      for (int i = 0; i < N / 4; ++i)
        to[i] = ((*this)(x[4 * i]) & 255) | ((*this)(x[4 * i + 1]) & 255) << 8 | ((*this)(x[4 * i + 2]) & 255) << 16 |
                (int)((unsigned)(*this)(x[4 * i + 3]) << 24);
    } else {
#pragma unroll
      for (int i = 0; i < N / 4; ++i) {
        const unsigned lo = __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b[4 * i + 1]), __builtin_bit_cast(unsigned, b[4 * i]), 0x0c0c0400u);
        const unsigned hi = __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b[4 * i + 3]), __builtin_bit_cast(unsigned, b[4 * i + 2]), 0x04000c0cu);
        to[i] = (int)(lo | hi);
      }
    }
  }
};

// N elements as they come, zeros from `have` on; wide accesses of global memory may
// begin at any element.
template <class E, int N>
struct Raw {
  typedef unsigned short v2h __attribute__((ext_vector_type(2)));
  static constexpr int WORDS = N * (int)sizeof(E) / 4;
  unsigned w[WORDS];
  __device__ void load(const E* p, int have) {
    struct __attribute__((packed, aligned(sizeof(E)))) Pack {
      unsigned w[WORDS];
    };
    if (have >= N) {
      const Pack k = *reinterpret_cast<const Pack*>(p);
#pragma unroll
      for (int i = 0; i < WORDS; ++i) w[i] = k.w[i];
    } else {
      struct {
        E e[N];
      } k;
#pragma unroll
      for (int i = 0; i < N; ++i) k.e[i] = i < have ? p[i] : (E)0.f;
      struct All {
        unsigned w[WORDS];
      };
      const All all = __builtin_bit_cast(All, k);
#pragma unroll
      for (int i = 0; i < WORDS; ++i) w[i] = all.w[i];
    }
  }
  __device__ void values(float (&v)[N]) const {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (sizeof(E) == 4) {
        v[i] = __builtin_bit_cast(float, w[i]);
      } else {
        v[2 * i] = (float)__builtin_bit_cast(E, (unsigned short)w[i]);
        v[2 * i + 1] = (float)__builtin_bit_cast(E, (unsigned short)(w[i] >> 16));
      }
    }
  }
  // The larger of `most` and the magnitudes, as their bits, whose order is theirs
  // (NaN above all); two of them a word where elements have 16 bits.
  __device__ unsigned larger(unsigned most) const {
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
      if constexpr (sizeof(E) == 4) {
        const unsigned m = w[i] & 0x7fffffffu;
        most = m > most ? m : most;
      } else {
        most = both(most, w[i] & 0x7fff7fffu);
      }
    }
    return most;
  }
  static __device__ unsigned both(unsigned a, unsigned b) {
    if constexpr (sizeof(E) == 4)
      return b > a ? b : a;
    else
      return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(v2h, a), __builtin_bit_cast(v2h, b)));
  }
  // The magnitude that `most` stands for.
  static __device__ float magnitude(unsigned most) {
    if constexpr (sizeof(E) == 4) {
      return __builtin_bit_cast(float, most);
    } else {
      const unsigned a = most & 0xffffu, b = most >> 16;
      return (float)__builtin_bit_cast(E, (unsigned short)(b > a ? b : a));
    }
  }
};

// Rows into tiles, WAVES waves a row, eight inputs a thread at a time, of which the
// first HELD times stay in registers while the row's largest magnitude is found
// (the others are read again).  Workgroup b runs on XCD b % 8: those of the rows of
// a tile are on one, whose L2 puts their codes of 16 bytes together.
template <class E, int WAVES>
__global__ __launch_bounds__(256) void k_q8_rows(const void* x, size_t x_stride, int rows, int K, int kb,
                                                 char* __restrict__ codes, float* __restrict__ scales) {
  constexpr int HELD = WAVES > 1 ? 4 : 2, STEP = 8 * 64 * WAVES;
  constexpr int EACH = 4 / WAVES, GROUPS = 16 / EACH;  // rows a workgroup, workgroups a tile
  typedef Raw<E, 8> R;
  __shared__ unsigned part[4];
  const unsigned id = blockIdx.y * gridDim.x + blockIdx.x, tile = id / (8 * GROUPS) * 8 + id % 8;
  const size_t row = (size_t)tile * 16 + id / 8 % GROUPS * EACH + threadIdx.x / (64 * WAVES);
  if (row >= (size_t)rows) return;  // (whole workgroups where there is a barrier)
  const E* p = static_cast<const E*>(x) + row * x_stride;
  const int first = 8 * ((int)threadIdx.x % (64 * WAVES)), end = kb * kTileK;
  R held[HELD];
  unsigned most = 0;
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    const int k = first + i * STEP;
    if (k < end) held[i].load(p + min(k, K - 1), K - k);
  }
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (first + i * STEP < end) most = held[i].larger(most);
  for (int k = first + HELD * STEP; k < end; k += STEP) {
    R v;
    v.load(p + min(k, K - 1), K - k);
    most = v.larger(most);
  }
#pragma unroll
  for (int m = 1; m < 64; m *= 2) most = R::both(most, __shfl_xor(most, m));
  if constexpr (WAVES > 1) {
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) most = R::both(most, part[w]);
  }
  const Codes code(R::magnitude(most));
  if (first == 0) scales[row] = code.s;
  char* to = codes + row / 16 * kb * 1024 + row % 16 * 16;
  auto store = [&](int k, const R& raw) {
    typedef int v2i __attribute__((ext_vector_type(2)));
    float v[8];
    raw.values(v);
    int w[2];
    code.words(v, w);
    *reinterpret_cast<v2i*>(to + (size_t)(k / kTileK) * 1024 + k % kTileK / 16 * 256 + k % 16) = v2i{w[0], w[1]};
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (first + i * STEP < end) store(first + i * STEP, held[i]);
  for (int k = first + HELD * STEP; k < end; k += STEP) {
    R v;
    v.load(p + min(k, K - 1), K - k);
    store(k, v);
  }
}

template <class E, int WAVES>
hipError_t launch_rows(const Q8Call& c, hipStream_t st) {
  const int each = 8 * 16 * WAVES / 4, tiles = ((c.rows + 15) / 16 + 7) / 8;  // workgroups for eight tiles
  const int x = tiles < 4096 ? tiles : 4096;
  hipLaunchKernelGGL((k_q8_rows<E, WAVES>), dim3((unsigned)(x * each), (unsigned)((tiles + x - 1) / x)), dim3(256), 0, st, c.x,
                     c.x_stride, c.rows, c.K, c.kb, c.row_codes, c.row_scales);
  return hipGetLastError();
}

// Weights: a wave a row, the codes one after another.
__global__ __launch_bounds__(256) void k_q8_quantize(const float* __restrict__ w, int rows, int K,
                                                     char* __restrict__ codes, float* __restrict__ scales) {
  const int lane = (int)threadIdx.x & 63;
  auto larger = [](unsigned a, unsigned b) { return b > a ? b : a; };
  for (long long row = (long long)blockIdx.x * 4 + threadIdx.x / 64; row < rows; row += (long long)gridDim.x * 4) {
    const float* p = w + (size_t)row * K;
    unsigned most = 0;
    for (int k = lane; k < K; k += 64) most = larger(most, __builtin_bit_cast(unsigned, fabsf(p[k])));
#pragma unroll
    for (int m = 1; m < 64; m *= 2) most = larger(most, __shfl_xor(most, m));
    const Codes code(__builtin_bit_cast(float, most));
    if (lane == 0) scales[row] = code.s;
    for (int k = lane; k < K; k += 64) codes[(size_t)row * K + k] = (char)code(p[k]);
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
// every so many'th tile along K, and their sums meet in LDS.  OWN: the workgroup
// quantizes the rows itself, into LDS, under the weights' loads: as long as they
// are few, that is less than a launch of its own.
constexpr int kAhead = 4;   // tiles along K on their way
constexpr int kPiece = 256;  // inputs of a row that a wave quantizes at once
constexpr int kPieces = 2;   // and how many of them

template <class E, int RT, int NT, bool OWN>
__global__ __launch_bounds__(512) void k_q8_few(Q8Call c) {
  static_assert(!OWN || RT == 1, "up to 16 rows");
  extern __shared__ __align__(16) v4i part[];  // [waves][NT][RT][64]; OWN: codes [rows][kb][4] before
  __shared__ unsigned most[16];                // of the rows, as the bits of magnitudes
  const int lane = (int)threadIdx.x & 63, nw = (int)blockDim.x >> 6;
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int nts = (c.N + 15) / 16, rts = (c.rows + 15) / 16;
  const int nt0 = (int)blockIdx.x * NT, rt0 = (int)blockIdx.y * RT;
  const v4i *w[NT], *x[RT];
#pragma unroll
  for (int t = 0; t < NT; ++t) w[t] = reinterpret_cast<const v4i*>(c.codes) + (size_t)min(nt0 + t, nts - 1) * c.kb * 64 + lane;
#pragma unroll
  for (int r = 0; r < RT; ++r) x[r] = reinterpret_cast<const v4i*>(c.row_codes) + (size_t)min(rt0 + r, rts - 1) * c.kb * 64 + lane;
  v4i a[kAhead][NT], b[kAhead][RT], acc[NT][RT];
  auto load = [&](int k0) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int k = min(k0 + u * nw, c.kb - 1);
#pragma unroll
      for (int t = 0; t < NT; ++t) a[u][t] = w[t][(size_t)k * 64];
      if (!OWN) {
#pragma unroll
        for (int r = 0; r < RT; ++r) b[u][r] = x[r][(size_t)k * 64];
      }
    }
  };
  load(wv);
  if constexpr (OWN) {
    const int pieces = (c.K + kPiece - 1) / kPiece, all = c.rows * pieces;
    typedef Raw<E, 4> R;
    R v[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int id = wv + j * nw, row = id / pieces, k = id % pieces * kPiece + 4 * lane;
      if (id < all) v[j].load(static_cast<const E*>(c.x) + (size_t)row * c.x_stride + min(k, c.K - 1), c.K - k);
    }
    if (threadIdx.x < 16) most[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int id = wv + j * nw;
      if (id >= all) break;
      unsigned m = v[j].larger(0);
#pragma unroll
      for (int e = 1; e < 64; e *= 2) m = R::both(m, __shfl_xor(m, e));
      // (the order of these changes nothing)
      if (lane == 0) atomicMax(&most[id / pieces], __builtin_bit_cast(unsigned, R::magnitude(m)));
    }
    __syncthreads();
    int* codes = reinterpret_cast<int*>(part);
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const int id = wv + j * nw, row = id / pieces, k = id % pieces * kPiece + 4 * lane;
      if (id >= all) break;
      const Codes code(__builtin_bit_cast(float, most[row]));
      float x[4];
      v[j].values(x);
      int word[1];
      code.words(x, word);
      if (k < c.kb * kTileK) codes[(row * c.kb * kTileK + k) / 4] = word[0];
    }
    __syncthreads();
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[t][r] = v4i{0, 0, 0, 0};
  for (int k0 = wv; k0 < c.kb; k0 += kAhead * nw) {
    if (k0 > wv) load(k0);
    if constexpr (OWN) {
      const int row = lane & 15, q = lane >> 4;
#pragma unroll
      for (int u = 0; u < kAhead; ++u)  // rows past the last one: what is made of them is not stored
        b[u][0] = part[(min(row, c.rows - 1) * c.kb + min(k0 + u * nw, c.kb - 1)) * 4 + q];
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
  if (OWN) __syncthreads();  // the codes have been read
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
    const float s = OWN ? Codes(__builtin_bit_cast(float, most[at])).s : c.row_scales[at];
    static_cast<E*>(c.y)[(size_t)at * c.y_stride + n] = (E)fmaf((float)v * c.scales[n], s, c.bias ? c.bias[n] : 0.f);
  }
}

template <class E, int RT, int NT, bool OWN>
hipError_t launch_few(const Q8Call& c, int waves, hipStream_t st) {
  if (waves > c.kb) waves = c.kb;
  const dim3 grid((unsigned)(((c.N + 15) / 16 + NT - 1) / NT), (unsigned)((c.rows + 16 * RT - 1) / (16 * RT)));
  size_t lds = (size_t)waves * NT * RT * 1024;
  if (OWN && lds < (size_t)c.rows * c.kb * kTileK) lds = (size_t)c.rows * c.kb * kTileK;
  hipLaunchKernelGGL((k_q8_few<E, RT, NT, OWN>), grid, dim3(64 * waves), lds, st, c);
  return hipGetLastError();
}

// Many rows.  A workgroup of WN x WX waves takes pieces of WN NT tiles of outputs and
// WX RT of rows, one after another, a wave NT x RT of them, in registers.  Stages
// of KT tiles of inputs go from memory straight into LDS, STAGES - 1 ahead of the
// one whose operands are read, which are read a stage ahead of their products; this goes on
// from one piece to the next, whose first stages arrive while the last piece's
// outputs are made and stored.
//
// In pieces of 256 x 256 with four stages, 8192 rows of 8192 inputs to 8192 outputs
// take 485 to 510 us with the rows' codes (a library product of 8-bit integers alone
// 460 to 490), and 16384 rows of 2048 inputs 278 (293).  There the outputs' conversion
// and stores after every 32 stages cost a fifth: stores of 32 bytes of a row took 5 %
// of the whole time more than those of 64, those of 128, for which rows have to change
// lanes too, the same as 64.  Products with a bias take the way of outputs that are not
// whole pieces, 16384 rows of 2048 inputs to 8192 outputs 405 to 413 us against 268 to
// 273.  Two workgroups of 256 x 128 a compute unit, five stages, and stores past the
// caches were slower.
template <class E, int WN, int WX, int NT, int RT, int KT, int STAGES>
__global__ __launch_bounds__(64 * WN * WX, 2) void k_q8_many(Q8Call c) {
  constexpr int WAVES = WN * WX, TN = WN * NT, TX = WX * RT, EACH = (TN + TX) / WAVES;  // rows of tiles that a wave fetches
  constexpr int STAGE = (TN + TX) * KT * 1024;
  static_assert((TN + TX) % WAVES == 0 && (STAGES - 1) * EACH * KT < 64, "the waits below count the transfers of a stage");
  extern __shared__ __align__(16) char lds[];
  const int lane = (int)threadIdx.x & 63, q = lane >> 4, l = lane & 15;
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wn = wv / WX, wx = wv % WX;
  const int nts = (c.N + 15) / 16, rts = (c.rows + 15) / 16, kb = c.kb, ns = kb / KT;
  const int gn = (nts + TN - 1) / TN, gx = (rts + TX - 1) / TX;
  // Workgroup b runs on XCD b % 8: each XCD (and its L2) takes a contiguous range
  // of the pieces, ordered so that those at work together share rows and outputs.
  constexpr int GROUP = 4;  // rows of pieces that go through the outputs together
  const int total = gn * gx, per = total / 8, rest = total % 8, xcd = (int)blockIdx.x % 8;
  const int begin = xcd * per + min(xcd, rest), end = begin + per + (xcd < rest ? 1 : 0);
  const int step = (int)gridDim.x / 8, mine = begin + (int)blockIdx.x / 8;
  if (mine >= end) return;
  const int turns = ((end - mine + step - 1) / step) * ns;
  auto place = [&](int id, int& pn, int& px) {
    const int first = id / (GROUP * gn) * GROUP, have = min(GROUP, gx - first), at = id - first * gn;
    pn = at / have;
    px = first + at % have;
  };
  // what this wave fetches: tiles of outputs first, then of rows (past the last
  // one the last one again: what is made of it is not stored)
  __amdgpu_buffer_rsrc_t from[EACH];
  int fetch_id = mine, fetch_k = 0;
  auto locate = [&]() {
    int pn, px;
    place(fetch_id, pn, px);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int t = wv * EACH + i;
      const char* p = t < TN ? c.codes + (size_t)min(pn * TN + t, nts - 1) * kb * 1024
                             : c.row_codes + (size_t)min(px * TX + t - TN, rts - 1) * kb * 1024;
      from[i] = uniform_buffer(p, (unsigned)kb * 1024u);
    }
  };
  int fetch_to = 0, read_at = 0;  // places in LDS
  auto fetch = [&]() {
#pragma unroll
    for (int i = 0; i < EACH; ++i)
#pragma unroll
      for (int j = 0; j < KT; ++j)
        fetch_to_lds(from[i], lane * 16u, (unsigned)(fetch_k + j) * 1024u, lds + fetch_to + ((wv * EACH + i) * KT + j) * 1024);
    fetch_to = fetch_to + STAGE < STAGES * STAGE ? fetch_to + STAGE : 0;
    fetch_k += KT;
    if (fetch_k == kb) {
      fetch_k = 0;
      fetch_id += step;
      if (fetch_id < end) locate();
    }
  };
  struct Operands {
    v4i a[KT][NT], b[KT][RT];
  };
  auto read = [&](Operands& to) {
    const v4i* at = reinterpret_cast<const v4i*>(lds + read_at) + lane;
#pragma unroll
    for (int j = 0; j < KT; ++j) {
#pragma unroll
      for (int r = 0; r < RT; ++r) to.b[j][r] = at[((TN + wx * RT + r) * KT + j) * 64];
#pragma unroll
      for (int t = 0; t < NT; ++t) to.a[j][t] = at[((wn * NT + t) * KT + j) * 64];
    }
    read_at = read_at + STAGE < STAGES * STAGE ? read_at + STAGE : 0;
  };
  v4i acc[NT][RT];
  // the products of stage g, whose operands are in registers, while those of the
  // next one are read
  auto turn = [&](int g, const Operands& now, Operands& next) {
    // this wave's transfers of stage g + 1 have arrived, those of the stages after it
    // may be on their way; then all waves' have, and stage g has been read
    if (g + STAGES > turns)
      wait_memory_but<0>();
    else
      wait_memory_but<(STAGES - 2) * EACH * KT>();
    barrier_for_lds();
    read(next);  // (after the last stage: what is not used)
    if (g + STAGES < turns) fetch();
#pragma unroll
    for (int j = 0; j < KT; ++j)
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < RT; ++r)
          acc[t][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(now.a[j][t], now.b[j][r], acc[t][r], 0, 0, 0);
  };
  locate();
#pragma unroll
  for (int g = 0; g < STAGES; ++g)
    if (g < turns) fetch();
  if (turns >= STAGES)
    wait_memory_but<(STAGES - 1) * EACH * KT>();
  else
    wait_memory_but<0>();
  barrier_for_lds();
  Operands even, odd;
  read(even);
  for (int id = mine, g = 0; id < end; id += step) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int r = 0; r < RT; ++r) acc[t][r] = v4i{0, 0, 0, 0};
    for (int k = 0; k + 1 < ns; k += 2, g += 2) {
      turn(g, even, odd);
      turn(g + 1, odd, even);
    }
    if (KT > 1 && ns % 2) {  // (tiles come in pairs)
      turn(g++, even, odd);
      even = odd;
    }
    // outputs 4 q ..+3 of tile t, row l of tile r; all scales are on their way before
    // the first is used
    int pn, px;
    place(id, pn, px);
    const int row0 = (px * TX + wx * RT) * 16 + l, n0 = (pn * TN + wn * NT) * 16 + 4 * q;
    const bool whole = (pn * TN + wn * NT + NT) * 16 <= c.N;  // the same for all lanes
    v4f scale[NT];
    float by[RT];
    auto four = [&](const float* p, int n) {
      struct __attribute__((packed, aligned(4))) Pack {
        float f[4];
      };
      v4f v;
      if (whole) {
        const Pack k = *reinterpret_cast<const Pack*>(p + n);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = k.f[i];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = p[min(n + i, c.N - 1)];
      }
      return v;
    };
#pragma unroll
    for (int t = 0; t < NT; ++t) scale[t] = four(c.scales, n0 + 16 * t);
#pragma unroll
    for (int r = 0; r < RT; ++r) by[r] = c.row_scales[min(row0 + 16 * r, c.rows - 1)];
    struct Out {
      E e[4];
    };
    struct Two {
      unsigned w[2];
    };
    auto make = [&](int t, int r) {
      Out out;
#pragma unroll
      for (int i = 0; i < 4; ++i) out.e[i] = (E)((float)acc[t][r][i] * scale[t][i] * by[r]);
      return out;
    };
    if (whole && !c.bias && c.wide && (px * TX + wx * RT + RT) * 16 <= c.rows) {
      const unsigned each = (unsigned)c.y_stride * (unsigned)sizeof(E);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const auto y = uniform_buffer(static_cast<E*>(c.y) + (size_t)(px * TX + wx * RT + r) * 16 * c.y_stride +
                                          (pn * TN + wn * NT) * 16, 15 * each + NT * 16 * (unsigned)sizeof(E));
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
          typedef unsigned v4u __attribute__((ext_vector_type(4)));
          if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
              __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, make(t + i, r)), y, (int)(l * each + 64 * (t + i) + 16 * q),
                                                     0, 0);
          } else {
            // lanes 16 apart exchange halves of two tiles, so that each has eight outputs of
            // one: 64 bytes of a row a store in place of 32
            const Two a = __builtin_bit_cast(Two, make(t, r)), b = __builtin_bit_cast(Two, make(t + 1, r));
            const auto lo = __builtin_amdgcn_permlane16_swap(a.w[0], b.w[0], false, false);
            const auto hi = __builtin_amdgcn_permlane16_swap(a.w[1], b.w[1], false, false);
            __builtin_amdgcn_raw_buffer_store_b128(v4u{lo[0], hi[0], lo[1], hi[1]}, y,
                                                   (int)(l * each + 32 * (t + (q & 1)) + 16 * (q >> 1)), 0, 0);
          }
        }
      }
    } else {
      E* y = static_cast<E*>(c.y) + (size_t)row0 * c.y_stride + n0;
#pragma unroll
      for (int r = 0; r < RT; ++r, y += 16 * c.y_stride) {
        if (row0 + 16 * r >= c.rows) break;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int n = n0 + 16 * t;
          struct __attribute__((packed, aligned(sizeof(E)))) Pack {
            E e[4];
          } out;
          if (c.bias) {
            const v4f bias = four(c.bias, n);
#pragma unroll
            for (int i = 0; i < 4; ++i) out.e[i] = (E)fmaf((float)acc[t][r][i] * scale[t][i], by[r], bias[i]);
          } else {
            const Out o = make(t, r);
#pragma unroll
            for (int i = 0; i < 4; ++i) out.e[i] = o.e[i];
          }
          if (whole || n + 4 <= c.N) {
            *reinterpret_cast<Pack*>(y + 16 * t) = out;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (n + i < c.N) y[16 * t + i] = out.e[i];
          }
        }
      }
    }
    // (stores count among the transfers that the turns wait for; to count them in
    // there, and leave them on their way, takes the same time)
    wait_memory_but<0>();
  }
}

template <class E, int WN, int WX, int NT, int RT, int KT, int STAGES>
hipError_t launch_many(const Q8Call& c, hipStream_t st) {
  constexpr int TN = WN * NT, TX = WX * RT, LDS = STAGES * (TN + TX) * KT * 1024;
  const long long gn = ((c.N + 15) / 16 + TN - 1) / TN, gx = ((c.rows + 15) / 16 + TX - 1) / TX;
  const long long room = LDS > 81920 ? 256 : 512;  // workgroups that fit the card
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_q8_many<E, WN, WX, NT, RT, KT, STAGES>),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
  if (e != hipSuccess) return e;
  const unsigned grid = (unsigned)(gn * gx < room ? (gn * gx + 7) / 8 * 8 : room);
  hipLaunchKernelGGL((k_q8_many<E, WN, WX, NT, RT, KT, STAGES>), dim3(grid), dim3(64 * WN * WX), LDS, st, c);
  return hipGetLastError();
}

template <class E>
hipError_t launch_q8(const Q8Call& c, hipStream_t st) {
  const int few = c.kb < 8 ? c.kb : 8;  // waves
  // Rows quantized in the product's launch: us with and without, rows x inputs -> 2048 outputs:
  //   1 x 2048  3.8  5.5   2 x 2048  4.7  5.7   3 x 2048  5.6  5.6   4 x 2048  6.4  5.6   4 x 512  3.8  5.2
  //   1 x 4096  5.2  6.4   2 x 4096  6.6  6.4   1 x 8192  8.0  8.4 (to 8192 outputs, 4 x 2048: 8.7 and 6.1)
  if (c.rows <= 16 && (long long)c.rows * ((c.K + kPiece - 1) / kPiece) <= kPieces * few)
    return launch_few<E, 1, 1, true>(c, few, st);
  // Waves a row: us of 1 and 4, for rows of bf16 x inputs with a small product:
  //   64 x 512    5.9   5.9    4096 x 512    9.4  11.5    16384 x 512   17.6  24.9    64 x 1000    6.9   6.0
  //   4096 x 1000 12.5  14.2   512 x 2048    9.2   6.9    4096 x 2048   19.9  18.4    16384 x 4096 58.9  50.8
  const hipError_t e = c.kb <= 16 ? launch_rows<E, 1>(c, st) : launch_rows<E, 4>(c, st);
  if (e != hipSuccess) return e;
  // Pieces of outputs and rows: the largest that still are workgroups enough, in tiles of 16.  us for
  // rows x inputs -> outputs, bf16, both launches, as few<RT, NT> 1,1 2,1 2,2, many 64 x 64, 128 x 64, 128 x 128, 256 x 256:
  //   32 x 2048 -> 2048     6.7  7.0  8.1  11.3   64 x 2048 -> 2048    7.3   7.2   8.2  11.3  13.4   17
  //   64 x 2048 -> 8192     11   10.5 10.3 11.4  128 x 2048 -> 8192   16    14.6  14.8 11.9  13.9   18
  //   256 x 8192 -> 2048    31   26   21   30    512 x 2048 -> 2048               16   13    15     20   37
  //   512 x 2048 -> 8192              42   24   21   22   38   1024 x 2048 -> 8192     80   42   36   31   43
  //   512 x 4096 -> 16384             150  69   53   45   64   2048 x 2048 -> 8192     158  83   69   60   56
  const long long n = (c.N + 15) / 16, r = (c.rows + 15) / 16;
  auto pieces = [&](int tn, int tr) { return ((n + tn - 1) / tn) * ((r + tr - 1) / tr); };
  if (r == 1 || pieces(1, 1) <= 512) return launch_few<E, 1, 1, false>(c, few, st);
  if (pieces(1, 2) <= 512) return launch_few<E, 2, 1, false>(c, few, st);
  if (pieces(2, 2) <= 640) return launch_few<E, 2, 2, false>(c, few, st);
  if (pieces(16, 16) >= 192) return launch_many<E, 2, 4, 8, 4, 1, 4>(c, st);
  if (pieces(8, 8) >= 384) return launch_many<E, 2, 2, 4, 4, 1, 5>(c, st);
  if (pieces(8, 4) >= 384) return launch_many<E, 2, 2, 4, 2, 2, 3>(c, st);
  return launch_many<E, 2, 2, 2, 2, 2, 5>(c, st);
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
    if ((double)rows * s.N > 4398046511104.0) return q8_fail(ctx, LCSM_EINVAL, "more than 2^42 outputs");
    if (!x || !y) return q8_fail(ctx, LCSM_EINVAL, "null input or output pointer");
    if (x_stride < (size_t)s.K || y_stride < (size_t)s.N)
      return q8_fail(ctx, LCSM_EINVAL, "a row stride is shorter than the row");
  }
  if (ctx->faulted) return LCSM_ESTATE;
  if (!rows) return LCSM_OK;
  const size_t m = (size_t)layer;
  const lcsm::Q8Call c{rows, s.N, s.K, ctx->kb, x, y, x_stride, y_stride, ctx->codes + m * ctx->nts * ctx->kb * 1024,
                       ctx->scales + m * s.N, ctx->bias ? ctx->bias + m * s.N : nullptr, ctx->row_codes,
                       ctx->row_scales,
                       (uintptr_t)y % 16 == 0 && y_stride * lcsm::dtype_size(dtype) % 16 == 0 && y_stride <= lcsm::kMaxStride};
  const hipError_t e = lcsm::with_dtype(dtype, [&](auto v) { return lcsm::launch_q8<decltype(v)>(c, ctx->stream); });
  return e == hipSuccess ? LCSM_OK : q8_fail(ctx, LCSM_EDEVICE, "product launch", e);
}

int lcsm_q8_quantize(const float* w, int rows, int K, void* codes, float* scales, void* stream) {
  if (rows < 0 || K < 1 || K > (1 << 24)) return LCSM_EINVAL;
  if (!rows) return LCSM_OK;
  if (!w || !codes || !scales) return LCSM_EINVAL;
  const long long blocks = ((long long)rows + 3) / 4;  // (a launch has less than 2^32 threads)
  hipLaunchKernelGGL(lcsm::k_q8_quantize, dim3((unsigned)(blocks < (1 << 20) ? blocks : 1 << 20)), dim3(256), 0, (hipStream_t)stream, w,
                     rows, K, (char*)codes, scales);
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
