// Matrix-vector products with 4-bit weights and group scales (lcsm_q4.h).
//
// The codes are kept as tiles of 16 outputs x 128 inputs, 16 bytes a lane: lane
// l's word j holds the eight codes of output l % 16 for the inputs 32 j + 8 (l
// / 16) ..+7, which is the lane's share of a 16x16x32 matrix product's right
// operand.  What x is multiplied by is code - 8, exactly, whatever its type:
// with anything larger in place of it (16 + code is one operation) sums of x
// come off again that are up to six times the result's terms, which costs three
// bits of them and overflows where the result does not.  A code is kept as sign
// and magnitude, so that a byte of them is an 8-bit float (below 2^-5 those are
// whole multiples of 2^-9), two of which are one conversion.  A product of x
// with ones gives the sum of x, in the same lanes, for zeros other than 8.
// fp32 rows are taken apart into three bf16 values that hold all of their bits.
//
// One token through 8512 x 2048 weights in groups of 128 takes 5.4 us, 1.7 TB/s of
// the 9 MB that are read (1.9 us at the copy rate): a launch, a round trip for
// the codes and the sum in LDS are most of it.  16 rows of fp16 through 2048 x
// 4096 in groups of 64 7.6 us, five of fp32 through 1543 x 773 4.8.  Rows of whole
// prompts take the same kernel, which reads x anew for every 64 outputs and unpacks
// the codes anew for every 64 rows: 4096 bf16 rows through 8512 x 2048 459 us, 311
// TFLOP/s, three times what a library product with weights of 16 bits takes.
#include <math.h>
#include <stdio.h>
#include <string.h>

#include <new>
#include <type_traits>

#include "lcsm_elem.h"
#include "lcsm_q4.h"

namespace lcsm {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef bf16_t v8bf __attribute__((ext_vector_type(8)));
typedef f16_t v8h __attribute__((ext_vector_type(8)));

constexpr int kTileN = 16, kTileK = 128;  // weights of a tile
constexpr int kMaxWaves = 16;

struct Q4Call {
  int rows, N, K, group, ng, kb;  // kb: tiles along K
  int scale_dtype;
  const void *x, *codes, *scales;
  const uint8_t* zeros;  // NULL: 8
  const float* bias;     // NULL: none
  void* y;
  size_t x_stride, y_stride;
};

// ---- what multiplies: the element's matrix operand, and x as one or three of them

template <class E>
struct Mat {  // fp16
  typedef v8h V;
  static constexpr int PARTS = 1;
  static __device__ v4f mul(V a, V b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};
struct MatBf {
  typedef v8bf V;
  static constexpr int PARTS = 1;
  static __device__ v4f mul(V a, V b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Mat<bf16_t> : MatBf {};
template <>
struct Mat<float> : MatBf {
  static constexpr int PARTS = 3;
};

// v = code - 8 of a word's eight codes (word_of).
template <class E>
__device__ __forceinline__ typename Mat<E>::V weights(unsigned w) {
  v4u r;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const unsigned k = half ? __builtin_rotateright32(w, 4) : w;
    // four bytes, the sign on top and |v|: what is kept is |v| - 1 of negative ones
    const unsigned bytes = (k & 0x87878787u) + (k >> 7 & 0x01010101u);
    if constexpr (std::is_same<E, f16_t>::value) {
      r[2 * half] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(bytes, 512.f, false));
      r[2 * half + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(bytes, 512.f, true));
    } else {
      r[2 * half] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes, 512.f, false));
      r[2 * half + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes, 512.f, true));
    }
  }
  return __builtin_bit_cast(typename Mat<E>::V, r);
}
// Eight codes as a word: e < 4 with the sign of code - 8 at bit 8 e + 7 and three
// bits of magnitude from 8 e on, the others likewise after a rotation by four.
__device__ __forceinline__ unsigned word_of(const unsigned (&code)[8]) {
  unsigned half[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) half[e / 4] |= (code[e] < 8 ? 0x80 | (7 - code[e]) : code[e] - 8) << (8 * (e % 4));
  return half[0] | __builtin_rotateleft32(half[1], 4);
}

template <class E, int XV>
__device__ __forceinline__ void operand(const v4u (&x)[XV], typename Mat<E>::V (&a)[Mat<E>::PARTS]) {
  if constexpr (std::is_same<E, float>::value) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const unsigned w = x[i / 4][i % 4];
      const float v = __builtin_bit_cast(float, w);
      const bf16_t hi = (bf16_t)v;
      const float r1 = v - (float)hi;
      const bf16_t mid = (bf16_t)r1;
      a[0][i] = hi;
      a[1][i] = mid;
      a[2][i] = (bf16_t)(r1 - (float)mid);
    }
  } else {
    a[0] = __builtin_bit_cast(typename Mat<E>::V, x[0]);
  }
}

__device__ __forceinline__ float scale_at(const void* p, int dtype, size_t i) {
  if (dtype == LCSM_BF16) return (float)static_cast<const bf16_t*>(p)[i];
  if (dtype == LCSM_F16) return (float)static_cast<const f16_t*>(p)[i];
  return static_cast<const float*>(p)[i];
}

// What a wave loads of a tile ahead of its products: codes, scales and zeros, and
// for up to 16 rows x as it comes (more rows would not leave the registers).
template <class E, int SPG, int RT, int NT>
struct Tile {
  static constexpr int GS = 4 / SPG;                 // scales a tile and output
  static constexpr int XV = sizeof(E) == 4 ? 2 : 1;  // 16-byte loads for eight inputs
  static constexpr int XA = RT == 1 ? 4 : 1;
  v4u w[NT], x[XA][RT][XV];
  float s[NT][GS], z[NT][GS];
};

// Waves of a workgroup at most: 16, with 128 registers each, where few are left
// over, else 8.  Pieces of four tiles with a scale for all 128 inputs spill 19 of
// them: one bf16 row through 8512 x 2048 takes 6.0 us, 7.3 by 8 waves, 16 rows 6.7
// and 8.1.  (With 8 waves, pieces of four tiles of rows and two of outputs with a
// scale every 32 inputs spill 65 of 256.)
template <class E, int SPG>
constexpr int q4_waves(int RT, int NT) {
  return RT == 1 && (NT == 1 || (sizeof(E) == 2 && (NT == 2 || SPG == 4))) ? kMaxWaves : kMaxWaves / 2;
}

// A workgroup takes NT tiles of 16 outputs and RT of 16 rows; its waves take
// every so many'th tile along K, their sums meet in LDS and are added in a
// fixed order.  SPG: 32-input products a scale (4: a scale for the whole tile).
// The next tile's loads are on their way while one is multiplied.
template <class E, int SPG, int RT, int NT>
__global__ __launch_bounds__((q4_waves<E, SPG>(RT, NT)) * 64) void k_q4(Q4Call c) {
  typedef Mat<E> T;
  typedef Tile<E, SPG, RT, NT> Tl;
  constexpr int GS = Tl::GS;
  extern __shared__ float part[];  // [waves][NT][RT][16 rows][16 outputs]
  const int lane = (int)threadIdx.x & 63, nw = (int)blockDim.x >> 6;
  const int wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int q = lane >> 4, col = lane & 15;
  const int nt0 = (int)blockIdx.x * NT, r0 = (int)blockIdx.y * 16 * RT;
  const int nts = (c.N + kTileN - 1) / kTileN;
  const unsigned one = std::is_same<E, f16_t>::value ? 0x3C003C00u : 0x3F803F80u;
  const typename T::V ones = __builtin_bit_cast(typename T::V, (v4u){one, one, one, one});
  const v4f none = {0.f, 0.f, 0.f, 0.f};
  v4f y[NT][RT];
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r) y[t][r] = none;
  // rows past the last one are the last one again: an output row has its x row
  // only, and these are not stored
  const E* row[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r)
    row[r] = static_cast<const E*>(c.x) + (size_t)min(r0 + 16 * r + col, c.rows - 1) * c.x_stride + 8 * q;

  // inputs 32 j + 8 q ..+7 of tile kb, zeros past K
  auto load_x = [&](int kb, int j, v4u (&to)[RT][Tl::XV]) {
    const int k0 = kb * kTileK + 32 * j;
    if ((kb + 1) * kTileK <= c.K) {
      // rows may begin anywhere: wide accesses of global memory allow that (44 rows of
      // 6386 fp16 values through 160 outputs: 9 us, 34 one value at a time)
      struct __attribute__((packed, aligned(sizeof(E)))) Wide {
        v4u v[Tl::XV];
      };
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const Wide x = *reinterpret_cast<const Wide*>(row[r] + k0);
#pragma unroll
        for (int v = 0; v < Tl::XV; ++v) to[r][v] = x.v[v];
      }
    } else {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        struct {
          E e[8];
        } p;
#pragma unroll
        for (int i = 0; i < 8; ++i) p.e[i] = k0 + i + 8 * q < c.K ? row[r][k0 + i] : (E)0.f;
        struct Words {
          v4u v[Tl::XV];
        };
        const Words w = __builtin_bit_cast(Words, p);
#pragma unroll
        for (int v = 0; v < Tl::XV; ++v) to[r][v] = w.v[v];
      }
    }
  };
  auto load = [&](int kb, Tl& to) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const size_t nt = (size_t)min(nt0 + t, nts - 1);
      to.w[t] = static_cast<const v4u*>(c.codes)[(nt * c.kb + kb) * 64 + lane];
#pragma unroll
      for (int g = 0; g < GS; ++g) {
        const int at = SPG == 4 ? kb * kTileK / c.group : min(kb * GS + g, c.ng - 1);
        const size_t i = (nt * c.ng + at) * kTileN + col;
        to.s[t][g] = scale_at(c.scales, c.scale_dtype, i);
        to.z[t][g] = 8.f - (c.zeros ? (float)c.zeros[i] : 8.f);
      }
    }
    if (RT == 1) {
#pragma unroll
      for (int j = 0; j < 4; ++j) load_x(kb, j, to.x[RT == 1 ? j : 0]);
    }
  };
  auto multiply = [&](int kb, Tl& tl) {
    v4f acc[NT][RT], sum[RT];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      typename T::V a[RT][T::PARTS];
      if (RT > 1) load_x(kb, j, tl.x[0]);
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        operand<E>(tl.x[RT == 1 ? j : 0][r], a[r]);
        if (j % SPG == 0) sum[r] = none;
#pragma unroll
        for (int p = 0; p < T::PARTS; ++p) sum[r] = T::mul(a[r][p], ones, sum[r]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const typename T::V b = weights<E>(tl.w[t][j]);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          if (j % SPG == 0) acc[t][r] = none;
#pragma unroll
          for (int p = 0; p < T::PARTS; ++p) acc[t][r] = T::mul(a[r][p], b, acc[t][r]);
        }
      }
      if (j % SPG == SPG - 1) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              y[t][r][e] = fmaf(tl.s[t][j / SPG], fmaf(tl.z[t][j / SPG], sum[r][e], acc[t][r][e]), y[t][r][e]);
      }
    }
  };
  Tl a, b;
  int kb = wv;
  if (kb < c.kb) load(kb, a);
  while (kb < c.kb) {
    if (kb + nw < c.kb) load(kb + nw, b);
    multiply(kb, a);
    kb += nw;
    if (kb >= c.kb) break;
    if (kb + nw < c.kb) load(kb + nw, a);
    multiply(kb, b);
    kb += nw;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        part[(((wv * NT + t) * RT + r) * 16 + 4 * q + e) * 16 + col] = y[t][r][e];
  __syncthreads();
  constexpr int OUT = NT * RT * 256;
  for (int o = (int)threadIdx.x; o < OUT; o += (int)blockDim.x) {
    const int t = o / (RT * 256), r = o / 16 % (RT * 16), n = (nt0 + t) * kTileN + o % 16;
    const int at = r0 + r;
    if (n >= c.N || at >= c.rows) continue;
    float v = c.bias ? c.bias[n] : 0.f;
    for (int w = 0; w < nw; ++w) v += part[w * OUT + o];
    static_cast<E*>(c.y)[(size_t)at * c.y_stride + n] = (E)v;
  }
}

// The codes of one lane's 16 bytes: a thread per 32-bit word.
__global__ __launch_bounds__(256) void k_q4_codes(const uint8_t* __restrict__ src, unsigned* __restrict__ dst,
                                                  int M, int N, int K, int nts, int kb) {
  const size_t n = (size_t)M * nts * kb * 256, step = (size_t)gridDim.x * 256;
  const size_t bytes = ((size_t)K + 1) / 2;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    const int j = (int)(i % 4), lane = (int)(i / 4 % 64);
    const size_t tile = i / 256, tk = tile % kb, tn = tile / kb % nts, m = tile / kb / nts;
    const size_t out = tn * kTileN + lane % 16, k0 = tk * kTileK + 32 * j + 8 * (lane / 16);
    unsigned code[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const size_t k = k0 + e;
      code[e] = out < (size_t)N && k < (size_t)K ? src[(m * N + out) * bytes + k / 2] >> (4 * (k & 1)) & 15u : 8u;
    }
    dst[i] = word_of(code);
  }
}

// [M][N][ng] values of SZ bytes as [M][tile][ng][16].
template <class T>
__global__ __launch_bounds__(256) void k_q4_groups(const T* __restrict__ src, T* __restrict__ dst, int M, int N,
                                                   int ng, int nts, T mask) {
  const size_t n = (size_t)M * nts * ng * 16, step = (size_t)gridDim.x * 256;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    const size_t g = i / 16 % ng, tn = i / 16 / ng % nts, m = i / 16 / ng / nts, out = tn * 16 + i % 16;
    dst[i] = out < (size_t)N ? (T)(src[(m * N + out) * ng + g] & mask) : (T)0;
  }
}

// A wave per group of a row: the largest magnitude (NaN where one is), then the
// codes of two neighbouring weights a lane at a time.
__global__ __launch_bounds__(256) void k_q4_quantize(const float* __restrict__ w, int rows, int K, int group,
                                                     int ng, int scale_dtype, uint8_t* __restrict__ codes,
                                                     void* __restrict__ scales) {
  const int lane = (int)threadIdx.x & 63;
  const size_t groups = (size_t)rows * ng, bytes = ((size_t)K + 1) / 2;
  for (size_t i = (size_t)blockIdx.x * 4 + threadIdx.x / 64; i < groups; i += (size_t)gridDim.x * 4) {
    const size_t row = i / ng;
    const int k0 = (int)(i % ng) * group, k1 = min(k0 + group, K);
    const float* p = w + row * K;
    float most = 0.f;
    auto larger = [](float a, float b) { return b > a || b != b ? b : a; };
    for (int k = k0 + lane; k < k1; k += 64) most = larger(most, fabsf(p[k]));
#pragma unroll
    for (int m = 1; m < 64; m *= 2) most = larger(most, __shfl_xor(most, m));
    float s = __fdiv_rn(most, 7.f);
    if (scale_dtype == LCSM_BF16) s = (float)(bf16_t)s;
    if (scale_dtype == LCSM_F16) s = (float)(f16_t)s;
    if (lane == 0) {
      if (scale_dtype == LCSM_BF16) static_cast<bf16_t*>(scales)[i] = (bf16_t)s;
      if (scale_dtype == LCSM_F16) static_cast<f16_t*>(scales)[i] = (f16_t)s;
      if (scale_dtype == LCSM_F32) static_cast<float*>(scales)[i] = s;
    }
    auto code = [&](int k) -> unsigned {
      if (k >= k1 || s == 0.f || !(s < INFINITY)) return 8u;
      return (unsigned)(int)fminf(fmaxf(rintf(__fdiv_rn(p[k], s)) + 8.f, 0.f), 15.f);
    };
    for (int k = k0 + 2 * lane; k < k1; k += 128)  // groups begin at even k
      codes[row * bytes + k / 2] = (uint8_t)(code(k) | code(k + 1) << 4);
  }
}

template <class E, int SPG, int RT, int NT>
hipError_t launch(const Q4Call& c, int most, hipStream_t st) {
  constexpr int MOST = q4_waves<E, SPG>(RT, NT);
  if (most > MOST) most = MOST;
  const int waves = c.kb < most ? c.kb : most;
  const size_t lds = (size_t)waves * NT * RT * 1024;
  const dim3 grid((unsigned)(((c.N + 15) / 16 + NT - 1) / NT), (unsigned)((c.rows + 16 * RT - 1) / (16 * RT)));
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_q4<E, SPG, RT, NT>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((k_q4<E, SPG, RT, NT>), grid, dim3(64 * waves), lds, st, c);
  return hipGetLastError();
}

// The largest pieces that still are workgroups enough: a piece of NT tiles reads
// x once for all of them, one of RT tiles of rows unpacks the codes once.  bf16,
// groups of 128, us (workgroups' pieces as RT NT / waves):
//   one row, 8512 x 2048: 11/8 5.4, 12/8 5.9, 14/16 6.0;  2048 x 4096: 11/16 4.4,
//   12/16 5.9;  16384 x 8192: 12/8 19.1, 11/8 20.6, 14/16 21.6
//   16 rows, 8512 x 2048: 14/16 6.6, 12/8 7.5, 11/8 8.5;  2048 x 4096: 11/16 6.5,
//   12/16 7.5, 14/16 10.8;  16384 x 8192: 12/8 23.5, 14/16 24.4, 11/8 34.4
//   32 rows, 8512 x 2048: 24/8 9.0, 12/8 10.6;  4096 x 1024: 12/8 3.9, 11/16 4.5;
//   2048 x 4096: 11/16 6.7, 12/16 7.5
//   64 rows, 8512 x 2048: 44/8 13.6, 22/8 15.9;  4096 x 1024: 12/8 5.1, 14/16 5.3;
//   2048 x 4096: 12/16 7.7, 11/16 11.6
// fp16 is the same.  fp32 and shorter groups follow the same thresholds, which were
// not chosen for them: up to 2048 x 4096 what the rule takes is within 6 % of the
// best of these pieces (4096 x 1024 with 64 rows in groups of 32 19 %), for more
// outputs it falls behind by up to a half in fp32 (64 rows 16384 x 8192: 22/8 134,
// 24/8 90) and three quarters in groups of 32 (64 rows 8512 x 2048: 42/8 41, 22/8 23).
template <class E, int SPG>
hipError_t launch_rows(const Q4Call& c, hipStream_t st) {
  const long long tiles = (c.N + 15) / 16, rows = (c.rows + 15) / 16;
  auto groups = [&](int rt, int nt) { return (tiles + nt - 1) / nt * ((rows + rt - 1) / rt); };
  if (rows > 2) {
    // (scales for every 32 or 64 inputs, or fp32 rows in three parts, leave no
    // registers for pieces as large)
    constexpr int RT = sizeof(E) == 4 ? 2 : 4, NT = SPG == 4 && sizeof(E) == 2 ? 4 : 2;
    if (groups(4, 4) >= 128) return launch<E, SPG, RT, NT>(c, 8, st);
    if (groups(1, 4) >= 256) return launch<E, SPG, 1, 4>(c, 16, st);
    return launch<E, SPG, 1, 2>(c, 16, st);
  }
  if (rows == 2) {
    constexpr int NT = SPG == 4 && sizeof(E) == 2 ? 4 : 2;
    if (groups(2, 4) >= 128) return launch<E, SPG, 2, NT>(c, 8, st);
    if (groups(1, 2) >= 256) return launch<E, SPG, 1, 2>(c, 8, st);
    return launch<E, SPG, 1, 1>(c, 16, st);
  }
  if (tiles < 512) return launch<E, SPG, 1, 1>(c, 16, st);
  if (c.kb <= 16) return launch<E, SPG, 1, 4>(c, 16, st);
  return launch<E, SPG, 1, 2>(c, 8, st);
}

template <class E>
hipError_t launch_q4(const Q4Call& c, hipStream_t st) {
  if (c.group == 32) return launch_rows<E, 1>(c, st);
  if (c.group == 64) return launch_rows<E, 2>(c, st);
  return launch_rows<E, 4>(c, st);
}

unsigned blocks(size_t n) {
  const size_t b = (n + 255) / 256;
  return (unsigned)(b < 16384 ? b : 16384);
}

}  // namespace
}  // namespace lcsm

struct lcsm_q4 {
  lcsm_q4_shape s;
  int nts, kb, ng;
  hipStream_t stream;
  char* mem;
  void* owned;
  char *codes, *scales;
  uint8_t* zeros;
  float* bias;
  bool faulted;
  char msg[256];
};

namespace {

struct Plan {
  int nts, kb, ng;
  size_t codes, scales, zeros, bias, total;
};

bool group_ok(int g) { return g == 32 || g == 64 || (g > 0 && g % 128 == 0); }

bool q4_plan(const lcsm_q4_shape* s, Plan* p) {
  if (!s || s->M < 1 || s->M > 16384 || s->N < 1 || s->K < 1 || s->N > (1 << 24) || s->K > (1 << 24) ||
      !group_ok(s->group) || !lcsm::dtype_ok(s->scale_dtype))
    return false;
  for (int r : s->reserved)
    if (r) return false;
  if ((double)s->N * s->K > 1099511627776.0) return false;
  p->nts = (s->N + 15) / 16;
  p->kb = (s->K + 127) / 128;
  p->ng = (int)(((long long)s->K + s->group - 1) / s->group);
  const size_t M = (size_t)s->M, groups = M * p->nts * p->ng * 16;
  size_t at = 0;
  auto take = [&](size_t* where, size_t bytes) {
    *where = at;
    at = (at + bytes + 255) / 256 * 256;
  };
  take(&p->codes, M * p->nts * p->kb * 1024);
  take(&p->scales, groups * lcsm::dtype_size(s->scale_dtype));
  take(&p->zeros, groups);
  take(&p->bias, M * s->N * sizeof(float));
  p->total = at;
  return true;
}

int q4_fail(lcsm_q4* c, int code, const char* what, hipError_t e = hipSuccess) {
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

int lcsm_q4_workspace_bytes(const lcsm_q4_shape* shape, size_t* bytes) {
  Plan p;
  if (!bytes || !q4_plan(shape, &p)) return LCSM_EINVAL;
  *bytes = p.total;
  return LCSM_OK;
}

int lcsm_q4_init(lcsm_q4** out, const lcsm_q4_shape* shape, const void* codes, const void* scales,
                 const void* zeros, const float* bias, void* stream, void* workspace,
                 size_t workspace_bytes) {
  if (!out) return LCSM_EINVAL;
  *out = nullptr;
  Plan p;
  if (!codes || !scales || !q4_plan(shape, &p)) return LCSM_EINVAL;
  if (workspace && ((uintptr_t)workspace & 255)) return LCSM_EINVAL;
  if (workspace && workspace_bytes < p.total) return LCSM_ENOMEM;
  lcsm_q4* c = new (std::nothrow) lcsm_q4();
  if (!c) return LCSM_ENOMEM;
  c->s = *shape;
  c->nts = p.nts;
  c->kb = p.kb;
  c->ng = p.ng;
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
  c->codes = c->mem + p.codes;
  c->scales = c->mem + p.scales;
  c->zeros = zeros ? (uint8_t*)(c->mem + p.zeros) : nullptr;
  c->bias = bias ? (float*)(c->mem + p.bias) : nullptr;
  const int M = shape->M, N = shape->N;
  const size_t words = (size_t)M * p.nts * p.kb * 256, groups = (size_t)M * p.nts * p.ng * 16;
  hipLaunchKernelGGL(lcsm::k_q4_codes, dim3(lcsm::blocks(words)), dim3(256), 0, c->stream,
                     (const uint8_t*)codes, (unsigned*)c->codes, M, N, shape->K, p.nts, p.kb);
  if (shape->scale_dtype == LCSM_F32)
    hipLaunchKernelGGL(lcsm::k_q4_groups<uint32_t>, dim3(lcsm::blocks(groups)), dim3(256), 0, c->stream,
                       (const uint32_t*)scales, (uint32_t*)c->scales, M, N, p.ng, p.nts, 0xffffffffu);
  else
    hipLaunchKernelGGL(lcsm::k_q4_groups<uint16_t>, dim3(lcsm::blocks(groups)), dim3(256), 0, c->stream,
                       (const uint16_t*)scales, (uint16_t*)c->scales, M, N, p.ng, p.nts, (uint16_t)0xffff);
  if (zeros)
    hipLaunchKernelGGL(lcsm::k_q4_groups<uint8_t>, dim3(lcsm::blocks(groups)), dim3(256), 0, c->stream,
                       (const uint8_t*)zeros, c->zeros, M, N, p.ng, p.nts, (uint8_t)15);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess && bias)
    e = hipMemcpyAsync(c->bias, bias, (size_t)M * N * sizeof(float), hipMemcpyDeviceToDevice, c->stream);
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

int lcsm_q4_matvec(lcsm_q4* ctx, int layer, int rows, int dtype, const void* x, size_t x_stride,
                   void* y, size_t y_stride) {
  if (!ctx) return LCSM_EINVAL;
  const lcsm_q4_shape& s = ctx->s;
  if (layer < 0 || layer >= s.M) return q4_fail(ctx, LCSM_EINVAL, "layer out of range");
  if (rows < 0 || !lcsm::dtype_ok(dtype)) return q4_fail(ctx, LCSM_EINVAL, "rows below zero or unknown type");
  if (rows > 0) {
    if (!x || !y) return q4_fail(ctx, LCSM_EINVAL, "null input or output pointer");
    if (x_stride < (size_t)s.K || y_stride < (size_t)s.N)
      return q4_fail(ctx, LCSM_EINVAL, "a row stride is shorter than the row");
    if (rows > 65535 * 16) return q4_fail(ctx, LCSM_EINVAL, "too many rows");
  }
  if (ctx->faulted) return LCSM_ESTATE;
  if (!rows) return LCSM_OK;
  const size_t m = (size_t)layer, groups = (size_t)ctx->nts * ctx->ng * 16;
  const lcsm::Q4Call c{rows, s.N, s.K, s.group, ctx->ng, ctx->kb, s.scale_dtype, x,
                       ctx->codes + m * ctx->nts * ctx->kb * 1024,
                       ctx->scales + m * groups * lcsm::dtype_size(s.scale_dtype),
                       ctx->zeros ? ctx->zeros + m * groups : nullptr,
                       ctx->bias ? ctx->bias + m * s.N : nullptr, y, x_stride, y_stride};
  const hipError_t e = lcsm::with_dtype(dtype, [&](auto v) { return lcsm::launch_q4<decltype(v)>(c, ctx->stream); });
  return e == hipSuccess ? LCSM_OK : q4_fail(ctx, LCSM_EDEVICE, "product launch", e);
}

int lcsm_q4_quantize(const float* w, int rows, int K, int group, int scale_dtype, void* codes,
                     void* scales, void* stream) {
  if (rows < 0 || K < 1 || K > (1 << 24) || !group_ok(group) || !lcsm::dtype_ok(scale_dtype)) return LCSM_EINVAL;
  if (!rows) return LCSM_OK;
  if (!w || !codes || !scales) return LCSM_EINVAL;
  const int ng = (int)(((long long)K + group - 1) / group);
  // (a wave a group, up to what a grid holds; 64 lanes each, as blocks() counts)
  const size_t lanes = (size_t)rows * ng * 64;
  hipLaunchKernelGGL(lcsm::k_q4_quantize, dim3(lcsm::blocks(lanes)), dim3(256), 0, (hipStream_t)stream, w, rows, K,
                     group, ng, scale_dtype, (uint8_t*)codes, scales);
  return hipGetLastError() == hipSuccess ? LCSM_OK : LCSM_EDEVICE;
}

int lcsm_q4_reset(lcsm_q4* ctx) {
  if (!ctx) return LCSM_EINVAL;
  ctx->faulted = false;
  ctx->msg[0] = 0;
  return LCSM_OK;
}

void lcsm_q4_destroy(lcsm_q4* ctx) {
  if (!ctx) return;
  (void)hipStreamSynchronize(ctx->stream);
  if (ctx->owned) (void)hipFree(ctx->owned);
  delete ctx;
}

const char* lcsm_q4_last_error(const lcsm_q4* ctx) { return ctx ? ctx->msg : ""; }

}  // extern "C"
