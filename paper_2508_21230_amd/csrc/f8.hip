// Rows in 8-bit floating point with a power-of-two scale for each block of 128 coordinates, and products of them.
//
// The matrix cores of gfx950 take, with every step of 128 coordinates, one E8M0 scale byte per row and 32 coordinates.  A
// scale per 128 is the same byte four times over, so applying it costs no instruction, and the order of the coordinates
// within a step is free as long as both operands have the same one.
//
// Of eight 8-bit products that a lane supplies side by side, the matrix cores lose what lies below 2^-14 of the largest (between the
// eights 25 bits are kept).  A product of random rows is 1.5e-5 off by that, in norm: nothing beside the rounding to 16 bits (2e-4 for
// FP16, 1.7e-3 for BF16), so results of 16 bits are computed there; but 200 times FP32's own error.  FP32 results are computed from the
// same rows expanded to BF16 with their scale, which is exact (but for values below 2^-126, which BF16 holds to 2^-133), on the BF16 matrix cores,
// which sum in FP32 at half the rate.
#include "embed.h"

namespace {

typedef int int8v __attribute__((ext_vector_type(8)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef float float4v __attribute__((ext_vector_type(4)));

#define EJ_LDS(p) ((__attribute__((address_space(3))) void*)(p))
#define EJ_GLB(p) ((const __attribute__((address_space(1))) void*)(p))

constexpr int BLOCK = 128;  // coordinates that share a scale, and of one matrix-core step
constexpr int NUM_XCD = 8;

inline int64_t f8_blocks(int64_t d) { return (d + BLOCK - 1) / BLOCK; }

// ------------------------------------------------------------------------------------------
// Quantisation
// ------------------------------------------------------------------------------------------
// Magnitude for the maximum of a block: the bits of |x|, 0 for Inf and NaN.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}

// Scale byte of a block whose largest magnitude has these bits.  The formats' largest values are 1.75 * 2^8 and 1.75 * 2^15: the
// exponent of the maximum less 8 or 15, one more where its mantissa is above 1.75.
template <int FMT>
__device__ __forceinline__ uint32_t scale_byte(uint32_t max_bits) {
  if (max_bits == 0) return 127u;
  const int e = (int)(max_bits >> 23) - (FMT == EJOIN_E4M3 ? 8 : 15) + ((max_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return e < 0 ? 0u : (uint32_t)e;
}
// 2^-e of a scale byte e + 127 (0 .. 247).
__device__ __forceinline__ float inverse_scale(uint32_t byte) { return __builtin_bit_cast(float, (254u - byte) << 23); }

// Four scaled values as bytes.
template <int FMT>
__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
  if (FMT == EJOIN_E4M3) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
  }
  const int lo = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(c, d, lo, true);
}

// Eight values of a block with this scale byte, scaled, as bytes.  The largest FP32 values, above 1.9375 * 2^127, would round up to 2^128, which is
// no FP32 value and an infinity to whatever expands the rows: they are held as the format's value below it.
template <int FMT>
__device__ __forceinline__ uint2 scaled8(const float (&x)[8], uint32_t byte) {
  constexpr uint32_t TOP = FMT == EJOIN_E4M3 ? 247u : 240u;
  constexpr float MOST_AT_TOP = FMT == EJOIN_E4M3 ? 240.f : 28672.f;
  const float f = inverse_scale(byte);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i] * f;
  if (__builtin_expect(byte == TOP, 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (fabsf(y[i]) > MOST_AT_TOP && fabsf(y[i]) < INFINITY) y[i] = copysignf(MOST_AT_TOP, y[i]);
  }
  return {pack4<FMT>(y[0], y[1], y[2], y[3]), pack4<FMT>(y[4], y[5], y[6], y[7])};
}

struct QuantArgs {
  const void* X;
  int64_t n, d, ldx;
  int64_t first;    // row that the launch begins with (k_quantize_rows)
  uint32_t blocks;  // of a row
  uint8_t* rows;
  uint8_t* row_scales;
  int64_t ld_rows, ld_row_scales;
  uint8_t* cols;
  uint8_t* col_scales;
  int64_t ld_cols, ld_col_scales;
};

// Bytes past the last block of a row's scales.
__device__ __forceinline__ void pad_scales(uint8_t* scales, int64_t blocks) {
  for (int64_t b = blocks; (b & 3) != 0; ++b) scales[b] = 127;
}

typedef short short2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Eight neighbours of a row as they are in memory, 16-bit ones two to a word.  Maxima are taken of the bits of magnitudes, in words of as many;
// two values at a time are scaled and rounded by one instruction, which divides by the scale it is given.
template <typename T>
struct Octet {
  static constexpr int N = (int)sizeof(T) * 2;
  static constexpr uint32_t INF = sizeof(T) == 4 ? 0x7F800000u : (Element<T>::type == EJOIN_F16 ? 0x7C00u : 0x7F80u);  // bits of infinity
  uint32_t w[N];

  __device__ __forceinline__ void load(const T* p, int64_t left) {
    if (left >= 8) {
      struct __attribute__((packed, aligned(sizeof(T)))) At { uint32_t w[N]; };
      const At x = *reinterpret_cast<const At*>(p);
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = x.w[i];
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (sizeof(T) == 4) {
          w[i] = i < left ? __builtin_bit_cast(uint32_t, p[i]) : 0u;
        } else {
          const uint32_t lo = 2 * i < left ? __builtin_bit_cast(uint16_t, p[2 * i]) : 0u, hi = 2 * i + 1 < left ? __builtin_bit_cast(uint16_t, p[2 * i + 1]) : 0u;
          w[i] = lo | hi << 16;
        }
      }
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = 0;
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
    else return Element<T>::get(__builtin_bit_cast(T, (uint16_t)(w[i >> 1] >> (16 * (i & 1)))));
  }
  // Half h of a word, of 16-bit values.
  static __device__ __forceinline__ float value(uint32_t word, int h) {
    if constexpr (sizeof(T) == 4) return 0.f;
    else return Element<T>::get(__builtin_bit_cast(T, (uint16_t)(word >> (16 * h))));
  }
  // Keeps the long way's conversions out of the short one's registers.
  __device__ __forceinline__ void pin() {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+v"(w[i]));
  }
  static __device__ __forceinline__ uint32_t magnitude(uint32_t x) { return x & (sizeof(T) == 4 ? 0x7FFFFFFFu : 0x7FFF7FFFu); }
  static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {
    if constexpr (sizeof(T) == 4) {
      return max(a, b);
    } else {
      typedef unsigned short Two __attribute__((ext_vector_type(2)));
      return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(Two, a), __builtin_bit_cast(Two, b)));
    }
  }
  // Largest magnitudes of the words, each half of its own.
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = magnitude(w[0]);
#pragma unroll
    for (int i = 1; i < N; ++i) m = larger(m, magnitude(w[i]));
    return m;
  }
  // The bits of a magnitude (the larger of a word's halves) in FP32; infinity's or NaN's stay such.
  static __device__ __forceinline__ uint32_t widen(uint32_t m) {
    if constexpr (sizeof(T) == 4) {
      return m;
    } else {
      m = max(m & 0xFFFFu, m >> 16);
      if constexpr (Element<T>::type == EJOIN_F16) return __builtin_bit_cast(uint32_t, Element<f16>::get(__builtin_bit_cast(f16, (uint16_t)m)));
      else return m << 16;
    }
  }
};

// Maximum over 16 lanes.
template <typename T>
__device__ __forceinline__ uint32_t largest_of_16(uint32_t m) {
  m = Octet<T>::larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x128, 0xF, 0xF, true));  // row_ror:8, 4, 2, 1
  m = Octet<T>::larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x124, 0xF, 0xF, true));
  m = Octet<T>::larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x122, 0xF, 0xF, true));
  return Octet<T>::larger(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x121, 0xF, 0xF, true));
}

// Whether a block with this maximum (FP32 bits) takes the long way: values that are not finite are to be left out of the maximum, values above
// 1.75 * 2^127 may be too large (see scaled8), and the scale of the smallest blocks is no normal number.
__device__ __forceinline__ bool unusual(uint32_t max_bits, uint32_t byte) { return max_bits > 0x7F600000u || byte == 0; }

// Two values of a pair of words (16 bits) or two words (FP32), scaled, into the lower or upper half of q.
template <int FMT, typename T, bool HIGH>
__device__ __forceinline__ uint32_t scaled2(uint32_t q, uint32_t a, uint32_t b, float scale) {
  const short2v old = __builtin_bit_cast(short2v, q);
  short2v r;
  if constexpr (sizeof(T) == 4) {
    const float x = __builtin_bit_cast(float, a), y = __builtin_bit_cast(float, b);
    r = FMT == EJOIN_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(old, x, y, scale, HIGH) : __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(old, x, y, scale, HIGH);
  } else if constexpr (Element<T>::type == EJOIN_F16) {
    const f16x2 x = __builtin_bit_cast(f16x2, a);
    r = FMT == EJOIN_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(old, x, scale, HIGH) : __builtin_amdgcn_cvt_scalef32_pk_bf8_f16(old, x, scale, HIGH);
  } else {
    const bf16x2 x = __builtin_bit_cast(bf16x2, a);
    r = FMT == EJOIN_E4M3 ? __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(old, x, scale, HIGH) : __builtin_amdgcn_cvt_scalef32_pk_bf8_bf16(old, x, scale, HIGH);
  }
  return __builtin_bit_cast(uint32_t, r);
}

// Rows only: sixteen lanes a row's block, eight coordinates a lane, QUANT_ROWS rows a lane, whose loads are under way together.  Bound by the
// memory: 100,000 x 960 FP16 (289 MB read and written) 50 us, 5.8 TB/s, part of it from the memory-side cache; 50,021 x 384 FP32 16 us.
constexpr int QUANT_ROWS = 4;
template <typename T, int FMT>
__global__ __launch_bounds__(256) void k_quantize_rows(const QuantArgs a) {
  const uint32_t group = blockIdx.x / a.blocks, block = blockIdx.x - group * a.blocks, lane = threadIdx.x & 15;
  const int64_t row0 = a.first + (int64_t)group * (16 * QUANT_ROWS) + (threadIdx.x >> 4), at = (int64_t)block * BLOCK + lane * 8;
  Octet<T> x[QUANT_ROWS];
#pragma unroll
  for (int i = 0; i < QUANT_ROWS; ++i) {
    if (row0 + 16 * i < a.n) x[i].load(static_cast<const T*>(a.X) + (row0 + 16 * i) * a.ldx + at, a.d - at);
    else x[i].clear();
  }
#pragma unroll
  for (int i = 0; i < QUANT_ROWS; ++i) {
    const int64_t row = row0 + 16 * i;
    uint32_t m = Octet<T>::widen(largest_of_16<T>(x[i].largest())), byte = scale_byte<FMT>(m);
    uint2 q{0, 0};
    if (unusual(m, byte)) {
      x[i].pin();
      m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, finite_bits(x[i].get(j)));
      m = largest_of_16<float>(m);
      byte = scale_byte<FMT>(m);
      float y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = x[i].get(j);
      q = scaled8<FMT>(y, byte);
    } else {
      const float f = __builtin_bit_cast(float, byte << 23);
      constexpr int S = sizeof(T) == 4 ? 2 : 1;  // words of a pair
      q.x = scaled2<FMT, T, true>(scaled2<FMT, T, false>(0, x[i].w[0], x[i].w[S - 1], f), x[i].w[S], x[i].w[2 * S - 1], f);
      q.y = scaled2<FMT, T, true>(scaled2<FMT, T, false>(0, x[i].w[2 * S], x[i].w[3 * S - 1], f), x[i].w[3 * S], x[i].w[4 * S - 1], f);
    }
    if (row < a.n) {
      *reinterpret_cast<uint2*>(a.rows + row * a.ld_rows + at) = q;
      if (lane == 0) {
        uint8_t* s = a.row_scales + row * a.ld_row_scales;
        s[block] = (uint8_t)byte;
        if (block == a.blocks - 1) pad_scales(s, a.blocks);
      }
    }
  }
}

// Columns, or both: a tile of 128 x 128 a workgroup, held in registers: 16 lanes across (eight columns each), 16 thread rows of eight
// rows each.  The transposed bytes go out by way of the LDS, whose columns stand TSTRIDE bytes apart.  One read of X serves both results;
// bound by the memory: 4,096 x 50,021 BF16 into both (819 MB) 175 us, 4.7 TB/s.
constexpr int TSTRIDE = 136;
template <typename T, int FMT, bool ROWS>
__global__ __launch_bounds__(256) void k_quantize_tile(const QuantArgs a) {
  constexpr int W = Octet<T>::N, PER = sizeof(T) == 4 ? 1 : 2;  // words of eight columns, columns of a word
  __shared__ uint32_t col_max[4][16 * W];
  __shared__ __align__(16) uint8_t turned[BLOCK * TSTRIDE];
  const uint32_t row_tile = blockIdx.x / a.blocks, col_tile = blockIdx.x - row_tile * a.blocks;
  const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = threadIdx.x >> 6;
  const int64_t r0 = (int64_t)row_tile * BLOCK + rg * 8, c0 = (int64_t)col_tile * BLOCK + cg * 8;
  Octet<T> x[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (r0 + i < a.n) x[i].load(static_cast<const T*>(a.X) + (r0 + i) * a.ldx + c0, a.d - c0);
    else x[i].clear();
  }
  // columns' maxima: over the thread's rows, over the wavefront's four thread rows, over the wavefronts
#pragma unroll
  for (int j = 0; j < W; ++j) {
    uint32_t m = Octet<T>::magnitude(x[0].w[j]);
#pragma unroll
    for (int i = 1; i < 8; ++i) m = Octet<T>::larger(m, Octet<T>::magnitude(x[i].w[j]));
    m = Octet<T>::larger(m, (uint32_t)__shfl_xor((int)m, 16));
    m = Octet<T>::larger(m, (uint32_t)__shfl_xor((int)m, 32));
    if ((threadIdx.x & 48) == 0) col_max[wave][cg * W + j] = m;
  }
  constexpr int S = sizeof(T) == 4 ? 2 : 1;
  if (ROWS) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      uint32_t m = Octet<T>::widen(largest_of_16<T>(x[i].largest())), byte = scale_byte<FMT>(m);
      uint2 q{0, 0};
      if (unusual(m, byte)) {
        x[i].pin();
        m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, finite_bits(x[i].get(j)));
        m = largest_of_16<float>(m);
        byte = scale_byte<FMT>(m);
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[i].get(j);
        q = scaled8<FMT>(y, byte);
      } else {
        const float f = __builtin_bit_cast(float, byte << 23);
        q.x = scaled2<FMT, T, true>(scaled2<FMT, T, false>(0, x[i].w[0], x[i].w[S - 1], f), x[i].w[S], x[i].w[2 * S - 1], f);
        q.y = scaled2<FMT, T, true>(scaled2<FMT, T, false>(0, x[i].w[2 * S], x[i].w[3 * S - 1], f), x[i].w[3 * S], x[i].w[4 * S - 1], f);
      }
      if (r0 + i < a.n) {
        *reinterpret_cast<uint2*>(a.rows + (r0 + i) * a.ld_rows + c0) = q;
        if (cg == 0) {
          uint8_t* s = a.row_scales + (r0 + i) * a.ld_row_scales;
          s[col_tile] = (uint8_t)byte;
          if (col_tile == a.blocks - 1) pad_scales(s, a.blocks);
        }
      }
    }
  }
  __syncthreads();
  const int64_t col_blocks = (a.n + BLOCK - 1) / BLOCK;
  bool odd = false;  // one of the thread's columns takes the long way: they all do, after the maxima of the tile's finite values are known
  uint32_t both[W];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    const int k = cg * W + j;
    both[j] = Octet<T>::larger(Octet<T>::larger(col_max[0][k], col_max[1][k]), Octet<T>::larger(col_max[2][k], col_max[3][k]));
#pragma unroll
    for (int h = 0; h < PER; ++h) {
      const uint32_t m = Octet<T>::widen(PER == 1 ? both[j] : (both[j] >> (16 * h)) & 0xFFFFu);
      odd |= unusual(m, scale_byte<FMT>(m));
    }
  }
  const bool any_odd = __syncthreads_or(odd);
  uint32_t* finite = reinterpret_cast<uint32_t*>(turned);  // (before the bytes are put there)
  if (any_odd) {
    if (threadIdx.x < BLOCK) finite[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, finite_bits(x[i].get(j)));
      atomicMax(&finite[cg * 8 + j], m);
    }
    __syncthreads();
  }
  auto put_column = [&](int j, uint2 q, uint32_t byte) {
    *reinterpret_cast<uint2*>(turned + (cg * 8 + j) * TSTRIDE + rg * 8) = q;
    if (rg == 0 && c0 + j < a.d) {
      uint8_t* s = a.col_scales + (c0 + j) * a.ld_col_scales;
      s[row_tile] = (uint8_t)byte;
      if (row_tile == col_blocks - 1) pad_scales(s, col_blocks);
    }
  };
  if (any_odd) {
    uint32_t exact[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) exact[j] = finite[cg * 8 + j];
    __syncthreads();
#pragma unroll 1
    for (int h = 0; h < PER; ++h) {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = PER == 1 ? __builtin_bit_cast(float, x[i].w[j]) : Octet<T>::value(x[i].w[j], h);
        const uint32_t byte = scale_byte<FMT>(PER == 1 ? exact[j] : (h ? exact[2 * j + 1 < 8 ? 2 * j + 1 : 0] : exact[2 * j < 8 ? 2 * j : 0]));
        put_column(PER * j + h, scaled8<FMT>(y, byte), byte);
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      uint2 q{0, 0};
      const uint32_t byte = scale_byte<FMT>(Octet<T>::widen(PER == 1 ? both[j / PER] : (both[j / PER] >> (16 * (j & 1))) & 0xFFFFu));
      const float f = __builtin_bit_cast(float, byte << 23);
      if constexpr (sizeof(T) == 4) {
        q.x = scaled2<FMT, T, true>(scaled2<FMT, T, false>(0, x[0].w[j], x[1].w[j], f), x[2].w[j], x[3].w[j], f);
        q.y = scaled2<FMT, T, true>(scaled2<FMT, T, false>(0, x[4].w[j], x[5].w[j], f), x[6].w[j], x[7].w[j], f);
      } else {
        const uint32_t half = j & 1 ? 0x07060302u : 0x05040100u;  // of two rows' words
        auto pair = [&](int i) { return __builtin_amdgcn_perm(x[i + 1].w[j >> 1], x[i].w[j >> 1], half); };
        q.x = scaled2<FMT, T, true>(scaled2<FMT, T, false>(0, pair(0), 0, f), pair(2), 0, f);
        q.y = scaled2<FMT, T, true>(scaled2<FMT, T, false>(0, pair(4), 0, f), pair(6), 0, f);
      }
      put_column(j, q, byte);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = rg + 16 * i;
    if ((int64_t)col_tile * BLOCK + c < a.d)
      *reinterpret_cast<uint2*>(a.cols + ((int64_t)col_tile * BLOCK + c) * a.ld_cols + (int64_t)row_tile * BLOCK + cg * 8) =
          *reinterpret_cast<const uint2*>(turned + c * TSTRIDE + cg * 8);
  }
}

// ------------------------------------------------------------------------------------------
// Product
// ------------------------------------------------------------------------------------------
// A workgroup computes tiles of 256 (rows of A) x 64 WN (rows of B) with 2 x WN wavefronts, 128 x 64 each, one tile after the other without a
// pause: the panels of a slice of 64 coordinates are copied straight into a ring of LDS stages, all but one of them ahead, past the end of a
// tile into the next, and the results are stored while the next tile's slices arrive.  The rows of B are the matrix cores' first operand, so
// that a lane's results of a step are neighbours in a row of C.
// WN = 4: eight wavefronts, four stages of 32 KB, one workgroup a CU.  WN = 2: four wavefronts, three stages of 24 KB, two workgroups a CU, of which
// one computes while the other waits; half as much again has to be copied for the same work.
// A wavefront's 128 x 64 results are the largest that its registers hold: 85 operations for each byte that it reads from the LDS.
// The tiles of an XCD are neighbours, GROUP_ROWS row tiles at a time, so that panels are fetched into its L2 once.
constexpr int TILE = 256;              // rows of A
constexpr int SLICE = 64;              // coordinates, bytes
constexpr int GROUP_ROWS = 4;          // row tiles that are gone through together, column by column, so that their panels stay in an XCD's L2
template <int WM, int WN>
struct Shape {
  static constexpr int COLS = 64 * WN, WAVES = WM * WN, STAGES = COLS == 256 ? 4 : 3, AHEAD = STAGES - 1;
  static constexpr int PANEL = TILE * SLICE, STAGE = PANEL + COLS * SLICE;  // bytes: A's panel, both
  static constexpr int COPIES_A = TILE / 16 / WAVES, COPIES_B = COLS / 16 / WAVES, COPIES = COPIES_A + COPIES_B;  // copy instructions of a wavefront and slice, of 16 rows each
  static constexpr int SCALES = (TILE + COLS) * 4;  // bytes: a dword a row, of four blocks
  static constexpr int LDS = STAGES * STAGE + 2 * SCALES;
  static constexpr int PER_CU = COLS == 256 ? 1 : 2;
};

struct ProductArgs {
  const uint8_t* A;
  const uint8_t* B;
  const uint8_t* sA;
  const uint8_t* sB;
  int64_t lda, ldb, lsa, lsb;
  int64_t m, n;
  int32_t blocks;      // k-blocks
  int32_t per_split;   // k-blocks of a split, a multiple of four
  uint32_t tiles_m, tiles_n;
  uint32_t count;      // tiles
  uint32_t tiles;      // of all splits
  uint32_t per_xcd;    // tiles that the workgroups of an XCD share
  float scale;
  void* C;
  int64_t ldc;
  float* parts;        // results of the splits, tile by tile (dense); null without splits
};

// 16-byte chunk (of four) of an LDS row that holds chunk c of the row's 64 bytes: c ^ swizzle(row).  The sixteen lanes that read together
// read chunk c of sixteen neighbouring rows, in whatever order: those fill the 64 banks once.
__device__ __forceinline__ int swizzle(int row) { return (row >> 2) & 3; }

// One copy of 64 lanes x 16 (or 4) bytes, from base + offset to LDS address at + 16 (4) * lane; base and at are uniform.  In assembly, as for the
// builtin the compiler waits for all copies under way before it reads the LDS; here they are waited for by count.
__device__ __forceinline__ void copy16(uint32_t at, const void* base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(at), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void copy4(uint32_t at, const void* base, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(at), "v"(offset), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
  const uint64_t b = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)b), hi = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
  return reinterpret_cast<const uint8_t*>(((uint64_t)hi << 32) | lo);
}

// Sixteen 8-bit values of a row times their block's scale, in BF16: exact (the instruction takes the scale's exponent).
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
struct Sixteen {
  bf16x8 half[2];
};
template <int FMT>
__device__ __forceinline__ Sixteen expand(int4v x, float scale) {
  Sixteen r;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    bf16x2 lo, hi;
    if (FMT == EJOIN_E4M3) {
      lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)x[w], scale, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)x[w], scale, true);
    } else {
      lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((uint32_t)x[w], scale, false);
      hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8((uint32_t)x[w], scale, true);
    }
    r.half[w >> 1][(w & 1) * 4 + 0] = lo[0];
    r.half[w >> 1][(w & 1) * 4 + 1] = lo[1];
    r.half[w >> 1][(w & 1) * 4 + 2] = hi[0];
    r.half[w >> 1][(w & 1) * 4 + 3] = hi[1];
  }
  return r;
}
// 2^e of a scale byte e + 127 in the low bits of x.
__device__ __forceinline__ float scale_of(uint32_t x) {
  const uint32_t b = (x & 255u) << 23;
  return __builtin_bit_cast(float, b ? b : 0x400000u);
}

// Stores of whole 128-byte lines: a wavefront's store instruction writes eight rows of them.  Sixteen bytes x and y of a lane's row, r16 = lane % 16, go
// to different halves of a line; afterwards x holds rows r16 % 8, y rows r16 % 8 + 8, each lane the half r16 / 8.
__device__ __forceinline__ void exchange_halves(uint32_t& x, uint32_t& y) {
  const uint32_t a = x, b = y;
  x = (uint32_t)__builtin_amdgcn_update_dpp((int)a, (int)b, 0x128 /* row_ror:8 */, 0xF, 0xC, false);  // lanes 8 .. 15 of 16: y of lanes 0 .. 7
  y = (uint32_t)__builtin_amdgcn_update_dpp((int)b, (int)a, 0x128, 0xF, 0x3, false);                 // lanes 0 .. 7: x of lanes 8 .. 15
}
// Of four times sixteen lanes, the odd ones of x exchanged with the even ones of y.
__device__ __forceinline__ void exchange_rows(uint32_t& x, uint32_t& y) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
  x = r[0];
  y = r[1];
}
struct Line16 {
  uint32_t w[4];
};
// Two results in a word.
template <typename OUT>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef float Two __attribute__((ext_vector_type(2)));
  typedef OUT Out __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(Two{a, b}, Out));
}
// Sixteen bytes to any address, past the caches: results as large as these are not read again from there (4,096 x 50,021 x 384: 159 us through them, 137 past).
__device__ __forceinline__ void put16(void* p, const Line16& x) {
  typedef uint32_t Words __attribute__((ext_vector_type(4), aligned(2)));
  __builtin_nontemporal_store(__builtin_bit_cast(Words, x), static_cast<Words*>(p));
}
template <typename OUT>
__device__ __forceinline__ void store_some(OUT* c, int64_t left, const Line16& x) {
  constexpr int N = 16 / (int)sizeof(OUT);
  if (left >= N) {
    put16(c, x);
  } else {
    struct { OUT v[N]; } y;
    memcpy(&y, &x, 16);
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) c[e] = y.v[e];
  }
}

// Where a tile lies: split, first row of A and of B, k-blocks.
template <int COLS>
struct TilePlace {
  int64_t m0, n0;
  uint32_t part;
  int split, k0, k1;
  __device__ __forceinline__ TilePlace(const ProductArgs& a, uint32_t t) {
    const uint32_t in = t % a.count;
    split = t / a.count;
    part = t;
    const uint32_t first = in / (GROUP_ROWS * a.tiles_n) * GROUP_ROWS, high = min((uint32_t)GROUP_ROWS, a.tiles_m - first), r = in - first * a.tiles_n;
    m0 = (int64_t)(first + r % high) * TILE;
    n0 = (int64_t)(r / high) * COLS;
    k0 = split * a.per_split;
    k1 = min(a.blocks, k0 + a.per_split);
  }
};

// A wavefront's 128 x 64 results.  On the 8-bit matrix cores: steps of 32 x 32 x 64.  A lane (r, h) = (lane % 32, lane / 32) feeds chunks 2 h and
// 2 h + 1 of a row and gets rows 8 v + 4 h .. + 3 of B (v = 0 .. 3), row r of A; so that they are two times eight neighbours, lane r feeds the row
// of B that is r with bits 2 and 3 exchanged.
template <int FA, int FB, typename OUT, int MI>
struct WaveTile8 {
  typedef float float16v __attribute__((ext_vector_type(16)));
  static constexpr int STORES = 4 * MI;
  float16v acc[MI][2];
  uint32_t sa[MI], sb[2];
  int a_at, b_at;
  __device__ __forceinline__ WaveTile8(int wm, int wn, int lane) {
    const int r = lane & 31, h = lane >> 5, rb = (r & 19) | ((r & 8) >> 1) | ((r & 4) << 1);
    a_at = (wm * (32 * MI) + r) * SLICE + (((2 * h) ^ swizzle(r)) << 4);
    b_at = TILE * SLICE + (wn * 64 + rb) * SLICE + (((2 * h) ^ swizzle(rb)) << 4);
    sa_at = (wm * (32 * MI) + r) * 4;
    sb_at = (TILE + wn * 64 + rb) * 4;
  }
  int sa_at, sb_at;
  __device__ __forceinline__ void scales(const uint8_t* s) {
#pragma unroll
    for (int i = 0; i < MI; ++i) sa[i] = *reinterpret_cast<const uint32_t*>(s + sa_at + i * 128);
#pragma unroll
    for (int j = 0; j < 2; ++j) sb[j] = *reinterpret_cast<const uint32_t*>(s + sb_at + j * 128);
  }
  __device__ __forceinline__ void next_block() {
#pragma unroll
    for (int i = 0; i < MI; ++i) sa[i] >>= 8;
#pragma unroll
    for (int j = 0; j < 2; ++j) sb[j] >>= 8;
  }
  // Operands of the slice to be multiplied; those of B for the slice after it too, those of A take the places of the ones that are done with.
  int8v fa[MI], fb[2], fb_next[2];
  __device__ __forceinline__ int8v a_of(const uint8_t* stage, int i) const { return lds_chunks(stage + a_at + i * 32 * SLICE, stage + (a_at ^ 16) + i * 32 * SLICE); }
  __device__ __forceinline__ int8v b_of(const uint8_t* stage, int j) const { return lds_chunks(stage + b_at + j * 32 * SLICE, stage + (b_at ^ 16) + j * 32 * SLICE); }
  __device__ __forceinline__ void read(const uint8_t* stage) {
#pragma unroll
    for (int j = 0; j < 2; ++j) fb[j] = b_of(stage, j);
#pragma unroll
    for (int i = 0; i < MI; ++i) fa[i] = a_of(stage, i);
  }
  template <bool FIRST>
  __device__ __forceinline__ void multiply(const uint8_t* next_stage) {
#pragma unroll
    for (int j = 0; j < 2; ++j) fb_next[j] = b_of(next_stage, j);
#pragma unroll
    for (int i = 0; i < MI; ++i) {
#pragma unroll
      for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb[j], fa[i], FIRST ? float16v{} : acc[i][j], FB, FA, 0, (int)sb[j], 0, (int)sa[i]);
      fa[i] = a_of(next_stage, i);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) fb[j] = fb_next[j];
  }
  // After two exchanges a lane has eight neighbours of rows 32 i + 8 q + lane % 8, q = 0 .. 3.
  template <bool WHOLE, typename PLACE>
  __device__ __forceinline__ void store(const ProductArgs& a, const PLACE& p, int wm, int wn, int lane) {
    const int64_t row = p.m0 + wm * (32 * MI) + (lane & 7), col = p.n0 + wn * 64 + ((lane >> 4) & 1) * 32 + ((lane >> 3) & 1) * 16 + (lane >> 5) * 8, left = a.n - col;
    OUT* c = static_cast<OUT*>(a.C) + row * a.ldc + col;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      Line16 x[2][2];  // of j and u
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int e = 0; e < 4; ++e) x[j][u].w[e] = pack2<OUT>(acc[i][j][u * 8 + 2 * e] * a.scale, acc[i][j][u * 8 + 2 * e + 1] * a.scale);
        }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        exchange_rows(x[0][0].w[e], x[1][0].w[e]);  // x[0]: rows 0 .. 15 of both j, x[1]: rows 16 .. 31
        exchange_rows(x[0][1].w[e], x[1][1].w[e]);
        exchange_halves(x[0][0].w[e], x[0][1].w[e]);
        exchange_halves(x[1][0].w[e], x[1][1].w[e]);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (WHOLE) put16(c, x[q >> 1][q & 1]);
        else if (row + 32 * i + 8 * q < a.m) store_some(c, left, x[q >> 1][q & 1]);
        c += 8 * a.ldc;
      }
    }
  }
  static __device__ __forceinline__ int8v lds_chunks(const uint8_t* p, const uint8_t* q) {
    const int4v lo = *reinterpret_cast<const int4v*>(p), hi = *reinterpret_cast<const int4v*>(q);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};

// On the BF16 matrix cores: steps of 16 x 16 x 32, two of a lane's 16 bytes.  FP32 results only.
template <int FA, int FB, int COLS>
struct WaveTile16 {
  static constexpr int STORES = 32;
  float4v acc[8][4];
  uint32_t sa[8], sb[4];
  int a_at, b_at, sa_at, sb_at;
  __device__ __forceinline__ WaveTile16(int wm, int wn, int lane) {
    const int r = lane & 15, g = lane >> 4;
    a_at = (wm * 128 + r) * SLICE + ((g ^ swizzle(r)) << 4);
    b_at = TILE * SLICE + (wn * 64 + r) * SLICE + ((g ^ swizzle(r)) << 4);
    sa_at = (wm * 128 + r) * 4;
    sb_at = (TILE + wn * 64 + r) * 4;
  }
  __device__ __forceinline__ void scales(const uint8_t* s) {
#pragma unroll
    for (int i = 0; i < 8; ++i) sa[i] = *reinterpret_cast<const uint32_t*>(s + sa_at + i * 64);
#pragma unroll
    for (int j = 0; j < 4; ++j) sb[j] = *reinterpret_cast<const uint32_t*>(s + sb_at + j * 64);
  }
  __device__ __forceinline__ void next_block() {
#pragma unroll
    for (int i = 0; i < 8; ++i) sa[i] >>= 8;
#pragma unroll
    for (int j = 0; j < 4; ++j) sb[j] >>= 8;
  }
  template <bool FIRST>
  __device__ __forceinline__ void slice(const uint8_t* stage) {
    Sixteen fb[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) fb[j] = expand<FB>(*reinterpret_cast<const int4v*>(stage + b_at + j * 16 * SLICE), scale_of(sb[j]));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const Sixteen fa = expand<FA>(*reinterpret_cast<const int4v*>(stage + a_at + i * 16 * SLICE), scale_of(sa[i]));
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j].half[q], fa.half[q], FIRST && q == 0 ? float4v{} : acc[i][j], 0, 0, 0);
    }
  }
  template <bool WHOLE, typename PLACE>
  __device__ __forceinline__ void store(const ProductArgs& a, const PLACE& p, int wm, int wn, int lane) {
    const int r = wm * 128 + (lane & 7), c0 = wn * 64 + ((lane >> 3) & 1) * 16 + (lane >> 4) * 4;
    const int64_t row = p.m0 + r, left = a.n - (p.n0 + c0), ldc = a.parts ? COLS : a.ldc;
    float* c = a.parts ? a.parts + (int64_t)p.part * (TILE * COLS) + r * COLS + c0 : static_cast<float*>(a.C) + row * ldc + p.n0 + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        Line16 x, y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x.w[e] = __builtin_bit_cast(uint32_t, acc[i][j][e] * a.scale);
          y.w[e] = __builtin_bit_cast(uint32_t, acc[i][j + 1][e] * a.scale);
          exchange_halves(x.w[e], y.w[e]);
        }
        if (WHOLE) {
          put16(c + 16 * j, x);
          put16(c + 8 * ldc + 16 * j, y);
        } else {
          if (row + 16 * i < a.m) store_some(c + 16 * j, left - 16 * j, x);
          if (row + 16 * i + 8 < a.m) store_some(c + 8 * ldc + 16 * j, left - 16 * j, y);
        }
      }
      c += 16 * ldc;
    }
  }
};

// What a workgroup's copies bring, slice after slice of tile after tile.  A wavefront brings its share of each panel, 16 rows at a time, and the scales
// of 64 rows of A, of B, or of both.  Rows past the end are the last one again.  Everything here is uniform but the offsets within a panel.
template <typename L>
struct Copies {
  const ProductArgs& a;
  const uint32_t lds0, end, slots;
  const int lane, wave;
  const bool brings_sa, brings_sb;
  uint32_t t, stage = 0, scale_buffer = 0;
  int slice = 0, slices = 0;
  int ahead = 0;  // slices under way or waiting in the ring
  const uint8_t* pa = nullptr;
  const uint8_t* pb = nullptr;
  const uint8_t* psa = nullptr;
  const uint8_t* psb = nullptr;
  uint32_t va[L::COPIES_A], vb[L::COPIES_B], vsa = 0, vsb = 0;

  __device__ __forceinline__ Copies(const ProductArgs& a_, uint32_t lds0_, uint32_t t_, uint32_t end_, uint32_t slots_, int lane_, int wave_)
      : a(a_), lds0(lds0_), end(end_), slots(slots_), lane(lane_), wave(wave_), brings_sa(wave_ < 4),
        brings_sb(L::WAVES == 8 ? wave_ >= 4 && wave_ < 4 + L::COLS / 64 : wave_ < L::COLS / 64), t(t_) {}

  __device__ __forceinline__ void begin_tile() {
    const TilePlace<L::COLS> p(a, t);
    slice = 0;
    slices = 2 * (p.k1 - p.k0);
    pa = a.A + p.m0 * a.lda + (int64_t)p.k0 * BLOCK;
    pb = a.B + p.n0 * a.ldb + (int64_t)p.k0 * BLOCK;
    psa = a.sA + p.m0 * a.lsa + p.k0;
    psb = a.sB + p.n0 * a.lsb + p.k0;
    const uint32_t last_a = (uint32_t)min((int64_t)TILE, a.m - p.m0) - 1, last_b = (uint32_t)min((int64_t)L::COLS, a.n - p.n0) - 1;
#pragma unroll
    for (int q = 0; q < L::COPIES_A; ++q) {
      const uint32_t row = (wave * L::COPIES_A + q) * 16 + (lane >> 2);
      va[q] = min(row, last_a) * (uint32_t)a.lda + (((lane & 3) ^ swizzle(row)) << 4);
    }
#pragma unroll
    for (int q = 0; q < L::COPIES_B; ++q) {
      const uint32_t row = (wave * L::COPIES_B + q) * 16 + (lane >> 2);
      vb[q] = min(row, last_b) * (uint32_t)a.ldb + (((lane & 3) ^ swizzle(row)) << 4);
    }
    const uint32_t row = (wave % 4) * 64 + lane;
    vsa = min(row, last_a) * (uint32_t)a.lsa;
    vsb = min(row, last_b) * (uint32_t)a.lsb;
  }
  __device__ __forceinline__ void issue() {
    if (slice == slices) {
      if (slices) t += slots;
      if (t >= end) return;
      begin_tile();
    }
    if ((slice & 7) == 0) {
      const uint32_t to = lds0 + L::STAGES * L::STAGE + scale_buffer * L::SCALES;
      if (brings_sa) copy4(to + (wave % 4) * 256, uniform(psa), vsa);
      if (brings_sb) copy4(to + TILE * 4 + (wave % 4) * 256, uniform(psb), vsb);
      psa += 4;
      psb += 4;
      scale_buffer ^= 1;
    }
    const uint32_t to = lds0 + stage * L::STAGE;
#pragma unroll
    for (int q = 0; q < L::COPIES_A; ++q) copy16(to + (wave * L::COPIES_A + q) * 16 * SLICE, uniform(pa), va[q]);
#pragma unroll
    for (int q = 0; q < L::COPIES_B; ++q) copy16(to + L::PANEL + (wave * L::COPIES_B + q) * 16 * SLICE, uniform(pb), vb[q]);
    pa += SLICE;
    pb += SLICE;
    stage = stage + 1 == L::STAGES ? 0 : stage + 1;
    ++slice;
    ++ahead;
  }
};

// 16-bit results: a slice's operands are read into registers while the slice before it is multiplied, so that the matrix cores need not wait for the LDS
// behind every barrier (8,192^3 without that: 475 us).  The stage that a slice was read from is free a slice earlier too.
// Bound by the matrix cores and the stores, which add up: 8,192 x 100,000 x 960 into BF16 907 us, 1.73 PFLOP/s (its 1.64 GB of results alone are 240 us
// of a large fill's rate; 8,192^3, where they are few, runs at 2.2 to 2.3 PFLOP/s); 4,096 x 50,021 x 384 122 us, of them 410 MB of results.
template <typename WAVE_TILE, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_f8_product_ahead(const ProductArgs a) {
  typedef Shape<WM, WN> L;
  typedef TilePlace<L::COLS> Place;
  extern __shared__ __align__(1024) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)EJ_LDS(lds)), slots = gridDim.x / NUM_XCD;
  const uint32_t end = min(a.tiles, (blockIdx.x % NUM_XCD + 1) * a.per_xcd);
  uint32_t t = blockIdx.x % NUM_XCD * a.per_xcd + blockIdx.x / NUM_XCD;
  if (t >= end) return;
  Copies<L> copies(a, lds0, t, end, slots, lane, wave);
#pragma unroll
  for (int q = 0; q < L::STAGES; ++q) copies.issue();

  WAVE_TILE w(wm, wn, lane);
  uint32_t stage = 0, scale_buffer = 0;
  int stored = 0;  // slices that were under way before the last tile's results were stored
  // The first slice.  In the loop: the slice after the one about to be multiplied is in the LDS once no more is under way than what was issued after
  // it, the copies of STAGES - 2 slices and the stores of a whole tile where that came in between; every wavefront is then past its reads of the
  // stage that the next copies go to.
  if (copies.ahead < L::STAGES) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  else asm volatile("s_waitcnt vmcnt(%0)" ::"n"((L::STAGES - 1) * L::COPIES) : "memory");
  asm volatile("s_barrier" ::: "memory");
  w.read(lds);
  for (; t < end; t += slots) {
    const Place p(a, t);
    const int slices = 2 * (p.k1 - p.k0);
    for (int s = 0; s < slices; ++s) {
      if ((s & 7) == 0) {
        w.scales(lds + L::STAGES * L::STAGE + scale_buffer * L::SCALES);
        scale_buffer ^= 1;
      } else if ((s & 1) == 0) {
        w.next_block();
      }
      --copies.ahead;  // (now the slices that were issued after this one)
      if (copies.ahead < L::STAGES - 1) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      else if (stored > 0) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((L::STAGES - 2) * L::COPIES + WAVE_TILE::STORES) : "memory");
      else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((L::STAGES - 2) * L::COPIES) : "memory");
      --stored;
      asm volatile("s_barrier" ::: "memory");
      copies.issue();
      stage = stage + 1 == L::STAGES ? 0 : stage + 1;
      if (s == 0) w.template multiply<true>(lds + stage * L::STAGE);  // (after the last slice of all, what is read from the stage is of no use)
      else w.template multiply<false>(lds + stage * L::STAGE);
    }
    if (p.m0 + TILE <= a.m && p.n0 + L::COLS <= a.n) {
      w.template store<true>(a, p, wm, wn, lane);
      stored = L::STAGES - 1;
    } else {
      w.template store<false>(a, p, wm, wn, lane);
      stored = 0;
    }
  }
}

// FP32 results: expanding the operands keeps the wavefronts busy, and their registers full; two workgroups a CU make up for each other's waits.
// Bound by the BF16 matrix cores with the expansion beside them: 4,096 x 384, k = 50,021 172 us, 50,021 x 384, k = 4,096 181 us: 0.92 and 0.87 PFLOP/s, where
// a large BF16 product of the library reaches 1.17.
template <typename WAVE_TILE, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_f8_product(const ProductArgs a) {
  typedef Shape<WM, WN> L;
  typedef TilePlace<L::COLS> Place;
  extern __shared__ __align__(1024) uint8_t lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)EJ_LDS(lds)), slots = gridDim.x / NUM_XCD;
  const uint32_t end = min(a.tiles, (blockIdx.x % NUM_XCD + 1) * a.per_xcd);
  uint32_t t = blockIdx.x % NUM_XCD * a.per_xcd + blockIdx.x / NUM_XCD;
  if (t >= end) return;
  Copies<L> copies(a, lds0, t, end, slots, lane, wave);
#pragma unroll
  for (int q = 0; q < L::AHEAD; ++q) copies.issue();

  WAVE_TILE w(wm, wn, lane);
  uint32_t stage = 0, scale_buffer = 0;
  int stored = 0;  // slices that were under way before the last tile's results were stored
  for (; t < end; t += slots) {
    const Place p(a, t);
    const int slices = 2 * (p.k1 - p.k0);
    for (int s = 0; s < slices; ++s) {
      // This slice is in the LDS once no more is under way than what was issued after it: the copies of the slices ahead of it, and the stores of
      // a whole tile where that came in between.  Reads of the stage that the next copies go to are done when every wavefront is here.
      --copies.ahead;
      if (copies.ahead < L::AHEAD - 1) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      else if (stored > 0) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((L::AHEAD - 1) * L::COPIES + WAVE_TILE::STORES) : "memory");
      else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((L::AHEAD - 1) * L::COPIES) : "memory");
      --stored;
      asm volatile("s_barrier" ::: "memory");
      copies.issue();
      if ((s & 7) == 0) {
        w.scales(lds + L::STAGES * L::STAGE + scale_buffer * L::SCALES);
        scale_buffer ^= 1;
      } else if ((s & 1) == 0) {
        w.next_block();
      }
      if (s == 0) w.template slice<true>(lds + stage * L::STAGE);
      else w.template slice<false>(lds + stage * L::STAGE);
      stage = stage + 1 == L::STAGES ? 0 : stage + 1;
    }
    if (a.parts || (p.m0 + TILE <= a.m && p.n0 + L::COLS <= a.n)) {
      w.template store<true>(a, p, wm, wn, lane);
      stored = L::AHEAD;
    } else {
      w.template store<false>(a, p, wm, wn, lane);
      stored = 0;
    }
  }
}

// ------------------------------------------------------------------------------------------
// Product with few rows of A: scores of query rows against a table
// ------------------------------------------------------------------------------------------
// What counts is that the table is read once, at the rate of the memory: 1 row against 100,000 of 384 (38.7 MB) 12.2 us, 33 against 200,011 of 200 24.5 us,
// where bringing in 33 rows for every workgroup is the rest (64 rows a workgroup and four wavefronts, half as many: 27 us).  The query rows, quantised by every workgroup for itself where
// they come as they are (that is less than a launch), stand in the LDS expanded to BF16, in the order in which the matrix cores take them;
// a wavefront takes 16 rows of the table at a time straight into registers, four k-blocks ahead, and expands them there.
constexpr int FEW_ROWS = 64;      // of A, in steps of 16
constexpr int FEW_LDS = 128 << 10;  // of their fragments: 4 KB for 16 rows and a k-block
constexpr int FEW_UNIT = 16;      // rows of B
constexpr int FEW_AHEAD = 4;      // k-blocks under way

struct FewArgs {
  // rows of A: elements of type `source` (EJOIN_F32 ...), or 8-bit ones (FEW_E4M3, FEW_E5M2) with their scales
  const void* A;
  const uint8_t* sA;
  int64_t lda, lsa;
  int32_t source;
  int32_t m, d, blocks;
  const uint8_t* B;
  const uint8_t* sB;
  int64_t ldb, lsb, n;
  float scale;
  void* C;
  int64_t ldc;
};
constexpr int FEW_E4M3 = 8, FEW_E5M2 = 9;

// Eight values with a scale in BF16.
template <int FMT>
__device__ __forceinline__ bf16x8 expand8(uint2 x, float scale) {
  const Sixteen r = expand<FMT>(int4v{(int)x.x, (int)x.y, 0, 0}, scale);
  return r.half[0];
}

// A in the LDS: sixteen lanes a row's k-block, FEW_FILL of them under way at a time.  Coordinates (h, g, q, 0 .. 7) of a block stand in
// fragment (h, q) at lane 16 g + row: a lane's 16 bytes of a row of B hold those of (h, g), q = 0 and 1.
constexpr int FEW_FILL = 4;
template <int MT>
__device__ __forceinline__ void few_put(uint8_t* lds, int row, int block, int lane16, bf16x8 x) {
  const int h = lane16 >> 3, q = lane16 & 1, at = ((lane16 & 7) >> 1) * 16 + (row & 15);
  *reinterpret_cast<bf16x8*>(lds + (((block * 4 + h * 2 + q) * MT + (row >> 4)) << 10) + at * 16) = x;
}
template <typename T, int MT>
__device__ __forceinline__ void few_fill(const FewArgs& a, uint8_t* lds) {  // from rows as they are
  const int lane16 = threadIdx.x & 15, groups = blockDim.x >> 4, units = a.m * a.blocks;
  for (int u0 = threadIdx.x >> 4; u0 < units; u0 += FEW_FILL * groups) {
    float x[FEW_FILL][8];
    int row[FEW_FILL], block[FEW_FILL];
#pragma unroll
    for (int i = 0; i < FEW_FILL; ++i) {
      const int u = min(u0 + i * groups, units - 1);  // (past the end: the last one again, with the same result)
      row[i] = u / a.blocks;
      block[i] = u - row[i] * a.blocks;
      const int k = block[i] * BLOCK + lane16 * 8, left = a.d - k;
      load8(static_cast<const T*>(a.A) + row[i] * a.lda + k, left < 0 ? 0 : (left < 8 ? left : 8), x[i]);
    }
#pragma unroll
    for (int i = 0; i < FEW_FILL; ++i) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) m = max(m, finite_bits(x[i][j]));
#pragma unroll
      for (int s = 1; s < 16; s <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, s));
      const uint32_t byte = scale_byte<EJOIN_E4M3>(m);
      const uint2 q = scaled8<EJOIN_E4M3>(x[i], byte);
      few_put<MT>(lds, row[i], block[i], lane16, expand8<EJOIN_E4M3>(q, scale_of(byte)));
    }
  }
}
template <int FMT, int MT>
__device__ __forceinline__ void few_fill_f8(const FewArgs& a, uint8_t* lds) {  // from 8-bit rows
  const int lane16 = threadIdx.x & 15, groups = blockDim.x >> 4, units = a.m * a.blocks;
  for (int u0 = threadIdx.x >> 4; u0 < units; u0 += FEW_FILL * groups) {
    uint2 x[FEW_FILL];
    uint32_t byte[FEW_FILL];
    int row[FEW_FILL], block[FEW_FILL];
#pragma unroll
    for (int i = 0; i < FEW_FILL; ++i) {
      const int u = min(u0 + i * groups, units - 1);
      row[i] = u / a.blocks;
      block[i] = u - row[i] * a.blocks;
      x[i] = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.A) + row[i] * a.lda + block[i] * BLOCK + lane16 * 8);
      byte[i] = a.sA[row[i] * a.lsa + block[i]];
    }
#pragma unroll
    for (int i = 0; i < FEW_FILL; ++i) few_put<MT>(lds, row[i], block[i], lane16, expand8<FMT>(x[i], scale_of(byte[i])));
  }
}

template <int FB, typename OUT, int MT>
__global__ __launch_bounds__(512, 4) void k_f8_few(const FewArgs a) {
  extern __shared__ __align__(1024) uint8_t lds[];
  const int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
  const int64_t units = (a.n + FEW_UNIT - 1) / FEW_UNIT, waves = (int64_t)gridDim.x * (blockDim.x >> 6);
  int64_t unit = (int64_t)blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6);
  const int64_t steps = unit < units ? ((units - 1 - unit) / waves + 1) * a.blocks : 0;  // k-blocks of all the wavefront's units
  // the next k-block to load, of which unit; the loads run FEW_AHEAD of them ahead of the products, past the end of a unit into the next
  int64_t next_unit = unit;
  int next = 0;
  int4v raw[FEW_AHEAD][2];
  uint32_t sb[FEW_AHEAD];
  auto load = [&](int o) {
    const int64_t row = min(next_unit * FEW_UNIT + r16, a.n - 1);  // (rows past the end are the last one)
    const uint8_t* p = a.B + row * a.ldb + (int64_t)next * BLOCK + g * 16;
    raw[o][0] = *reinterpret_cast<const int4v*>(p);
    raw[o][1] = *reinterpret_cast<const int4v*>(p + 64);
    sb[o] = a.sB[row * a.lsb + next];
    if (++next == a.blocks) next = 0, next_unit += waves;
  };
#pragma unroll
  for (int o = 0; o < FEW_AHEAD; ++o)
    if (o < steps) load(o);  // (under way while A is brought in)
  switch (a.source) {
    case EJOIN_F32: few_fill<float, MT>(a, lds); break;
    case EJOIN_F16: few_fill<f16, MT>(a, lds); break;
    case EJOIN_BF16: few_fill<bf16, MT>(a, lds); break;
    case FEW_E4M3: few_fill_f8<EJOIN_E4M3, MT>(a, lds); break;
    default: few_fill_f8<EJOIN_E5M2, MT>(a, lds); break;
  }
  __syncthreads();
  float4v acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = float4v{0.f, 0.f, 0.f, 0.f};
  int b = 0;
  for (int64_t i = 0; i < steps; i += FEW_AHEAD) {
#pragma unroll
    for (int o = 0; o < FEW_AHEAD; ++o) {
      if (i + o >= steps) break;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Sixteen fb = expand<FB>(raw[o][h], scale_of(sb[o]));
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
          for (int t = 0; t < MT; ++t) {
            const bf16x8 fa = *reinterpret_cast<const bf16x8*>(lds + (((b * 4 + h * 2 + q) * MT + t) << 10) + lane * 16);
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb.half[q], fa, acc[t], 0, 0, 0);
          }
      }
      if (i + o + FEW_AHEAD < steps) load(o);
      if (++b < a.blocks) continue;
      b = 0;
      // the unit is done: a lane holds row 16 t + r16 of C, four neighbours of it
      const int64_t n = unit * FEW_UNIT + 4 * g;
      unit += waves;
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const int m = t * 16 + r16;
        struct __attribute__((packed, aligned(sizeof(OUT)))) Four { OUT x[4]; } f;
#pragma unroll
        for (int e = 0; e < 4; ++e) f.x[e] = Element<OUT>::put(acc[t][e] * a.scale);
        acc[t] = float4v{0.f, 0.f, 0.f, 0.f};
        OUT* c = static_cast<OUT*>(a.C) + (int64_t)m * a.ldc + n;
        if (m >= a.m) continue;
        if (n + 4 <= a.n) {
          *reinterpret_cast<Four*>(c) = f;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (n + e < a.n) c[e] = f.x[e];
        }
      }
    }
  }
}

// The splits' results of a launch's tiles added up in their order, four neighbours a thread.
template <typename OUT, int COLS>
__global__ __launch_bounds__(256) void k_add_parts(const ProductArgs a, const int32_t splits) {
  constexpr uint32_t PER_TILE = TILE * COLS / 1024;  // workgroups
  const uint32_t tile = blockIdx.x / PER_TILE, at = (blockIdx.x - tile * PER_TILE) * 1024 + threadIdx.x * 4;
  const TilePlace<COLS> p(a, tile);
  const int64_t row = p.m0 + at / COLS, col = p.n0 + at % COLS;
  if (row >= a.m || col >= a.n) return;
  const float* from = a.parts + (int64_t)tile * (TILE * COLS) + at;
  float4v sum = *reinterpret_cast<const float4v*>(from);
  for (int s = 1; s < splits; ++s) sum += *reinterpret_cast<const float4v*>(from + (int64_t)s * a.count * (TILE * COLS));
  OUT* c = static_cast<OUT*>(a.C) + row * a.ldc + col;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (col + e < a.n) c[e] = Element<OUT>::put(sum[e]);
}

// ------------------------------------------------------------------------------------------ host side
constexpr int64_t MOST = 1ll << 23;  // coordinates of a row: 256 rows of them are within 31 bits of their first
constexpr int64_t MOST_SCALES = 1ll << 24;  // bytes between rows of scales: those of 256 rows are within 32 bits of their first

bool bad_rows(const ejoin_f8_rows* r, int64_t most_rows) {
  if (!r || !r->values || !r->scales || (r->format != EJOIN_E4M3 && r->format != EJOIN_E5M2)) return true;
  if (r->n < 1 || r->n >= most_rows || r->d < 1 || r->d >= MOST) return true;
  const int64_t width = up(r->d, BLOCK), scales = up(f8_blocks(r->d), 4);
  if (r->ld < width || r->ld % BLOCK != 0 || r->ld > MOST || r->ld_scales < scales || r->ld_scales % 4 != 0 || r->ld_scales > MOST_SCALES) return true;
  return (reinterpret_cast<uintptr_t>(r->values) & 127) != 0 || (reinterpret_cast<uintptr_t>(r->scales) & 3) != 0;
}

int launch_quantize(ejoin_ctx* ctx, const void* X, int32_t type, int64_t n, int64_t d, int64_t ldx, const ejoin_f8_rows* rows, const ejoin_f8_rows* columns,
                    hipStream_t st) {
  QuantArgs a;
  memset(&a, 0, sizeof(a));
  a.X = X;
  a.n = n;
  a.d = d;
  a.ldx = ldx;
  a.blocks = (uint32_t)f8_blocks(d);
  if (rows) a.rows = rows->values, a.row_scales = rows->scales, a.ld_rows = rows->ld, a.ld_row_scales = rows->ld_scales;
  if (columns) a.cols = columns->values, a.col_scales = columns->scales, a.ld_cols = columns->ld, a.ld_col_scales = columns->ld_scales;
  const bool e4m3 = (rows ? rows : columns)->format == EJOIN_E4M3;
  const int64_t tiles = f8_blocks(n) * a.blocks;
  if (columns && tiles > 4 * MOST_GROUPS) return EJOIN_EUNSUPPORTED;  // (of 256 threads: X would be 2^37 values)
  with_type(type, [&](auto t) {
    typedef decltype(t) T;
    void (*kernel)(QuantArgs) = nullptr;
    if (!columns) kernel = e4m3 ? &k_quantize_rows<T, EJOIN_E4M3> : &k_quantize_rows<T, EJOIN_E5M2>;
    else if (!rows) kernel = e4m3 ? &k_quantize_tile<T, EJOIN_E4M3, false> : &k_quantize_tile<T, EJOIN_E5M2, false>;
    else kernel = e4m3 ? &k_quantize_tile<T, EJOIN_E4M3, true> : &k_quantize_tile<T, EJOIN_E5M2, true>;
    if (columns) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(256), 0, st, a);
      return;
    }
    constexpr int64_t ROWS = 16 * QUANT_ROWS;  // of a workgroup
    const int64_t most = MOST_GROUPS / a.blocks * ROWS;
    for (a.first = 0; a.first < n; a.first += most) {
      const int64_t here = n - a.first < most ? n - a.first : most;
      hipLaunchKernelGGL(kernel, dim3((unsigned)((here + ROWS - 1) / ROWS * a.blocks)), dim3(256), 0, st, a);
    }
  });
  EJ_TRY(hipGetLastError());
  return EJOIN_OK;
}

typedef void (*FewKernel)(FewArgs);
template <typename OUT>
FewKernel few_kernel(int32_t format, int tiles) {
  static const FewKernel of[2][4] = {{&k_f8_few<0, OUT, 1>, &k_f8_few<0, OUT, 2>, &k_f8_few<0, OUT, 3>, &k_f8_few<0, OUT, 4>},
                                     {&k_f8_few<1, OUT, 1>, &k_f8_few<1, OUT, 2>, &k_f8_few<1, OUT, 3>, &k_f8_few<1, OUT, 4>}};
  return of[format][tiles - 1];
}
int few_tiles(int64_t m) { return (int)((m + 15) / 16); }
// Whether m rows are few: their fragments fit the LDS.
bool few(int64_t m, int64_t d) { return m <= FEW_ROWS && few_tiles(m) * f8_blocks(d) * 4096 <= FEW_LDS; }

int launch_few(ejoin_ctx* ctx, const void* X, const uint8_t* sX, int32_t source, int64_t m, int64_t ldx, int64_t lsx, const ejoin_f8_rows* B, float scale, void* C,
               int32_t type, int64_t ldc, hipStream_t st) {
  const int tiles = few_tiles(m);
  const FewArgs a{X, sX, ldx, lsx, source, (int32_t)m, (int32_t)B->d, (int32_t)f8_blocks(B->d), B->values, B->scales, B->ld, B->ld_scales, B->n, scale, C, ldc};
  const int lds = tiles * a.blocks * 4096;
  // workgroups of eight wavefronts, two a CU where the LDS holds two
  constexpr int threads = 512, waves = threads / 64;
  const int64_t units = (a.n + FEW_UNIT - 1) / FEW_UNIT, groups = (units + waves - 1) / waves, most = (int64_t)ctx->num_cu * (lds > (80 << 10) ? 1 : 2);
  FewKernel kernel = type == EJOIN_F32 ? few_kernel<float>(B->format, tiles) : type == EJOIN_F16 ? few_kernel<f16>(B->format, tiles) : few_kernel<bf16>(B->format, tiles);
  hipLaunchKernelGGL(kernel, dim3((unsigned)(groups < most ? groups : most)), dim3(threads), lds, st, a);
  EJ_TRY(hipGetLastError());
  return EJOIN_OK;
}

typedef void (*ProductKernel)(ProductArgs);
template <typename OUT, int WM, int WN>
ProductKernel product_kernel(int32_t fa, int32_t fb) {
  if constexpr (sizeof(OUT) == 4) {
    if (fa == EJOIN_E4M3) return fb == EJOIN_E4M3 ? &k_f8_product<WaveTile16<0, 0, 64 * WN>, WM, WN> : &k_f8_product<WaveTile16<0, 1, 64 * WN>, WM, WN>;
    return fb == EJOIN_E4M3 ? &k_f8_product<WaveTile16<1, 0, 64 * WN>, WM, WN> : &k_f8_product<WaveTile16<1, 1, 64 * WN>, WM, WN>;
  } else {
    constexpr int MI = 8 / WM;
    if (fa == EJOIN_E4M3) return fb == EJOIN_E4M3 ? &k_f8_product_ahead<WaveTile8<0, 0, OUT, MI>, WM, WN> : &k_f8_product_ahead<WaveTile8<0, 1, OUT, MI>, WM, WN>;
    return fb == EJOIN_E4M3 ? &k_f8_product_ahead<WaveTile8<1, 0, OUT, MI>, WM, WN> : &k_f8_product_ahead<WaveTile8<1, 1, OUT, MI>, WM, WN>;
  }
}

// The tiles of a product, in `splits` pieces of k.
template <typename OUT, int WM, int WN>
int launch_tiles(ejoin_ctx* ctx, const ejoin_f8_rows* A, const ejoin_f8_rows* B, ProductArgs& a, int splits, hipStream_t st) {
  typedef Shape<WM, WN> L;
  a.count = a.tiles_m * a.tiles_n;
  a.per_split = (int32_t)up((a.blocks + splits - 1) / splits, 4);
  a.tiles = a.count * (uint32_t)splits;
  a.per_xcd = (a.tiles + NUM_XCD - 1) / NUM_XCD;
  const ProductKernel kernel = product_kernel<OUT, WM, WN>(A->format, B->format);
  const uint32_t slots = (uint32_t)(ctx->num_cu * L::PER_CU) / NUM_XCD;
  hipLaunchKernelGGL(kernel, dim3((slots < a.per_xcd ? slots : a.per_xcd) * NUM_XCD), dim3(64 * L::WAVES), L::LDS, st, a);
  EJ_TRY(hipGetLastError());
  return EJOIN_OK;
}

// Pieces of k that a product of so many tiles of 256 x 128 is cut into: as many as bring all workgroups work, of eight k-blocks each at least, while their
// results fit the memory that is set aside for them.  (Only the tiles past the last whole round cut, and joined: 50,021 x 384, k = 4,096, 588 tiles for 512
// workgroups: 190 us, in two rounds 181.)
int splits_of(int64_t workgroups, int64_t tiles, int64_t blocks) {
  int64_t s = workgroups / tiles;
  s = s < blocks / 8 ? s : blocks / 8;
  const int64_t fit = EJOIN_F8_PRODUCT_BYTES / (tiles * TILE * 128 * 4);
  s = s < fit ? s : fit;
  if (s < 2) return 1;
  const int64_t per = up((blocks + s - 1) / s, 4);  // (four blocks share a dword of scales)
  return (int)((blocks + per - 1) / per);
}

// `parts_at`: where in the context's memory the splits' results may stand.
int launch_product(ejoin_ctx* ctx, const ejoin_f8_rows* A, const ejoin_f8_rows* B, float scale, void* C, int32_t type, int64_t ldc, int64_t parts_at,
                   hipStream_t st) {
  ProductArgs a;
  memset(&a, 0, sizeof(a));
  a.A = A->values, a.sA = A->scales, a.lda = A->ld, a.lsa = A->ld_scales, a.m = A->n;
  a.B = B->values, a.sB = B->scales, a.ldb = B->ld, a.lsb = B->ld_scales, a.n = B->n;
  a.blocks = (int32_t)f8_blocks(A->d);
  a.scale = scale;
  a.C = C;
  a.ldc = ldc;
  const int64_t tiles_m = (a.m + TILE - 1) / TILE, tiles = tiles_m * ((a.n + 127) / 128), wide = tiles_m * ((a.n + 255) / 256);
  if (tiles > 0x7FFFFFF0ll) return EJOIN_EUNSUPPORTED;
  a.tiles_m = (uint32_t)tiles_m;
  const int64_t workgroups = 2 * (int64_t)ctx->num_cu;
  const int splits = splits_of(workgroups, tiles, a.blocks);
  if (splits == 1 && type != EJOIN_F32) {
    // Tiles of 256 x 256 where there is one for every CU, of 256 x 128 where there is not: 500 x 5,000 x 300 in 40 of the larger 12.4 us, in 80 of the
    // others 9.4; 4,096 x 4,096 x 1,024 in 256 and 512 23.6 and 26.2.
    if (wide >= ctx->num_cu) {
      a.tiles_n = (uint32_t)((a.n + 255) / 256);
      return (type == EJOIN_F16 ? launch_tiles<f16, 2, 4> : launch_tiles<bf16, 2, 4>)(ctx, A, B, a, 1, st);
    }
    a.tiles_n = (uint32_t)((a.n + 127) / 128);
    return (type == EJOIN_F16 ? launch_tiles<f16, 2, 2> : launch_tiles<bf16, 2, 2>)(ctx, A, B, a, 1, st);
  }
  a.tiles_n = (uint32_t)((a.n + 127) / 128);
  if (splits == 1) return launch_tiles<float, 2, 2>(ctx, A, B, a, 1, st);
  EJ_RC(ensure_embed(ctx, parts_at + splits * tiles * (TILE * 128 * 4), st));
  a.parts = reinterpret_cast<float*>(ctx->embed + parts_at);  // (pieces are joined in FP32, whatever the results are rounded to then)
  EJ_RC((launch_tiles<float, 2, 2>(ctx, A, B, a, splits, st)));
  with_type(type, [&](auto t) {
    typedef decltype(t) T;
    hipLaunchKernelGGL((k_add_parts<T, 128>), dim3((unsigned)(tiles * (TILE * 128 / 1024))), dim3(256), 0, st, a, splits);
  });
  EJ_TRY(hipGetLastError());
  return EJOIN_OK;
}

template <typename KERNEL>
hipError_t allow_lds(hipError_t e, KERNEL kernel, int bytes) {
  return e != hipSuccess ? e : hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

bool bad_result(const void* C, int32_t type, int64_t n, int64_t ldc, float scale) { return !C || bad_type(type) || ldc < n || !isfinite(scale); }

}  // namespace

hipError_t f8_prepare_kernels() {
  hipError_t e = hipSuccess;
  for (int fa : {EJOIN_E4M3, EJOIN_E5M2}) {
    for (int tiles = 1; tiles <= FEW_ROWS / 16; ++tiles)
      for (FewKernel kernel : {few_kernel<float>(fa, tiles), few_kernel<f16>(fa, tiles), few_kernel<bf16>(fa, tiles)}) e = allow_lds(e, kernel, FEW_LDS);
    for (int fb : {EJOIN_E4M3, EJOIN_E5M2}) {
      for (ProductKernel kernel : {product_kernel<float, 2, 2>(fa, fb), product_kernel<f16, 2, 2>(fa, fb), product_kernel<bf16, 2, 2>(fa, fb)})
        e = allow_lds(e, kernel, Shape<2, 2>::LDS);
      for (ProductKernel kernel : {product_kernel<f16, 2, 4>(fa, fb), product_kernel<bf16, 2, 4>(fa, fb)}) e = allow_lds(e, kernel, Shape<2, 4>::LDS);
    }
  }
  return e;
}

extern "C" {

int ejoin_embed_reserve(ejoin_ctx* ctx, int64_t bytes) {
  if (!ctx || bytes < 0) return EJOIN_EINVAL;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return EJOIN_EHIP;
  return ensure_embed(ctx, bytes);
}

int ejoin_f8_quantize(ejoin_ctx* ctx, const void* X, int32_t type, int64_t n, int64_t d, int64_t ldx, const ejoin_f8_rows* rows,
                      const ejoin_f8_rows* columns, void* stream) {
  if (!ctx || !X || bad_type(type) || n < 1 || n >= (columns ? MOST : 1ll << 31) || d < 1 || d >= MOST || ldx < d || (!rows && !columns)) return EJOIN_EINVAL;
  if (rows && (bad_rows(rows, 1ll << 31) || rows->n != n || rows->d != d)) return EJOIN_EINVAL;
  if (columns && (bad_rows(columns, MOST) || columns->n != d || columns->d != n)) return EJOIN_EINVAL;
  if (rows && columns && rows->format != columns->format) return EJOIN_EINVAL;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return EJOIN_EHIP;
  return launch_quantize(ctx, X, type, n, d, ldx, rows, columns, static_cast<hipStream_t>(stream));
}

int ejoin_f8_product(ejoin_ctx* ctx, const ejoin_f8_rows* A, const ejoin_f8_rows* B, float scale, void* C, int32_t type, int64_t ldc, void* stream) {
  if (!ctx || bad_rows(A, 1ll << 31) || bad_rows(B, 1ll << 31) || A->d != B->d || bad_result(C, type, B->n, ldc, scale)) return EJOIN_EINVAL;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return EJOIN_EHIP;
  if (few(A->n, A->d))
    return launch_few(ctx, A->values, A->scales, A->format == EJOIN_E4M3 ? FEW_E4M3 : FEW_E5M2, A->n, A->ld, A->ld_scales, B, scale, C, type, ldc,
                      static_cast<hipStream_t>(stream));
  return launch_product(ctx, A, B, scale, C, type, ldc, 0, static_cast<hipStream_t>(stream));
}

int ejoin_f8_scores(ejoin_ctx* ctx, const void* X, int32_t xtype, int64_t m, int64_t ldx, const ejoin_f8_rows* B, float scale, void* C, int32_t type,
                    int64_t ldc, void* stream) {
  if (!ctx || !X || bad_type(xtype) || bad_rows(B, 1ll << 31) || m < 1 || m >= MOST || ldx < B->d || bad_result(C, type, B->n, ldc, scale)) return EJOIN_EINVAL;
  DeviceGuard guard(ctx->device);
  if (!guard.ok) return EJOIN_EHIP;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (few(m, B->d)) return launch_few(ctx, X, nullptr, xtype, m, ldx, 0, B, scale, C, type, ldc, st);
  const int64_t width = up(B->d, BLOCK), scales = up(f8_blocks(B->d), 4), bytes = up(m * (width + scales), 256);
  // room for the splits' results as well: growing in between would free what the first launch writes
  EJ_RC(ensure_embed(ctx, bytes + EJOIN_F8_PRODUCT_BYTES, st));
  const ejoin_f8_rows A{ctx->embed, ctx->embed + m * width, width, scales, m, B->d, EJOIN_E4M3};
  EJ_RC(launch_quantize(ctx, X, xtype, m, B->d, ldx, &A, nullptr, st));
  return launch_product(ctx, &A, B, scale, C, type, ldc, bytes, st);
}

}  // extern "C"
