// Device-side pieces of the kernels on real-valued tokens: loads and stores of rows in 32 or 16 bits, reductions over the
// threads of a row, and the 8-bit format of a token,
//
//   scale = max(max |v| / 127, 2^-126),   code = round_half_even(v / scale)  (0 where v / scale is not a number),
//
// which never divides by zero (a row of zeros has codes 0) and keeps what is not finite visible: a row with a NaN or an
// infinity has a scale that is not finite, so that every value and every product made from it is NaN.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../../include/f8.h"
#include "../f8_device.h"

namespace f8 {

typedef _Float16 f16;
typedef __bf16 bf16;

// 16 bytes at any address (a vector store of its own type: as elements the compiler would split it where another branch stores some)
typedef int v4i_any __attribute__((ext_vector_type(4), aligned(1), may_alias));

constexpr int ROW_MOST = 65536;   // columns of a row that a workgroup holds in registers

__device__ __forceinline__ int64_t row_block() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }   // see block_grid

// How the elements of a row lie in its threads: `TPR` threads share a row, each has NV pieces of 8 neighbours, one or two 16-byte
// accesses.  The accesses are taken at any address an element may have: this chip's loads and stores do not need alignment, a row
// off the 16-byte grid costs up to a second line per access.
template <int TPR, int NV>
struct RowMap {
  static constexpr int most = TPR * NV * 8;
  static __device__ __forceinline__ int col(int i, int j, int t) { return (i * TPR + t) * 8 + j; }
};

template <typename T>
__device__ __forceinline__ void unpack8(const v4i *raw, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __int_as_float(raw[j >> 2][j & 3]);
  } else if constexpr (__is_same(T, bf16)) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __int_as_float(raw[0][j] << 16);
      v[2 * j + 1] = __int_as_float(raw[0][j] & 0xffff0000);
    }
  } else {
    typedef f16 h8 __attribute__((ext_vector_type(8)));
    const h8 h = __builtin_bit_cast(h8, raw[0]);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)h[j];
  }
}

// 8 elements of piece i of a row into v; what lies past the row's end reads as 0.
template <typename T, typename Map>
__device__ __forceinline__ void load_piece(const T *row, int i, int t, int cols, float (&v)[8]) {
  const int c = Map::col(i, 0, t);
  if (c + 8 <= cols) {
    v4i raw[2];
    __builtin_memcpy(raw, row + c, 8 * sizeof(T));
    unpack8<T>(raw, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = Map::col(i, j, t);
      v[j] = e < cols ? (float)row[e] : 0.0f;
    }
  }
}

template <typename T, typename Map>
__device__ __forceinline__ void store_piece(T *row, int i, int t, int cols, const float (&v)[8]) {
  const int c = Map::col(i, 0, t);
  if (c + 8 <= cols) {
    typedef T t8 __attribute__((ext_vector_type(8)));
    t8 o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = (T)v[j];
#pragma unroll
    for (int q = 0; q < (int)sizeof(T) / 2; ++q) reinterpret_cast<v4i_any *>(row + c)[q] = reinterpret_cast<const v4i *>(&o)[q];
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = Map::col(i, j, t);
      if (e < cols) row[e] = (T)v[j];
    }
  }
}

template <typename Map>
__device__ __forceinline__ void store_codes(int8_t *row, int i, int t, int cols, const int (&q)[8]) {
  const int c = Map::col(i, 0, t);
  if (c + 8 <= cols) {
    const v2i o{(int)pack4(q[0], q[1], q[2], q[3]), (int)pack4(q[4], q[5], q[6], q[7])};
    __builtin_memcpy(row + c, &o, 8);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = Map::col(i, j, t);
      if (e < cols) row[e] = (int8_t)q[j];
    }
  }
}

// Reductions over the TPR threads of a row, every thread gets the result; the order is fixed.  `lds`: a word for each wave, used
// by one reduction at a time (a second one on the same words needs another set: see `turn`).
template <int TPR, typename V, typename Op>
__device__ __forceinline__ V reduce_row(V v, V *lds, Op op) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v = op(v, __shfl_xor(v, d));
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < W; ++w) v = op(v, lds[w]);
  }
  return v;
}
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *lds) {
  return reduce_row<TPR>(v, lds, [](float a, float b) { return a + b; });
}
// The largest magnitude by its bits: a NaN's bits lie above an infinity's, so one that is there wins.
template <int TPR>
__device__ __forceinline__ float row_amax(uint32_t bits, float *lds) {
  return __uint_as_float(reduce_row<TPR>(bits, reinterpret_cast<uint32_t *>(lds), [](uint32_t a, uint32_t b) { return a > b ? a : b; }));
}
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

struct TokenScale {
  float scale, by, inv;                   // `by`: the scale that elements are divided by (see lift), inv: its reciprocal
  uint32_t real;                          // all bits set where the scale is finite, else 0
};
// Rows below about 2^-93 are divided as 2^64 times themselves: the remainder in over_scale would leave the normal range.
constexpr float SMALL_SCALE = 0x1p-100f, LIFT = 0x1p64f;
__device__ __forceinline__ TokenScale token_scale(float amax) {
  float s = amax / 127.0f;
  s = s < 1.17549435e-38f ? 1.17549435e-38f : s;   // (false for a NaN, which stays)
  const float by = s < SMALL_SCALE ? s * LIFT : s;
  return TokenScale{s, by, 1.0f / by, s < __builtin_inff() ? 0xffffffffu : 0u};
}
__device__ __forceinline__ void lift(float (&v)[8], const TokenScale &s) {
  if (s.scale < SMALL_SCALE) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= LIFT;
  }
}
template <int NV>
__device__ __forceinline__ void lift(float (&v)[NV][8], const TokenScale &s) {
  if (s.scale < SMALL_SCALE) {
#pragma unroll
    for (int i = 0; i < NV; ++i) lift(v[i], s);
  }
}
// A lifted v over its scale, correctly rounded without a division for each element: the product with the reciprocal, corrected by its exact
// remainder.  (One operation off in the last place would turn codes at ties.)
__device__ __forceinline__ float over_scale(float v, const TokenScale &s) {
  const float q = v * s.inv;
  return __builtin_fmaf(__builtin_fmaf(-q, s.by, v), s.inv, q);
}
// The code in the low byte: at 1.5 * 2^23 the unit of the sum is 1, so the addition rounds half to even and leaves the integer in
// the low bits.  Codes of a row whose scale is not finite are 0.
__device__ __forceinline__ int code_of(float v, const TokenScale &s) {
  return (int)(__float_as_uint(over_scale(v, s) + 12582912.0f) & s.real);
}
// The value that the code stands for; NaN where the scale is not finite (an infinite one times 0, or what is no number itself).
__device__ __forceinline__ float value_of(float v, const TokenScale &s) { return __builtin_rintf(over_scale(v, s)) * s.scale; }

}  // namespace f8
