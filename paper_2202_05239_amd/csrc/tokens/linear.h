// The product of 8-bit tokens and weights: what its kernels share, and which of them takes a call.
#pragma once

#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {

struct LinearParams {
  const int8_t *x, *w;
  const float *sx, *sw, *bias;
  void *y;
  int64_t ldx, ldw, ldy;
  int M, N, K;
  int x_vec;                          // real tokens' rows start on 16 bytes
};

typedef int v16i __attribute__((ext_vector_type(16)));

// 16 bytes of a row from column k on, at any address; past the row's end zeros.
__device__ __forceinline__ v4i load_row16(const int8_t *row, bool real, int k, int K) {
  v4i v{0, 0, 0, 0};
  if (real && k + 16 <= K) {
    __builtin_memcpy(&v, row + k, 16);
  } else if (real) {
    int8_t b[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) b[i] = k + i < K ? row[k + i] : 0;
    __builtin_memcpy(&v, b, 16);
  }
  return v;
}

// 8 real elements of a row from column k on (a multiple of 8); past the row's end zeros.
template <typename X>
__device__ __forceinline__ void load_row8(const X *row, int k, int K, int vec, float (&v)[8]) {
  if (vec && k + 8 <= K) {
    v4i raw[2];
    raw[0] = *reinterpret_cast<const v4i *>(row + k);
    if (sizeof(X) == 4) raw[1] = *reinterpret_cast<const v4i *>(row + k + 4);
    unpack8<X>(raw, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < K ? (float)row[k + j] : 0.0f;
  }
}

// The 16 channels n .. n + 15 of token m (n a multiple of 16).  VEC: y, its rows, sw and bias start on 16 bytes.
template <typename T>
__device__ __forceinline__ void store_scaled(const LinearParams &p, const v16i &acc, int m, int n, bool vec) {
  if (m >= p.M || n >= p.N) return;
  const float sx = p.sx[m];
  T *y = static_cast<T *>(p.y) + m * p.ldy + n;
  if (vec && n + 16 <= p.N) {
    typedef T t16 __attribute__((ext_vector_type(16)));
    t16 o;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 s = reinterpret_cast<const float4 *>(p.sw + n)[q];
      const float4 b = p.bias ? reinterpret_cast<const float4 *>(p.bias + n)[q] : make_float4(0, 0, 0, 0);
      o[4 * q] = (T)__builtin_fmaf((float)acc[4 * q] * sx, s.x, b.x);
      o[4 * q + 1] = (T)__builtin_fmaf((float)acc[4 * q + 1] * sx, s.y, b.y);
      o[4 * q + 2] = (T)__builtin_fmaf((float)acc[4 * q + 2] * sx, s.z, b.z);
      o[4 * q + 3] = (T)__builtin_fmaf((float)acc[4 * q + 3] * sx, s.w, b.w);
    }
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<v4i *>(y)[i] = reinterpret_cast<const v4i *>(&o)[i];
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (n + i < p.N) y[i] = (T)__builtin_fmaf((float)acc[i] * sx, p.sw[n + i], p.bias ? p.bias[n + i] : 0.0f);
  }
}

// Tiles through LDS by its own loads, for operands whose rows start on 4 bytes.  `tile`: which (linear_tile.hip).
f8_status launch_linear_tile(const LinearParams &p, int y_type, int tile, hipStream_t s);
int linear_tile_of(int M, int N, int K, float *us);   // the tile that takes least, and its estimated microseconds

// At most LINEAR_FEW tokens, any strides and alignment (linear_few.hip).  x_type F8_S8: codes with scales sx; real: p.x points to the
// tokens themselves, p.sx is not read, M * ceil(K / 512) at most LINEAR_FEW_HELD.
f8_status launch_linear_few(const LinearParams &p, int x_type, int y_type, hipStream_t s);
constexpr int LINEAR_FEW = 16, LINEAR_FEW_HELD = 16;

}  // namespace f8
