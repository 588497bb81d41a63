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
};

typedef int v16i __attribute__((ext_vector_type(16)));

// 16 bytes of a row from column k on, at any address; past the row's end zeros (there the row's last 16 bytes, shifted down).
__device__ __forceinline__ v4i load_row16(const int8_t *row, bool real, int k, int K) {
  unsigned __int128 v = 0;
  if (real && k < K) {
    if (K >= 16) {
      const int over = max(k + 16 - K, 0);
      __builtin_memcpy(&v, row + k - over, 16);
      v >>= 8 * over;
    } else {
#pragma nounroll
      for (int i = k; i < K; ++i) v |= (unsigned __int128)(uint8_t)row[i] << (8 * (i - k));
    }
  }
  return __builtin_bit_cast(v4i, v);
}

// 8 real elements of a row from column k on (a multiple of 8); past the row's end zeros.
template <typename X>
__device__ __forceinline__ void load_row8(const X *row, int k, int K, float (&v)[8]) {
  if (k + 8 <= K) {
    v4i raw[2];
    __builtin_memcpy(raw, row + k, 8 * sizeof(X));
    unpack8<X>(raw, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < K ? (float)row[k + j] : 0.0f;
  }
}

// The 16 channels n .. n + 15 of token m from a lane's registers (n a multiple of 16), at any address.
template <typename T>
__device__ __forceinline__ void scale16(const LinearParams &p, const v16i &acc, float sx, int n, T (&o)[16]) {
  float s[16], b[16];
  if (n + 16 <= p.N) {
    __builtin_memcpy(s, p.sw + n, 64);
    if (p.bias) __builtin_memcpy(b, p.bias + n, 64);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = n + i < p.N ? p.sw[n + i] : 0.0f;
      if (p.bias) b[i] = n + i < p.N ? p.bias[n + i] : 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) o[i] = (T)__builtin_fmaf((float)acc[i] * sx, s[i], p.bias ? b[i] : 0.0f);
}
template <typename T>
__device__ __forceinline__ void store_scaled(const LinearParams &p, const v16i &acc, int m, int n) {
  if (m >= p.M || n >= p.N) return;
  T o[16];
  scale16(p, acc, p.sx[m], n, o);
  T *y = static_cast<T *>(p.y) + m * p.ldy + n;
  if (n + 16 <= p.N) {
#pragma unroll
    for (int q = 0; q < (int)sizeof(T); ++q) {
      v4i v;
      __builtin_memcpy(&v, o + q * (16 / sizeof(T)), 16);
      reinterpret_cast<v4i_any *>(y)[q] = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (n + i < p.N) y[i] = o[i];
  }
}

constexpr int64_t LINEAR_TILES_MOST = 1 << 22;   // workgroups of a launch (2^32 threads)

// Tiles through LDS by its own loads, for operands whose rows start on 4 bytes.  `tile`: which (linear_tile.hip).
f8_status launch_linear_tile(const LinearParams &p, int y_type, int tile, hipStream_t s);
// What takes least, by estimate: `tile` over tokens 0 .. M1 - 1 and channels 0 .. N1 - 1, and if that is not all, `tile2` over the rest.
// (The rest is less than a round of the first tile: its workgroups always fit a launch.)
struct LinearPlan {
  int tile, M1, N1, tile2;
  float us;
  int64_t wgs;                             // of the first launch
};
LinearPlan linear_plan(int M, int N, int K);

// LINEAR_FEW tokens to a workgroup, any strides and alignment (linear_few.hip).  x_type F8_S8: codes with scales sx; real: p.x points to the
// tokens themselves, p.sx is not read, M at most
// LINEAR_FEW, M * ceil(K / 512) at most LINEAR_FEW_HELD.
f8_status launch_linear_few(const LinearParams &p, int x_type, int y_type, hipStream_t s);
constexpr int LINEAR_FEW = 16, LINEAR_FEW_HELD = 16, LINEAR_FEW_MOST = 512;

}  // namespace f8
