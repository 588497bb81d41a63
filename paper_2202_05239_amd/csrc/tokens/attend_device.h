// Pieces that the attention kernels share: sums over a workgroup, equal runs of units, 8-bit codes as f16, the matrix instruction and the
// weights of either 16-bit type, rows as dwords.
#pragma once

#include "tokens_device.h"

namespace f8 {

typedef f16 h8 __attribute__((ext_vector_type(8)));
typedef bf16 b8 __attribute__((ext_vector_type(8)));
typedef f16 h2 __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef long long v2l __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.4426950408889634f;
// The least that a value's scale counts for in the maximum, as a power of two: 2^31 tokens of 2^(15 - SMALL) each stay below the largest
// 32-bit number.  Values whose scales all lie below it (1e-24) only lose bits below 2^-109, where their weights leave f16's normal range.
constexpr float SMALL = -80.0f;

struct Runs {                                // equal runs of `total` units, the first `more` of them one longer
  int64_t per, more;
  __device__ __forceinline__ Runs(int64_t total, int wgs) : per(total / (uint32_t)wgs), more(total - per * wgs) {}
  __device__ __forceinline__ int64_t start(int64_t i) const { return i * per + (i < more ? i : more); }
  __device__ __forceinline__ int64_t of(int64_t unit) const {
    const int64_t longer = more * (per + 1);
    return unit < longer ? unit / (per + 1) : more + (unit - longer) / per;
  }
};
__device__ __forceinline__ int64_t uniform64(int64_t v) {
  return (int64_t)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)v);
}

// Two sums over a workgroup; `lds`: a pair of words per wave.
template <int W>
__device__ __forceinline__ void wg_sum(int64_t (&v)[2], int64_t (*lds)[2]) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v[k] += __shfl_xor((long long)v[k], d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6][k] = v[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    v[k] = 0;
#pragma unroll
    for (int w = 0; w < W; ++w) v[k] += lds[w][k];
  }
  __syncthreads();
}

// Codes of four neighbouring bytes as f16, exactly: byte + 128 under the exponent of 1024, minus 1152.
__device__ __forceinline__ h2 codes_lo(uint32_t u) { return __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - h2{(f16)1152, (f16)1152}; }
__device__ __forceinline__ h2 codes_hi(uint32_t u) { return __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - h2{(f16)1152, (f16)1152}; }

template <typename C>
struct Operand {                            // 16-bit type of the products
  typedef f16 t;
  static constexpr float UP = 15.0f;        // the largest weight as a power of two
  // Two weights, cut to 16 bits, and what is left of them: never negative, nor 0 where the weight is a normal number, so that an infinite
  // value times both is infinite
  static __device__ __forceinline__ uint32_t cut(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b)); }
  static __device__ __forceinline__ t rest(float w, uint32_t pair, int k) {
    const float left = w - (float)__builtin_bit_cast(h2, pair)[k];
    return (t)fmaxf(left, fminf(w * 0x1p-10f, 0x1p-24f));
  }
  static __device__ __forceinline__ v4f mfma(v4i a, v4i b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
};
template <>
struct Operand<bf16> {
  typedef bf16 t;
  static constexpr float UP = 0.0f;         // (has the range of 32 bits)
  static __device__ __forceinline__ uint32_t cut(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
  static __device__ __forceinline__ t rest(float w, uint32_t pair, int k) {
    const float left = w - __uint_as_float(k ? pair & 0xffff0000u : pair << 16);
    return (t)fmaxf(left, fminf(w, 0x1p-100f));
  }
  static __device__ __forceinline__ v4f mfma(v4i a, v4i b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  }
};

template <int BYTES>
struct Raw {                                // BYTES of a row, as dwords
  uint32_t d[BYTES / 4];
};
template <int BYTES>
__device__ __forceinline__ Raw<BYTES> load_raw(const void *p) {
  Raw<BYTES> r;
  if constexpr (BYTES == 4) {
    r.d[0] = *static_cast<const uint32_t *>(p);
  } else if constexpr (BYTES == 8) {
    const v2i v = *static_cast<const v2i *>(p);
    r.d[0] = v[0], r.d[1] = v[1];
  } else {
#pragma unroll
    for (int i = 0; i < BYTES / 16; ++i) {
      const v4i v = static_cast<const v4i *>(p)[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) r.d[4 * i + j] = v[j];
    }
  }
  return r;
}

}  // namespace f8
