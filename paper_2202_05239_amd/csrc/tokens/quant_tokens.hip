// Tokens into 8 bits with a scale each, from real tensors, with the gate of a gated block in front:
//
//   v = x,  or  act(gate) * x;   scale and code of a row as in tokens_device.h;
//   result: the codes and scales, or the values code * scale that they stand for, in the type of x.
//
// Bound by HBM: every element is read once, its row stays in registers between the maximum and the codes, and is written once (8192 x
// 16384 bf16 with a silu gate, 805 MB: 140 us, 5.7 TB/s).  Few rows are one chain of load, maximum and store: 33 x 1111 3.8 us.
#include <math.h>

#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

struct QuantParams {
  const void *x, *gate;
  void *y;
  float *scale;
  int64_t ldx, ldg, ldy;
  int rows, cols, act, codes;
  int pad;                                          // codes are written up to this column, zeros from `cols` on
};

// silu(g) = g / (1 + e^-g); gelu(g) = g / (1 + e^(-2 u)), u = sqrt(2/pi) (g + 0.044715 g^3), the tanh form.  For large -g the
// exponential is infinite and the quotient 0; g = -inf gives NaN, as the formulas do.  For 16-bit tensors, which round at 2^-11 or above,
// the exponential is 2^(u log2 e), off by up to |u| units in the last place of 32 bits (2^-17 at u = -100), and the quotient a product
// with a reciprocal: with exact calls the kernel is bound by its instructions (8192 x 16384 bf16 177 us against 140).  32-bit tensors
// get the exact calls (8192 x 16384 305 us either way, 64 x 4096 4.6 and 5.4).
template <typename T>
__device__ __forceinline__ float act_of(int act, float g) {
  if (act == F8_ACT_NONE) return g;
  const float u = act == F8_ACT_SILU ? g : 1.5957691216057308f * g * __builtin_fmaf(0.044715f * g, g, 1.0f);
  if constexpr (sizeof(T) == 4) return g / (1.0f + expf(-u));
  return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * u));
}

template <typename T, int TPR, int NV>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void quant_tokens_kernel(QuantParams p) {
  typedef RowMap<TPR, NV> Map;
  constexpr int THREADS = TPR == 64 ? 256 : TPR, RPB = THREADS / TPR;
  __shared__ float lds[THREADS / 64];
  const int64_t row = row_block() * RPB + (int)threadIdx.x / TPR;
  const int t = (int)threadIdx.x % TPR;
  if (row >= p.rows) return;                         // (a whole workgroup, or waves on their own: no barrier below)
  const T *x = static_cast<const T *>(p.x) + row * p.ldx;
  float v[NV][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) load_piece<T, Map>(x, i, t, p.cols, v[i]);
  if (p.gate) {
    const T *gate = static_cast<const T *>(p.gate) + row * p.ldg;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float g[8];
      load_piece<T, Map>(gate, i, t, p.cols, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= act_of<T>(p.act, g[j]);
    }
  }
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[i][j]));
  const TokenScale s = token_scale(row_amax<TPR>(top, lds));
  if (t == 0 && p.scale) p.scale[row] = s.scale;
  lift(v, s);
  if (p.codes) {
    int8_t *y = static_cast<int8_t *>(p.y) + row * p.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      int q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = code_of(v[i][j], s);
      store_codes<Map>(y, i, t, p.pad, q);
    }
  } else {
    T *y = static_cast<T *>(p.y) + row * p.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = value_of(v[i][j], s);
      store_piece<T, Map>(y, i, t, p.cols, o);
    }
  }
}

// (false where the threads' pieces do not cover a row)
template <typename T, int TPR, int NV>
bool launch(const QuantParams &p, hipStream_t s) {
  if (p.pad > RowMap<TPR, NV>::most) return false;
  constexpr int THREADS = TPR == 64 ? 256 : TPR, RPB = THREADS / TPR;
  hipLaunchKernelGGL((quant_tokens_kernel<T, TPR, NV>), block_grid(((int64_t)p.rows + RPB - 1) / RPB), dim3(THREADS), 0, s, p);
  return true;
}

// Threads to a row: as many as leave each one or two pieces, up to 1024 (16384 gated columns, 8192 rows, us: 1024 threads of two pieces
// 141, 512 of four 170, 256 of eight 201).  Widths from 4097 to 6144 leave a quarter to a half of 512 threads' pieces empty: 256 threads of three, unless
// rows are so few that each one's own time counts.  The line lies between 256 and 768 rows at all of these widths (bf16, three | two pieces, us): 4100
// columns 256 rows 3.9 | 3.6, 512 4.1 | 4.0, 768 4.5 | 4.6, 2048 7.0 | 8.4, 16384 41 | 52; 6144 columns 3.5 | 3.5, 3.9 | 4.0, 4.3 | 4.7, 7.7 | 9.1,
// 54 | 62; gated 5120 columns 5.8 | 5.0, 6.3 | 5.9, 6.7 | 7.0, 13.6 | 15.2, 85 | 102; 32 bits alike, behind only far out of the caches
// (16384 x 6144 91.6 | 90.6, gated 176 | 165).
template <typename T>
f8_status launch_row(const QuantParams &p, hipStream_t s) {
  static_assert(RowMap<1024, 8>::most == ROW_MOST, "the last shape takes every row");
  launch<T, 64, 1>(p, s) || launch<T, 64, 2>(p, s) || launch<T, 256, 1>(p, s) || launch<T, 256, 2>(p, s) || (p.rows >= 512 && launch<T, 256, 3>(p, s)) ||
      launch<T, 512, 2>(p, s) || launch<T, 1024, 2>(p, s) || launch<T, 1024, 8>(p, s);
  return launch_status();
}

f8_status enqueue(const QuantParams &p, int x_type, hipStream_t s) {
  return x_type == F8_F32 ? launch_row<float>(p, s) : x_type == F8_F16 ? launch_row<f16>(p, s) : launch_row<bf16>(p, s);
}

}  // namespace

f8_status enqueue_quant_tokens(const void *x, int64_t ldx, int x_type, int8_t *codes, int64_t ld, int pad, float *scale, int rows, int cols,
                               hipStream_t s) {
  return enqueue(QuantParams{x, nullptr, codes, scale, ldx, 0, ld, rows, cols, F8_ACT_NONE, 1, pad}, x_type, s);
}

}  // namespace f8

using namespace f8;

extern "C" f8_status f8_quant_tokens(const void *x, const void *gate, void *y, float *scale, const f8_quant_tokens_desc *d, void *stream) {
  if (!d) return F8_ERR_NULL;
  if (d->rows < 0 || d->cols < 1 || d->cols > ROW_MOST) return F8_ERR_SHAPE;
  if (!real_type(d->x_type) || (d->y_type != F8_S8 && d->y_type != d->x_type)) return F8_ERR_DTYPE;
  if (d->act != F8_ACT_NONE && d->act != F8_ACT_SILU && d->act != F8_ACT_GELU) return F8_ERR_UNSUPPORTED;
  if (d->ldx < d->cols || d->ldy < d->cols || (gate && d->ldg < d->cols)) return F8_ERR_SHAPE;
  if (d->rows == 0) return F8_OK;
  const bool codes = d->y_type == F8_S8;
  if (!x || !y || (codes && !scale) || (d->act != F8_ACT_NONE && !gate)) return F8_ERR_NULL;
  const size_t e = bytes_of(d->x_type), o = codes ? 1 : e;
  if (!aligned_to(x, e) || !aligned_to(y, o) || !aligned_to(gate, e) || !aligned_to(scale, 4)) return F8_ERR_ALIGN;
  const QuantParams p{x, gate, y, scale, d->ldx, d->ldg, d->ldy, d->rows, d->cols, d->act, codes, d->cols};
  return enqueue(p, d->x_type, static_cast<hipStream_t>(stream));
}
