// The update of the residual stream between two blocks and the norms on both sides of it, in one pass over the rows:
//
//   u = norm_post(a)  (or a);   r = res_scale * res + gate * u;   y = norm_pre(r)  (or r),
//   norm(v) = v / sqrt(mean v^2 + eps) * w + b                        (root mean square)
//           = (v - mean v) / sqrt(mean (v - mean v)^2 + eps) * w + b  (layer)
//
// y in the type of a, or as 8-bit tokens (tokens_device.h) for the product behind.  r is rounded where it is stored; y comes
// from the 32-bit one.  Bound by HBM: a row is held in registers in 32 bits from its first load to its last store, the sums run
// over the workgroup in a fixed order, and the variance of a layer norm is that of the centred row, not a difference of moments.
// 16384 x 4096 bf16 with norms on both sides and a gate, 537 MB: 100 - 106 us, 5.1 - 5.4 TB/s (a copy 5.5); 64 x 4096 4.6 us, a row's chain
// of loads and one or two reductions.
#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

struct NormParams {
  const void *a, *res, *post_w, *post_b, *gate, *pre_w, *pre_b;
  void *res_out, *y;
  float *scale;
  int64_t lda, ldr, ldg, ldo, ldy;
  int rows, cols, post, pre, codes, w_f32;
  float post_eps, pre_eps, res_scale, inv_cols;
  FastDiv gate_rows;
};

// The weights are vectors of `cols` in the type of the rows or in 32 bits, read by every row (from cache).
template <typename T, typename Map>
__device__ __forceinline__ void load_weight(const void *w, int w_f32, int i, int t, int cols, float (&v)[8]) {
  if (w_f32) load_piece<float, Map>(static_cast<const float *>(w), i, t, cols, v);
  else load_piece<T, Map>(static_cast<const T *>(w), i, t, cols, v);
}

template <typename T, int TPR, int NV>
__device__ __forceinline__ void normalise(float (&v)[NV][8], int form, float eps, const void *w, const void *b, const NormParams &p, int t,
                                          float *lds) {
  typedef RowMap<TPR, NV> Map;
  constexpr int W = TPR / 64;
  float mean = 0.0f;
  if (form == F8_NORM_LAYER) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s += Map::col(i, j, t) < p.cols ? v[i][j] : 0.0f;
    mean = row_sum<TPR>(s, lds) * p.inv_cols;
  }
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = v[i][j] - mean;
      v[i][j] = d;
      s += Map::col(i, j, t) < p.cols ? d * d : 0.0f;
    }
  const float r = 1.0f / sqrtf(row_sum<TPR>(s, lds + W) * p.inv_cols + eps);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    float g[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] *= r;
    if (w) {
      load_weight<T, Map>(w, p.w_f32, i, t, p.cols, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
    }
    if (b) {
      load_weight<T, Map>(b, p.w_f32, i, t, p.cols, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] += g[j];
    }
  }
}

template <typename T, int TPR, int NV>
__global__ __launch_bounds__(TPR == 64 ? 256 : TPR) void norm_tokens_kernel(NormParams p) {
  typedef RowMap<TPR, NV> Map;
  constexpr int THREADS = TPR == 64 ? 256 : TPR, RPB = THREADS / TPR, W = TPR / 64;
  __shared__ float lds[5 * (THREADS / 64)];          // a set of words for each of the five reductions of a row
  const int64_t row = row_block() * RPB + (int)threadIdx.x / TPR;
  const int t = (int)threadIdx.x % TPR;
  if (row >= p.rows) return;                         // (a whole workgroup, or waves on their own: no barrier below)
  float v[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) load_piece<T, Map>(static_cast<const T *>(p.a) + row * p.lda, i, t, p.cols, v[i]);
  if (p.post != F8_NORM_NONE) normalise<T, TPR, NV>(v, p.post, p.post_eps, p.post_w, p.post_b, p, t, lds);
  if (p.gate) {
    const T *gate = static_cast<const T *>(p.gate) + p.gate_rows.div((uint32_t)row) * p.ldg;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float g[8];
      load_piece<T, Map>(gate, i, t, p.cols, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
    }
  }
  if (p.res) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float g[8];
      load_piece<T, Map>(static_cast<const T *>(p.res) + row * p.ldr, i, t, p.cols, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = __builtin_fmaf(p.res_scale, g[j], v[i][j]);
    }
  }
  if (p.res_out) {
#pragma unroll
    for (int i = 0; i < NV; ++i) store_piece<T, Map>(static_cast<T *>(p.res_out) + row * p.ldo, i, t, p.cols, v[i]);
  }
  if (!p.y) return;
  if (p.pre != F8_NORM_NONE) normalise<T, TPR, NV>(v, p.pre, p.pre_eps, p.pre_w, p.pre_b, p, t, lds + 2 * W);
  if (!p.codes) {
#pragma unroll
    for (int i = 0; i < NV; ++i) store_piece<T, Map>(static_cast<T *>(p.y) + row * p.ldy, i, t, p.cols, v[i]);
    return;
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, Map::col(i, j, t) < p.cols ? magnitude(v[i][j]) : 0u);
  const TokenScale s = token_scale(row_amax<TPR>(top, lds + 4 * W));
  if (t == 0) p.scale[row] = s.scale;
  lift(v, s);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    int q[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) q[j] = code_of(v[i][j], s);
    store_codes<Map>(static_cast<int8_t *>(p.y) + row * p.ldy, i, t, p.cols, q);
  }
}

// (false where the threads' pieces do not cover a row)
template <typename T, int TPR, int NV>
bool launch(const NormParams &p, hipStream_t s) {
  if (p.cols > RowMap<TPR, NV>::most) return false;
  constexpr int THREADS = TPR == 64 ? 256 : TPR, RPB = THREADS / TPR;
  hipLaunchKernelGGL((norm_tokens_kernel<T, TPR, NV>), block_grid(((int64_t)p.rows + RPB - 1) / RPB), dim3(THREADS), 0, s, p);
  return true;
}

// Threads to a row: as many as leave each one or two pieces (registers, and so workgroups to a CU, are what counts: 4096 columns with
// 64 threads of 8 pieces 164 us where 512 of one take 90).  With a norm in front there are two reductions, which fewer threads pass
// faster: 256 of two pieces 101 us, 512 of one 105.
template <typename T>
f8_status launch_row(const NormParams &p, hipStream_t s) {
  static_assert(RowMap<1024, 8>::most == ROW_MOST, "the last shape takes every row");
  launch<T, 64, 1>(p, s) || launch<T, 64, 2>(p, s) || launch<T, 256, 1>(p, s) || (p.post == F8_NORM_NONE && launch<T, 512, 1>(p, s)) ||
      launch<T, 256, 2>(p, s) || launch<T, 512, 2>(p, s) || launch<T, 1024, 2>(p, s) || launch<T, 1024, 8>(p, s);
  return launch_status();
}

bool norm_form(int f) { return f == F8_NORM_NONE || f == F8_NORM_RMS || f == F8_NORM_LAYER; }

}  // namespace
}  // namespace f8

using namespace f8;

extern "C" f8_status f8_norm_tokens(const void *a, const void *res, const void *post_w, const void *post_b, const void *gate, const void *pre_w,
                                    const void *pre_b, void *res_out, void *y, float *scale, const f8_norm_tokens_desc *d, void *stream) {
  if (!d) return F8_ERR_NULL;
  if (d->rows < 0 || d->cols < 1 || d->cols > ROW_MOST) return F8_ERR_SHAPE;
  if (!real_type(d->type) || (d->y_type != F8_S8 && d->y_type != d->type) || (d->w_type != F8_F32 && d->w_type != d->type)) return F8_ERR_DTYPE;
  if (!norm_form(d->post) || !norm_form(d->pre)) return F8_ERR_UNSUPPORTED;
  if (!(d->post_eps >= 0.0f) || !(d->pre_eps >= 0.0f)) return F8_ERR_SHAPE;
  if (d->lda < d->cols || (res && d->ldr < d->cols) || (res_out && d->ldo < d->cols) || (y && d->ldy < d->cols)) return F8_ERR_SHAPE;
  if (gate && (d->gate_rows < 1 || d->ldg < d->cols)) return F8_ERR_SHAPE;
  if (d->rows == 0) return F8_OK;
  const bool codes = y && d->y_type == F8_S8;
  if (!a || (!y && !res_out) || (codes && !scale)) return F8_ERR_NULL;
  const size_t e = bytes_of(d->type), we = bytes_of(d->w_type);
  for (const void *t : {a, res, gate, static_cast<const void *>(res_out)})
    if (!aligned_to(t, e)) return F8_ERR_ALIGN;
  for (const void *t : {post_w, post_b, pre_w, pre_b})
    if (!aligned_to(t, we)) return F8_ERR_ALIGN;
  if (!aligned_to(y, codes ? 1 : e) || !aligned_to(scale, 4)) return F8_ERR_ALIGN;
  const NormParams p{a, res, post_w, post_b, gate, pre_w, pre_b, res_out, y, scale, d->lda, d->ldr, d->ldg, d->ldo, d->ldy,
                     d->rows, d->cols, d->post, d->pre, codes, d->w_type == F8_F32, d->post_eps, d->pre_eps, d->res_scale,
                     1.0f / (float)d->cols, FastDiv((uint32_t)(gate ? d->gate_rows : 1))};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return d->type == F8_F32 ? launch_row<float>(p, s) : d->type == F8_F16 ? launch_row<f16>(p, s) : launch_row<bf16>(p, s);
}
