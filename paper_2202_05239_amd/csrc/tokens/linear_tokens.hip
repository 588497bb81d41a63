// Matrix product of 8-bit tokens with 8-bit weights, a scale per token and per output channel:
//
//   y[m][n] = sx[m] sw[n] sum_k X[m][k] W[n][k] + b[n],     the sum exact in 32 bits (K <= 131071),
//
// scaled in 32-bit floating point and rounded once to the type of y.
//
// linear_any_kernel takes any size, stride and alignment: 128 x 128 outputs per workgroup, weights as the row operand of the
// 32 x 32 x 32 matrix instruction in the channel order of f8_device.h (weight_row), so that a lane ends with 16 neighbouring
// channels of one token and stores them from its registers; operands go through registers into two LDS buffers.
#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

typedef int v16i __attribute__((ext_vector_type(16)));

struct LinearParams {
  const int8_t *x, *w;
  const float *sx, *sw, *bias;
  void *y;
  int64_t ldx, ldw, ldy;
  int M, N, K;
};

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

// The 16 channels n .. n + 15 of token m.
template <typename T>
__device__ __forceinline__ void store_scaled(const LinearParams &p, const v16i &acc, int m, int n, bool vec) {
  if (m >= p.M || n >= p.N) return;
  const float sx = p.sx[m];
  T *y = static_cast<T *>(p.y) + m * p.ldy + n;
  T o[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const bool real = n + i < p.N;
    o[i] = (T)__builtin_fmaf((float)acc[i] * sx, real ? p.sw[n + i] : 0.0f, real && p.bias ? p.bias[n + i] : 0.0f);
  }
  if (vec && n + 16 <= p.N) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<v4i *>(y)[i] = reinterpret_cast<const v4i *>(o)[i];
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (n + i < p.N) y[i] = o[i];
  }
}

constexpr int ANY_TILE = 128, ANY_K = 64, ANY_PITCH = ANY_K + 16;

template <typename T>
__global__ __launch_bounds__(256) void linear_any_kernel(LinearParams p, int tiles_m, int vec) {
  __shared__ uint8_t lds[2][2 * ANY_TILE * ANY_PITCH];
  const int tile = (int)xcd_remap(blockIdx.x, gridDim.x);
  const int m0 = tile % tiles_m * ANY_TILE, n0 = tile / tiles_m * ANY_TILE;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
  const int wn = (wave & 1) * 64, wm = (wave >> 1) * 64;
  const int row = threadIdx.x >> 2, piece = threadIdx.x & 3;    // 64 rows x 4 pieces of 16 bytes at a time
  v4i st[4];
  auto load = [&](int k0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int n = n0 + row + 64 * h, m = m0 + row + 64 * h, k = k0 + piece * 16;
      st[h] = load_row16(p.w + n * p.ldw, n < p.N, k, p.K);
      st[2 + h] = load_row16(p.x + m * p.ldx, m < p.M, k, p.K);
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int h = 0; h < 4; ++h) *reinterpret_cast<v4i *>(&lds[buf][((h & 1) * 64 + row + (h >> 1) * ANY_TILE) * ANY_PITCH + piece * 16]) = st[h];
  };
  v16i acc[2][2] = {};
  const int steps = (p.K + ANY_K - 1) / ANY_K;
  load(0);
  put(0);
  for (int s = 0; s < steps; ++s) {
    if (s + 1 < steps) load((s + 1) * ANY_K);
    __syncthreads();
    const uint8_t *b = lds[s & 1];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      v4i fw[2], fx[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fw[i] = *reinterpret_cast<const v4i *>(b + (wn + 32 * i + weight_row(l32)) * ANY_PITCH + ks * 32 + half * 16);
        fx[i] = *reinterpret_cast<const v4i *>(b + (ANY_TILE + wm + 32 * i + l32) * ANY_PITCH + ks * 32 + half * 16);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[i], fx[j], acc[i][j], 0, 0, 0);
    }
    if (s + 1 < steps) put((s + 1) & 1);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) store_scaled<T>(p, acc[i][j], m0 + wm + 32 * j + l32, n0 + wn + 32 * i + 16 * half, vec);
}

template <typename T>
f8_status launch_linear(const LinearParams &p, hipStream_t s) {
  const bool vec = aligned_to(p.y, 16) && p.ldy * sizeof(T) % 16 == 0;
  const int64_t tm = (p.M + ANY_TILE - 1) / ANY_TILE, tn = (p.N + ANY_TILE - 1) / ANY_TILE;
  if (tm * tn > 0x7fffffff) return F8_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(linear_any_kernel<T>, dim3((unsigned)(tm * tn)), dim3(256), 0, s, p, (int)tm, vec);
  return launch_status();
}

f8_status check(const f8_linear_desc *d) {
  if (!d) return F8_ERR_NULL;
  if (d->M < 0 || d->N < 0 || d->K < 1 || d->K > F8_LINEAR_MAX_K) return F8_ERR_SHAPE;
  if (!real_type(d->y_type)) return F8_ERR_DTYPE;
  if (d->ldx < d->K || d->ldw < d->K || d->ldy < d->N) return F8_ERR_SHAPE;
  return F8_OK;
}

f8_status check_pointers(const void *x, const void *w, const float *sw, const float *bias, const void *y, int y_type) {
  if (!x || !w || !sw || !y) return F8_ERR_NULL;
  if (!aligned_to(sw, 4) || !aligned_to(bias, 4) || !aligned_to(y, bytes_of(y_type))) return F8_ERR_ALIGN;
  return F8_OK;
}

f8_status enqueue_linear(const LinearParams &p, int y_type, hipStream_t s) {
  return y_type == F8_F32 ? launch_linear<float>(p, s) : y_type == F8_F16 ? launch_linear<f16>(p, s) : launch_linear<bf16>(p, s);
}

// Rows of codes in the workspace: whole 128 bytes, zeros behind the row's end.
int64_t code_pitch(int K) { return ((int64_t)K + 127) / 128 * 128; }

}  // namespace
}  // namespace f8

using namespace f8;

extern "C" {

f8_status f8_linear_scaled(const int8_t *x, const float *sx, const int8_t *w, const float *sw, const float *bias, void *y,
                           const f8_linear_desc *d, void *stream) {
  f8_status st = check(d);
  if (st != F8_OK) return st;
  if (d->x_type != F8_S8) return F8_ERR_DTYPE;
  if (d->M == 0 || d->N == 0) return F8_OK;
  st = check_pointers(x, w, sw, bias, y, d->y_type);
  if (st != F8_OK) return st;
  if (!sx) return F8_ERR_NULL;
  if (!aligned_to(sx, 4)) return F8_ERR_ALIGN;
  const LinearParams p{x, w, sx, sw, bias, y, d->ldx, d->ldw, d->ldy, d->M, d->N, d->K};
  return enqueue_linear(p, d->y_type, static_cast<hipStream_t>(stream));
}

size_t f8_linear_workspace_bytes(int M, int K) {
  return M < 1 || K < 1 ? 0 : (size_t)M * (size_t)code_pitch(K) + (size_t)M * sizeof(float);
}

f8_status f8_linear_tokens(const void *x, const int8_t *w, const float *sw, const float *bias, void *y, const f8_linear_desc *d,
                           void *workspace, size_t workspace_bytes, void *stream) {
  f8_status st = check(d);
  if (st != F8_OK) return st;
  if (!real_type(d->x_type)) return F8_ERR_DTYPE;
  if (d->K > ROW_MOST) return F8_ERR_SHAPE;
  if (d->M == 0 || d->N == 0) return F8_OK;
  st = check_pointers(x, w, sw, bias, y, d->y_type);
  if (st != F8_OK) return st;
  if (!workspace) return F8_ERR_NULL;
  if (!aligned_to(x, bytes_of(d->x_type)) || !aligned_to(workspace, 16)) return F8_ERR_ALIGN;
  if (workspace_bytes < f8_linear_workspace_bytes(d->M, d->K)) return F8_ERR_SHAPE;
  const int64_t pitch = code_pitch(d->K);
  int8_t *codes = static_cast<int8_t *>(workspace);
  float *sx = reinterpret_cast<float *>(codes + d->M * pitch);
  hipStream_t s = static_cast<hipStream_t>(stream);
  st = enqueue_quant_tokens(x, d->ldx, d->x_type, codes, pitch, (int)pitch, sx, d->M, d->K, s);
  if (st != F8_OK) return st;
  const LinearParams p{codes, w, sx, sw, bias, y, pitch, d->ldw, d->ldy, d->M, d->N, d->K};
  return enqueue_linear(p, d->y_type, s);
}

}  // extern "C"
