// Matrix product of 8-bit tokens with 8-bit weights, a scale per token and per output channel:
//
//   y[m][n] = sx[m] sw[n] sum_k X[m][k] W[n][k] + b[n],     the sum exact in 32 bits (K <= 131071),
//
// scaled in 32-bit floating point and rounded once to the type of y.
//
// Three kernels: at most 16 tokens, where the weights are the traffic (linear_few.hip); tiles through LDS for rows that start on 4
// bytes (linear_tile.hip); and linear_any_kernel here for any stride and alignment: 128 x 128 outputs per workgroup, weights as the
// row operand of the 32 x 32 x 32 matrix instruction in the channel order of f8_device.h (weight_row), so that a lane ends with 16
// neighbouring channels of one token and stores them from its registers; operands go through registers into two LDS buffers.  It
// takes 1.4 to 2.6 times as long as the tiles (1531 x 4096 x 5008 49 us against 35.5, 64 x 4096 x 4096 37 against 8.6, 8192 x 8192 x
// 8192 857 against 462): unaligned 16-byte pieces, one K step of 64 ahead.
#include "linear.h"

namespace f8 {
namespace {

constexpr int ANY_TILE = 128, ANY_K = 64, ANY_PITCH = ANY_K + 16;

template <typename T>
__global__ __launch_bounds__(256) void linear_any_kernel(LinearParams p, int tiles_m) {
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
    for (int j = 0; j < 2; ++j) store_scaled<T>(p, acc[i][j], m0 + wm + 32 * j + l32, n0 + wn + 32 * i + 16 * half);
}

template <typename T>
f8_status launch_any(const LinearParams &p, hipStream_t s) {
  const int64_t tm = (p.M + ANY_TILE - 1) / ANY_TILE, tn = (p.N + ANY_TILE - 1) / ANY_TILE;
  if (tm * tn > 0x7fffffff) return F8_ERR_UNSUPPORTED;
  hipLaunchKernelGGL(linear_any_kernel<T>, dim3((unsigned)(tm * tn)), dim3(256), 0, s, p, (int)tm);
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

// What linear_few_kernel takes: its weights at 5.9 TB/s, and every workgroup's reads of the tokens from L2 at 20.  Measured (us):
// 1 x 4096 x 4096 5.5, 16 x 4096 x 4096 6.5, 1 x 16384 x 4096 13.8, 16 x 4096 x 16384 17.2; the best tile takes 8.0, 8.2, 18.5 and 12.6.
float few_us(const LinearParams &p) {
  const float bytes = (float)p.N * (float)p.K;
  return 2.5f + bytes / 5.9e6f + bytes * (float)p.M / 16.0f / 20e6f;
}

// Whether linear_few_kernel also quantises the tokens.  A launch less is 2.3 us; every workgroup repeating the work costs about half of
// that for each stretch of 512 columns that a wave holds, and as often as there are rounds of workgroups.  Two launches | one (us):
// 1 x 4096 x 4096 8.4 | 6.4, 2 x 4096 x 4096 8.6 | 7.3, 4 x 2048 x 1000 5.7 | 4.9, 1 x 4096 x 16384 16.0 | 15.1, but 4 x 4096 x 4096
// 8.9 | 9.4 and 2 x 4096 x 16384 16.2 | 18.6.
bool few_quantises(int M, int N, int K) {
  const int64_t stretches = (int64_t)M * ((K + 511) / 512);
  return M <= LINEAR_FEW && stretches <= (N <= 8192 ? LINEAR_FEW_HELD : LINEAR_FEW_HELD / 2);
}

f8_status enqueue_linear(const LinearParams &p, int y_type, hipStream_t s) {
  // tiles: rows on 4 bytes, and within reach of 31-bit offsets inside a tile
  const bool tiles = aligned_to(p.x, 4) && aligned_to(p.w, 4) && p.ldx % 4 == 0 && p.ldw % 4 == 0 && p.ldx < (1 << 22) && p.ldw < (1 << 22);
  const LinearPlan plan = linear_plan(p.M, p.N, p.K);
  if (p.M <= LINEAR_FEW && (!tiles || few_us(p) < plan.us)) return launch_linear_few(p, F8_S8, y_type, s);
  if (tiles) {
    LinearParams part = p;
    part.M = plan.M1, part.N = plan.N1;
    const f8_status st = launch_linear_tile(part, y_type, plan.tile, s);
    if (st != F8_OK || (plan.M1 == p.M && plan.N1 == p.N)) return st;
    part = p;
    char *y = static_cast<char *>(p.y);
    if (plan.N1 < p.N) {
      part.N -= plan.N1, part.w += plan.N1 * p.ldw, part.sw += plan.N1, part.y = y + plan.N1 * bytes_of(y_type);
      if (p.bias) part.bias += plan.N1;
    } else {
      part.M -= plan.M1, part.x += plan.M1 * p.ldx, part.sx += plan.M1, part.y = y + plan.M1 * p.ldy * bytes_of(y_type);
    }
    return launch_linear_tile(part, y_type, plan.tile2, s);
  }
  return y_type == F8_F32 ? launch_any<float>(p, s) : y_type == F8_F16 ? launch_any<f16>(p, s) : launch_any<bf16>(p, s);
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
  hipStream_t s = static_cast<hipStream_t>(stream);
  LinearParams p{static_cast<const int8_t *>(x), w, nullptr, sw, bias, y, d->ldx, d->ldw, d->ldy, d->M, d->N, d->K};
  if (few_quantises(d->M, d->N, d->K)) return launch_linear_few(p, d->x_type, d->y_type, s);
  const int64_t pitch = code_pitch(d->K);
  int8_t *codes = static_cast<int8_t *>(workspace);
  float *sx = reinterpret_cast<float *>(codes + d->M * pitch);
  st = enqueue_quant_tokens(x, d->ldx, d->x_type, codes, pitch, (int)pitch, sx, d->M, d->K, s);
  if (st != F8_OK) return st;
  p.x = codes, p.sx = sx, p.ldx = pitch;
  return enqueue_linear(p, d->y_type, s);
}

}  // extern "C"
