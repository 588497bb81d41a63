// Matrix product of 8-bit tokens with 8-bit weights, a scale per token and per output channel:
//
//   y[m][n] = sx[m] sw[n] sum_k X[m][k] W[n][k] + b[n],     the sum exact in 32 bits (K <= 131071),
//
// scaled in 32-bit floating point and rounded once to the type of y.
//
// Three kernels: few tokens, where the weights are the traffic (linear_few.hip); tiles through LDS for rows that start on 4 bytes
// (linear_tile.hip); and linear_any_kernel here for any stride and alignment: 128 x 128 or 64 x 64 outputs per workgroup, weights as
// the row operand of the 32 x 32 x 32 matrix instruction in the channel order of f8_device.h (weight_row), so that a lane ends with
// 16 neighbouring channels of one token and stores them from its registers; operands go through two sets of registers into two LDS
// buffers, two steps of 128 columns ahead.  Every 16-byte piece off the grid is two lines: 4096 x 4097 x 4096 takes 141 us, 4096 x
// 4096 x 4096 on tiles 65; 1531 x 4097 x 5001 73 us, 1531 x 4100 x 5001 43.
#include <math.h>

#include "linear.h"

namespace f8 {
namespace {

constexpr int ANY_K = 128, ANY_PITCH = ANY_K + 16;       // (rows 36 words apart: sixteen neighbours' pieces lie on all 64 banks)

template <typename T, int TILE>
__global__ __launch_bounds__(256, 2) void linear_any_kernel(LinearParams p, int tiles_m) {
  constexpr int WT = TILE / 2, BL = WT / 32, PIECES = TILE * ANY_K / 16 / 256;      // a wave's share of a side, its blocks, 16-byte pieces per thread
  __shared__ __attribute__((aligned(16))) uint8_t lds[2][2 * TILE * ANY_PITCH];
  const int tile = (int)xcd_remap(blockIdx.x, gridDim.x);
  const int m0 = tile % tiles_m * TILE, n0 = tile / tiles_m * TILE;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
  const int wn = (wave & 1) * WT, wm = (wave >> 1) * WT;
  const int row = threadIdx.x >> 3, piece = (threadIdx.x & 7) * 16;               // 32 rows at a time
  // (rows past the end read the last one's; their results are not stored)
  const int8_t *w[PIECES], *x[PIECES];
#pragma unroll
  for (int h = 0; h < PIECES; ++h) w[h] = p.w + min(n0 + row + 32 * h, p.N - 1) * p.ldw, x[h] = p.x + min(m0 + row + 32 * h, p.M - 1) * p.ldx;
  v4i st[2][2 * PIECES];
  auto load = [&](int set, int k0) {
    if (k0 + ANY_K <= p.K) {
#pragma unroll
      for (int h = 0; h < PIECES; ++h) {
        __builtin_memcpy(&st[set][h], w[h] + k0 + piece, 16);
        __builtin_memcpy(&st[set][PIECES + h], x[h] + k0 + piece, 16);
      }
    } else {
#pragma unroll
      for (int h = 0; h < PIECES; ++h) {
        st[set][h] = load_row16(w[h], true, k0 + piece, p.K);
        st[set][PIECES + h] = load_row16(x[h], true, k0 + piece, p.K);
      }
    }
  };
  auto put = [&](int set) {
#pragma unroll
    for (int h = 0; h < 2 * PIECES; ++h)
      *reinterpret_cast<v4i *>(&lds[set][(h % PIECES * 32 + row + h / PIECES * TILE) * ANY_PITCH + piece]) = st[set][h];
  };
  v16i acc[BL][BL] = {};
  auto step = [&](int set, int k0) {      // the operands of k0 lie in LDS, those of the next step are in the registers of the other set
    load(set, k0 + 2 * ANY_K);
    __syncthreads();
    const uint8_t *b = lds[set];
#pragma unroll
    for (int ks = 0; ks < ANY_K / 32; ++ks) {
      v4i fw[BL], fx[BL];
#pragma unroll
      for (int i = 0; i < BL; ++i) {
        fw[i] = *reinterpret_cast<const v4i *>(b + (wn + 32 * i + weight_row(l32)) * ANY_PITCH + ks * 32 + half * 16);
        fx[i] = *reinterpret_cast<const v4i *>(b + (TILE + wm + 32 * i + l32) * ANY_PITCH + ks * 32 + half * 16);
      }
#pragma unroll
      for (int i = 0; i < BL; ++i)
#pragma unroll
        for (int j = 0; j < BL; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[i], fx[j], acc[i][j], 0, 0, 0);
    }
    put(set ^ 1);
  };
  load(0, 0);
  load(1, ANY_K);
  put(0);
  for (int k = 0; k < p.K; k += 2 * ANY_K) {
    step(0, k);
    if (k + ANY_K < p.K) step(1, k + ANY_K);
  }
#pragma unroll
  for (int i = 0; i < BL; ++i)
#pragma unroll
    for (int j = 0; j < BL; ++j) store_scaled<T>(p, acc[i][j], m0 + wm + 32 * j + l32, n0 + wn + 32 * i + 16 * half);
}

template <typename T, int TILE>
f8_status launch_any_tile(const LinearParams &p, hipStream_t s) {
  const int tm = (p.M + TILE - 1) / TILE, tn = (p.N + TILE - 1) / TILE;
  hipLaunchKernelGGL((linear_any_kernel<T, TILE>), dim3((unsigned)(tm * tn)), dim3(256), 0, s, p, tm);
  return launch_status();
}

// Tiles of 64 where those of 128 would leave CUs without one.
int64_t any_tiles(const LinearParams &p, int tile) { return (int64_t)((p.M + tile - 1) / tile) * ((p.N + tile - 1) / tile); }
int any_tile(const LinearParams &p) { return any_tiles(p, 128) < 256 ? 64 : 128; }
template <typename T>
f8_status launch_any(const LinearParams &p, hipStream_t s) {
  return any_tile(p) == 64 ? launch_any_tile<T, 64>(p, s) : launch_any_tile<T, 128>(p, s);
}

f8_status check(const f8_linear_desc *d) {
  if (!d) return F8_ERR_NULL;
  if (d->M < 0 || d->N < 0 || d->M > F8_LINEAR_MAX_ROWS || d->N > F8_LINEAR_MAX_ROWS || d->K < 1 || d->K > F8_LINEAR_MAX_K) return F8_ERR_SHAPE;
  if (!real_type(d->y_type)) return F8_ERR_DTYPE;
  if (d->ldx < d->K || d->ldw < d->K || d->ldy < d->N) return F8_ERR_SHAPE;
  return F8_OK;
}

f8_status check_pointers(const void *x, const void *w, const float *sw, const float *bias, const void *y, int y_type) {
  if (!x || !w || !sw || !y) return F8_ERR_NULL;
  if (!aligned_to(sw, 4) || !aligned_to(bias, 4) || !aligned_to(y, bytes_of(y_type))) return F8_ERR_ALIGN;
  return F8_OK;
}

// What linear_few_kernel takes: its weights at 5.9 TB/s (once more from L2 for every further 16 tokens), every workgroup's reads of
// the tokens from L2, and at least a memory latency for each batch of 8 slices that a wave walks through; rows at odd addresses cost
// 3.5 and 1.5 times that.  Measured (us), and the best tile: 1 x 4096 x 4096 5.5 | 8.0, 16 x 4096 x 4096 6.5 | 8.2, 1 x 16384 x 4096
// 13.8 | 18.5, 65 x 6144 x 432 7.8 | 9.5, 163 x 528 x 449 3.7 | 5.2, but 16 x 4096 x 16384 17.2 | 12.6 and 130 x 9712 x 1198 28.4 | 13.8; at odd
// addresses, and linear_any_kernel: 9 x 10123 x 2476 15 | 29, 189 x 13017 x 275 21 | 43, but 95 x 849 x 2742 12.9 | 7.0.
float few_us(const LinearParams &p, bool odd) {
  const float bytes = (float)p.N * (float)p.K, blocks = (float)((p.M + LINEAR_FEW - 1) / LINEAR_FEW);
  const float traffic = bytes / 5.9e6f + bytes * (blocks - 1.0f) / 12e6f + bytes * (float)p.M / 16.0f / 20e6f;
  const float batches = 0.9f * (float)((p.K + 4095) / 4096), t = odd ? 3.5f * traffic : traffic, l = odd ? 1.5f * batches : batches;
  return 2.5f + (t > l ? t : l);
}

// The same of linear_any_kernel: rounds of two workgroups to a CU, a step of the small or the large tile.
float any_us(const LinearParams &p) {
  const float large = (float)((p.M + 127) / 128) * (float)((p.N + 127) / 128), steps = (float)((p.K + ANY_K - 1) / ANY_K);
  if (large >= 256.0f) return 4.0f + ceilf(large / 512.0f) * steps * 1.3f;
  return 4.0f + ceilf((float)((p.M + 63) / 64) * (float)((p.N + 63) / 64) / 512.0f) * steps * 0.4f;
}

// Whether linear_few_kernel also quantises the tokens.  A launch less is 2.3 us; every workgroup repeating the work costs about half of
// that for each stretch of 512 columns that a wave holds, and as often as there are rounds of workgroups.  Two launches | one (us):
// 1 x 4096 x 4096 8.4 | 6.4, 2 x 4096 x 4096 8.6 | 7.3, 4 x 2048 x 1000 5.7 | 4.9, 1 x 4096 x 16384 16.0 | 15.1, but 4 x 4096 x 4096
// 8.9 | 9.4 and 2 x 4096 x 16384 16.2 | 18.6.
bool few_quantises(int M, int N, int K) {
  const int64_t stretches = (int64_t)M * ((K + 511) / 512);
  return M <= LINEAR_FEW && stretches <= (N <= 8192 ? LINEAR_FEW_HELD : LINEAR_FEW_HELD / 2);
}

// Which kernel takes a product.  What does not fit a launch is known before anything is enqueued.
struct Route {
  bool tiles, few, fits;
  LinearPlan plan;
};
Route route_of(const LinearParams &p) {
  // tiles: rows on 4 bytes, and within reach of 31-bit offsets inside a tile
  Route r;
  r.tiles = aligned_to(p.x, 4) && aligned_to(p.w, 4) && p.ldx % 4 == 0 && p.ldw % 4 == 0 && p.ldx < (1 << 22) && p.ldw < (1 << 22);
  r.plan = linear_plan(p.M, p.N, p.K);
  r.few = p.M <= LINEAR_FEW_MOST && few_us(p, !r.tiles) < (r.tiles ? r.plan.us : any_us(p));
  r.fits = r.few || (r.tiles ? r.plan.wgs : any_tiles(p, any_tile(p))) <= LINEAR_TILES_MOST;
  return r;
}

f8_status enqueue_linear(const LinearParams &p, const Route &r, int y_type, hipStream_t s) {
  const LinearPlan &plan = r.plan;
  if (r.few) return launch_linear_few(p, F8_S8, y_type, s);
  if (r.tiles) {
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
  const Route r = route_of(p);
  return r.fits ? enqueue_linear(p, r, d->y_type, static_cast<hipStream_t>(stream)) : F8_ERR_UNSUPPORTED;
}

size_t f8_linear_workspace_bytes(int M, int K) {
  if (M < 1 || K < 1 || few_quantises(M, INT32_MAX, K)) return 0;
  return (size_t)M * (size_t)code_pitch(K) + (size_t)M * sizeof(float);
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
  const size_t need = f8_linear_workspace_bytes(d->M, d->K);
  if (need && !workspace) return F8_ERR_NULL;
  if (!aligned_to(x, bytes_of(d->x_type)) || !aligned_to(workspace, 16)) return F8_ERR_ALIGN;
  if (workspace_bytes < need) return F8_ERR_SHAPE;
  hipStream_t s = static_cast<hipStream_t>(stream);
  LinearParams p{static_cast<const int8_t *>(x), w, nullptr, sw, bias, y, d->ldx, d->ldw, d->ldy, d->M, d->N, d->K};
  if (few_quantises(d->M, d->N, d->K)) return launch_linear_few(p, d->x_type, d->y_type, s);
  const int64_t pitch = code_pitch(d->K);
  int8_t *codes = static_cast<int8_t *>(workspace);
  float *sx = reinterpret_cast<float *>(codes + d->M * pitch);
  p.x = codes, p.sx = sx, p.ldx = pitch;
  const Route r = route_of(p);
  if (!r.fits) return F8_ERR_UNSUPPORTED;
  st = enqueue_quant_tokens(x, d->ldx, d->x_type, codes, pitch, (int)pitch, sx, d->M, d->K, s);
  return st == F8_OK ? enqueue_linear(p, r, d->y_type, s) : st;
}

}  // extern "C"
