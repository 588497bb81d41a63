// Products of few tokens: the weights are the traffic, each byte of them is needed once.
//
// A workgroup takes 16 output channels and up to 16 tokens, its eight waves a contiguous share of K each.  Weights go from memory straight into the
// registers that are the row operand of the 16 x 16 x 64 matrix instruction (lane l: channel l % 16, 16 bytes of K), U slices of 64
// columns in flight per wave; the tokens are the column operand, from L2 or, where they come as real numbers, from LDS: every
// workgroup then quantises them itself while its first weights are on their way, which saves a launch.  The waves' 32-bit sums meet
// in LDS by integer additions, whose order cannot matter.  Bound by HBM from some 30 MB on (1 x 16384 x 4096 13.8 us, 4.9 TB/s), below that
// by launch and latencies (1 x 4096 x 4096 5.5 us, 6.4 with the quantiser).
#include "linear.h"

namespace f8 {
namespace {

typedef int v4i_dword __attribute__((ext_vector_type(4), aligned(4), may_alias));

constexpr int WAVES = 8, THREADS = 64 * WAVES, U = 8, HELD = LINEAR_FEW_HELD / WAVES;

// 16 bytes at any address, from the dwords that cover them (each of those holds a byte that is asked for).  Sixteen rows an
// instruction at odd addresses are what the load unit is slow at: 5 x 4467 x 4886 17.4 us with plain loads.
template <bool ODD>
__device__ __forceinline__ v4i load16(const int8_t *p) {
  if constexpr (!ODD) {
    return *reinterpret_cast<const v4i_dword *>(p);
  } else {
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3);
    const int8_t *q = p - off;
    const v4i v = *reinterpret_cast<const v4i_dword *>(q);
    const int last = *reinterpret_cast<const int *>(q + (off ? 16 : 12));
    return v4i{(int)__builtin_amdgcn_alignbyte(v[1], v[0], off), (int)__builtin_amdgcn_alignbyte(v[2], v[1], off),
               (int)__builtin_amdgcn_alignbyte(v[3], v[2], off), (int)__builtin_amdgcn_alignbyte(last, v[3], off)};
  }
}

// X: int8_t, or the real type of tokens that are quantised here.  ODD: rows that do not all start on 4 bytes.
template <typename T, typename X, bool ODD>
__global__ __launch_bounds__(THREADS) void linear_few_kernel(LinearParams p) {
  const int m0 = blockIdx.y * LINEAR_FEW;
  p.M = min(p.M - m0, LINEAR_FEW);
  constexpr bool REAL = sizeof(X) > 1;
  __shared__ int sums[256];
  __shared__ uint32_t tops[LINEAR_FEW];
  __shared__ float scales[LINEAR_FEW];
  extern __shared__ __attribute__((aligned(16))) int8_t codes[];        // [M][pitch]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
  const int n0 = blockIdx.x * 16;
  if (threadIdx.x < 256) sums[threadIdx.x] = 0;
  const int slices = (p.K + 63) / 64, per = (slices + WAVES - 1) / WAVES, first = wave * per, last = min(slices, first + per);
  // (channels and tokens past the end read the last one's row; their sums are not used)
  const int8_t *w = p.w + min(n0 + c, p.N - 1) * p.ldw + g * 16;
  const int m = min(c, p.M - 1), pitch = slices * 64 + 16;
  auto whole = [&](int t) { return t + U <= last && (t + U) * 64 <= p.K; };
  v4i fw[U];
  if (whole(first)) {
#pragma unroll
    for (int u = 0; u < U; ++u) fw[u] = load16<ODD>(w + (first + u) * 64);
  }
  if constexpr (REAL) {
    const X *x = reinterpret_cast<const X *>(p.x);
    if (threadIdx.x < LINEAR_FEW) tops[threadIdx.x] = 0;
    __syncthreads();
    // stretches of 512 columns of a row, a wave holds up to HELD of them between the maximum and the codes
    const int stretches = (p.K + 511) / 512, tasks = p.M * stretches;
    float v[HELD][8];
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      const int task = wave + WAVES * h;
      if (task >= tasks) break;
      const int r = task / stretches, k = (task - r * stretches) * 512 + lane * 8;
      load_row8(x + r * p.ldx, k, p.K, v[h]);
    }
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      const int task = wave + WAVES * h;
      if (task >= tasks) break;
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[h][j]));
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
      if (lane == 0) atomicMax(&tops[task / stretches], top);
    }
    __syncthreads();
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      const int task = wave + WAVES * h;
      if (task >= tasks) break;
      const int r = task / stretches, k = (task - r * stretches) * 512 + lane * 8;
      const TokenScale s = token_scale(__uint_as_float(tops[r]));
      if (k == 0) scales[r] = s.scale;
      lift(v[h], s);
      int q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = code_of(v[h][j], s);
      if (k < slices * 64) *reinterpret_cast<v2i *>(codes + r * pitch + k) = v2i{(int)pack4(q[0], q[1], q[2], q[3]), (int)pack4(q[4], q[5], q[6], q[7])};
    }
  }
  __syncthreads();
  const int8_t *x = REAL ? codes + m * pitch + g * 16 : p.x + (m0 + m) * p.ldx + g * 16;
  v4i acc{0, 0, 0, 0};
  int t = first;
  while (whole(t)) {
    v4i fx[U];
#pragma unroll
    for (int u = 0; u < U; ++u) fx[u] = REAL ? *reinterpret_cast<const v4i *>(x + (t + u) * 64) : load16<ODD>(x + (t + u) * 64);
#pragma unroll
    for (int u = 0; u < U; ++u) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u], fx[u], acc, 0, 0, 0);
    t += U;
    if (whole(t)) {
#pragma unroll
      for (int u = 0; u < U; ++u) fw[u] = load16<ODD>(w + (t + u) * 64);
    }
  }
  for (; t < last; ++t) {
    const v4i a = load_row16(w - g * 16, true, t * 64 + g * 16, p.K);
    const v4i b = REAL ? *reinterpret_cast<const v4i *>(x + t * 64) : load_row16(x - g * 16, true, t * 64 + g * 16, p.K);
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, acc, 0, 0, 0);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) atomicAdd(&sums[c * 16 + 4 * g + e], acc[e]);
  __syncthreads();
  if (threadIdx.x < 256) {
    const int row = threadIdx.x / 16, n = n0 + threadIdx.x % 16;
    if (row < p.M && n < p.N)
      static_cast<T *>(p.y)[(m0 + row) * p.ldy + n] =
          (T)__builtin_fmaf((float)sums[threadIdx.x] * (REAL ? scales[row] : p.sx[m0 + row]), p.sw[n], p.bias ? p.bias[n] : 0.0f);
  }
}

template <typename T, typename X>
f8_status launch(const LinearParams &p, hipStream_t s) {
  const size_t lds = sizeof(X) > 1 ? (size_t)p.M * ((p.K + 63) / 64 * 64 + 16) : 0;
  const dim3 grid((p.N + 15) / 16, (p.M + LINEAR_FEW - 1) / LINEAR_FEW);
  const bool even = aligned_to(p.w, 4) && p.ldw % 4 == 0 && (sizeof(X) > 1 || (aligned_to(p.x, 4) && p.ldx % 4 == 0));
  if (even) hipLaunchKernelGGL((linear_few_kernel<T, X, false>), grid, dim3(THREADS), lds, s, p);
  else hipLaunchKernelGGL((linear_few_kernel<T, X, true>), grid, dim3(THREADS), lds, s, p);
  return launch_status();
}

template <typename T>
f8_status launch_type(const LinearParams &p, int x_type, hipStream_t s) {
  return x_type == F8_S8 ? launch<T, int8_t>(p, s) : x_type == F8_F32 ? launch<T, float>(p, s) : x_type == F8_F16 ? launch<T, f16>(p, s) : launch<T, bf16>(p, s);
}

}  // namespace

f8_status launch_linear_few(const LinearParams &p, int x_type, int y_type, hipStream_t s) {
  return y_type == F8_F32 ? launch_type<float>(p, x_type, s) : y_type == F8_F16 ? launch_type<f16>(p, x_type, s) : launch_type<bf16>(p, x_type, s);
}

}  // namespace f8
