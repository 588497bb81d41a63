// Products of many tokens on tiles through LDS (see linear_tokens.hip for the operator).
//
// The load unit copies both operands' next 128 columns into LDS directly (buffer loads that write LDS, 1 KiB an instruction, a
// descriptor of exactly the tile's rows: what lies outside arrives as zeros), into one of two buffers while the other one is
// multiplied.  Rows of 128 bytes, their 16-byte pieces permuted by the row number, so that no eight lanes of a fragment read
// share a bank.  Weights are the row operand, fetched in the channel order of f8_device.h (weight_row): a lane ends with 16
// neighbouring channels of one token and stores them from its registers.
//
// A K step is four slices of 32 columns with two sets of fragments, the reads of a slice issued between the matrix instructions
// of the one before.  The barrier that hands the buffers over lies in the middle of the last slice: its fragments are in
// registers by then, so the buffer is free for the loads of the step after next, and the first fragments of the next step arrive
// behind the second half of the slice.
//
// 8192 x 8192 x 8192 takes 449 - 478 us (2.3 - 2.45 Pop/s; a loop of nothing but matrix instructions on random bytes reaches 3.4 - 3.5).
// The matrix pipes are 61 - 64 % busy at 1.5 - 1.85 GHz: the clock is what power leaves (the loop holds 1.78 GHz on random bytes, its pipes 90 %
// busy, and 2.3 on zeros), the rest are stalls.  What was tried against those left the time as it is (468 us then): reads that
// collide two ways in LDS (half of all LDS cycles) or none; four waves with 128 x 128 outputs each and two thirds of the reads (467);
// the loads of a step spread over the slices instead of one burst (469); workgroups that stay and fetch the next tile's operands
// before they store the last one's results (468).
#include <math.h>

#include "linear.h"

namespace f8 {
namespace {

typedef __attribute__((address_space(3))) void lds_void;

constexpr int KS = 128;                  // columns of a step

__device__ __forceinline__ v4i lds_read(uint32_t at, const int imm) {
  v4i v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(at), "n"(imm) : "memory");
  return v;
}

template <typename T, int WN, int WM, int NB, int MB, int RING, int KG>
__global__ __launch_bounds__(64 * WN * WM * KG) void linear_tile_kernel(LinearParams p, int tiles_m, int tiles_n) {
  constexpr int BN = 32 * NB * WN, BM = 32 * MB * WM, W = WN * WM, BUF = (BN + BM) * KS, LOADS = (BN + BM) / 8 / W, GROUP = 8;
  static_assert(W % 2 == 0 && BN / 8 % W == 0 && BM / 8 % W == 0, "an instruction's rows are all weights or all tokens");
  __shared__ __attribute__((aligned(1024))) uint8_t lds[KG * RING * BUF];
  // tiles in groups of GROUP rows of tokens, so that what an XCD works on at a time is a compact block
  const int id = (int)xcd_remap(blockIdx.x, gridDim.x);
  const int g = id / (GROUP * tiles_n), rows = min(GROUP, tiles_m - g * GROUP), in = id - g * GROUP * tiles_n;
  const int m0 = (g * GROUP + in % rows) * BM, n0 = in / rows * BN;
  const int lane = threadIdx.x & 63, wave_wg = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l32 = lane & 31, half = lane >> 5;
  const int kg = wave_wg / W, wave = wave_wg % W;
  const int wn = wave % WN * NB * 32, wm = wave / WN * MB * 32;
  const int8_t *w = p.w + n0 * p.ldw, *x = p.x + m0 * p.ldx;
  const int rw = min(BN, p.N - n0), rx = min(BM, p.M - m0);
  const __amdgpu_buffer_rsrc_t wres = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(w), 0, (int)((rw - 1) * p.ldw + p.K), 0x00027000);
  const __amdgpu_buffer_rsrc_t xres = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t *>(x), 0, (int)((rx - 1) * p.ldx + p.K), 0x00027000);
  // each of KG groups of waves takes a share of the steps, through buffers of its own; all go through the same number of barriers
  const int k16 = p.K & ~15, steps = ((k16 + KS - 1) / KS + KG - 1) / KG, from = kg * steps;
  constexpr uint32_t NOWHERE = 0x80000000u;
  const int piece = ((lane & 7) ^ ((wave & 1) * 4 + (lane >> 4))) * 16;      // (W is even: a wave's rows are 8 (wave & 1) + lane / 8 modulo 16)
  uint32_t at[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = (i * W + wave) * 8 + (lane >> 3);
    if (i * W < BN / 8) {
      const int n = (r & ~31) + weight_row(r & 31);
      at[i] = n < rw ? (uint32_t)(n * (int)p.ldw + piece) : NOWHERE;
    } else {
      const int m = r - BN;
      at[i] = m < rx ? (uint32_t)(m * (int)p.ldx + piece) : NOWHERE;
    }
  }
  auto fetch = [&](int i, int s, int buf) {
    const int step_k = (from + s) * KS;
    const bool inside = step_k < k16 && s < steps;                           // (the scalar part of the address stays inside too)
    const int k = __builtin_amdgcn_readfirstlane(inside ? step_k : 0);
    const uint32_t v = inside && k + piece < k16 ? at[i] : NOWHERE;
    lds_void *to = (lds_void *)(lds + (kg * RING + buf) * BUF + (i * W + wave) * 1024);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(i * W < BN / 8 ? wres : xres, to, 16, v, k, 0, 0);
  };
  // where a lane's fragments of slice ks lie, from the block's first row on
  const uint32_t base = (uint32_t)(size_t)(lds_void *)lds + kg * RING * BUF + l32 * 128;
  uint32_t fr[4];
#pragma unroll
  for (int ks = 0; ks < 4; ++ks) fr[ks] = base + (((2 * ks + half) ^ ((l32 >> 1) & 7)) * 16);

  v16i acc[NB][MB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
  constexpr int AHEAD = RING - 1, PRODUCTS = NB * MB, READS = NB + MB;
  v4i fw[2][NB], fx[2][MB];
  auto read = [&](int set, int ks, int buf, int f) {
    const uint32_t a = fr[ks] + (uint32_t)(buf * BUF);
    if (f < NB) fw[set][f] = lds_read(a + wn * 128, f * 4096);
    else fx[set][f - NB] = lds_read(a + BN * 128 + wm * 128, (f - NB) * 4096);
  };
  auto arrived = [&](int set) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int f = 0; f < NB; ++f) asm volatile("" : "+v"(fw[set][f]));
#pragma unroll
    for (int f = 0; f < MB; ++f) asm volatile("" : "+v"(fx[set][f]));
  };
  auto product = [&](int set, int q) {
    acc[q / MB][q % MB] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[set][q / MB], fx[set][q % MB], acc[q / MB][q % MB], 0, 0, 0);
  };
  // (steps behind the last one are requested too, as nothing: the number of loads in flight is then the same at every step)
  auto landed = [&]() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 1) * LOADS) : "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  auto next = [](int buf) { return buf + 1 == RING ? 0 : buf + 1; };
  int buf = 0;                            // of the step at hand
#pragma unroll
  for (int s = 0; s < AHEAD; ++s)
#pragma unroll
    for (int i = 0; i < LOADS; ++i) fetch(i, s, s);
  landed();
#pragma unroll
  for (int i = 0; i < LOADS; ++i) fetch(i, AHEAD, AHEAD);
#pragma unroll
  for (int f = 0; f < READS; ++f) read(0, 0, 0, f);
  arrived(0);
  for (int s = 0; s < steps; ++s) {
#pragma unroll
    for (int ks = 0; ks < 3; ++ks) {
#pragma unroll
      for (int q = 0; q < (PRODUCTS > READS ? PRODUCTS : READS); ++q) {
        if (q < READS) read((ks + 1) & 1, ks + 1, buf, q);
        if (q < PRODUCTS) product(ks & 1, q);
        __builtin_amdgcn_sched_barrier(0);
      }
      arrived((ks + 1) & 1);
    }
#pragma unroll
    for (int q = 0; q < PRODUCTS / 2; ++q) product(1, q);
    __builtin_amdgcn_sched_barrier(0);
    landed();
    const int then = next(buf);
#pragma unroll
    for (int f = 0; f < READS; ++f) read(0, 0, then, f);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) fetch(i, s + 1 + AHEAD, buf);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = PRODUCTS / 2; q < PRODUCTS; ++q) product(1, q);
    __builtin_amdgcn_sched_barrier(0);
    arrived(0);
    buf = then;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // (nothing may land in LDS that is another workgroup's by then)
  if (p.K != k16 && kg == 0) {            // the last few columns, one slice straight from memory
#pragma unroll
    for (int f = 0; f < NB; ++f) {
      const int n = wn + 32 * f + weight_row(l32);
      fw[0][f] = load_row16(w + n * p.ldw, n < rw && half == 0, k16, p.K);
    }
#pragma unroll
    for (int f = 0; f < MB; ++f) {
      const int m = wm + 32 * f + l32;
      fx[0][f] = load_row16(x + m * p.ldx, m < rx && half == 0, k16, p.K);
    }
#pragma unroll
    for (int q = 0; q < PRODUCTS; ++q) product(0, q);
  }
  if constexpr (KG > 1) {                 // the groups' sums meet in LDS
    int *sums = reinterpret_cast<int *>(lds);
    static_assert((KG - 1) * BN * BM * 4 <= KG * RING * BUF, "the sums fit where the operands were");
    __syncthreads();
    if (kg > 0) {
#pragma unroll
      for (int q = 0; q < PRODUCTS; ++q)
#pragma unroll
        for (int e = 0; e < 16; e += 4)
          *reinterpret_cast<v4i *>(sums + ((((kg - 1) * W + wave) * PRODUCTS + q) * 4 + e / 4) * 256 + lane * 4) =
              v4i{acc[q / MB][q % MB][e], acc[q / MB][q % MB][e + 1], acc[q / MB][q % MB][e + 2], acc[q / MB][q % MB][e + 3]};
    }
    __syncthreads();
    if (kg > 0) return;
#pragma unroll
    for (int o = 0; o < KG - 1; ++o)
#pragma unroll
      for (int q = 0; q < PRODUCTS; ++q)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const v4i v = *reinterpret_cast<const v4i *>(sums + (((o * W + wave) * PRODUCTS + q) * 4 + e / 4) * 256 + lane * 4);
#pragma unroll
          for (int k = 0; k < 4; ++k) acc[q / MB][q % MB][e + k] += v[k];
        }
  }
#pragma unroll
  for (int j = 0; j < MB; ++j)
#pragma unroll
    for (int i = 0; i < NB; ++i) store_scaled<T>(p, acc[i][j], m0 + wm + 32 * j + l32, n0 + wn + 32 * i + 16 * half);
}

template <typename T, int WN, int WM, int NB, int MB, int RING, int KG>
f8_status launch(const LinearParams &p, hipStream_t s) {
  constexpr int BN = 32 * NB * WN, BM = 32 * MB * WM;
  const int tn = (p.N + BN - 1) / BN, tm = (p.M + BM - 1) / BM;
  hipLaunchKernelGGL((linear_tile_kernel<T, WN, WM, NB, MB, RING, KG>), dim3((unsigned)(tn * tm)), dim3(64 * WN * WM * KG), 0, s, p, tm, tn);
  return launch_status();
}

// The tiles, channels x tokens, and what a launch of T workgroups takes on them (us):  rounds (start + steps (step + more o)),
// o = workgroups to a CU in a round.  One line each from launches alone on the chip, K 2048 to 16384, 1 to 8192 tokens; the lines
// are within 12 % of the times measured, except where few tokens leave a tile nearly empty (up to 20 % over).  The best tile and
// the next one, measured: 8192 x 8192 x 8192 462 | 527 us (256 x 256 | 128 x 256), 1531 x 4096 x 5008 35.5 | 38 (128 x 128 | 128 x 256),
// 512 x 4096 x 4096 15.9 | 16.6 (128 x 64), 256 x 4096 x 4096 11.4 | 12.9 (64 x 64 with two shares of K | without), 48 x 4096 x 16384
// 13.1 | 13.8, 64 x 4096 x 4096 8.6 | 10.7 (32 x 64 with four | 64 x 64 with two).
struct Tile {
  int bn, bm, per_cu, kg;
  float start, step, more;
};
constexpr Tile TILES[] = {{256, 256, 1, 1, 9.0f, 1.10f, 0.59f}, {128, 256, 1, 1, 5.0f, 0.70f, 0.33f}, {128, 128, 2, 1, 4.0f, 0.58f, 0.26f},
                          {128, 64, 2, 1, 3.5f, 0.28f, 0.20f},  {64, 64, 2, 1, 3.0f, 0.25f, 0.09f},   {64, 64, 1, 2, 4.0f, 0.40f, 0.06f},
                          {32, 64, 1, 4, 4.5f, 0.45f, 0.08f}};

template <typename T>
f8_status launch_type(const LinearParams &p, int tile, hipStream_t s) {
  switch (tile) {
    case 0: return launch<T, 2, 4, 4, 2, 2, 1>(p, s);
    case 1: return launch<T, 2, 4, 2, 2, 3, 1>(p, s);
    case 2: return launch<T, 2, 2, 2, 2, 2, 1>(p, s);
    case 3: return launch<T, 2, 2, 2, 1, 3, 1>(p, s);
    case 4: return launch<T, 2, 2, 1, 1, 4, 1>(p, s);
    case 5: return launch<T, 2, 2, 1, 1, 4, 2>(p, s);
    default: return launch<T, 1, 2, 1, 1, 3, 4>(p, s);
  }
}

}  // namespace

f8_status launch_linear_tile(const LinearParams &p, int y_type, int tile, hipStream_t s) {
  return y_type == F8_F32 ? launch_type<float>(p, tile, s) : y_type == F8_F16 ? launch_type<f16>(p, tile, s) : launch_type<bf16>(p, tile, s);
}

namespace {

float tile_us(const Tile &t, int M, int N, int K) {
  const float wgs = (float)((M + t.bm - 1) / t.bm) * (float)((N + t.bn - 1) / t.bn), steps = (float)((K + KS * t.kg - 1) / (KS * t.kg));
  const float rounds = ceilf(wgs / (256.0f * t.per_cu)), o = wgs / (256.0f * rounds);
  return rounds * (t.start + steps * (t.step + t.more * o));
}

int best_tile(int M, int N, int K, float *us) {
  int best = 0;
  *us = tile_us(TILES[0], M, N, K);
  for (int i = 1; i < (int)(sizeof(TILES) / sizeof(TILES[0])); ++i) {
    const float t = tile_us(TILES[i], M, N, K);
    if (t < *us) best = i, *us = t;
  }
  return best;
}

}  // namespace

// Tiles that do not divide evenly among the CUs leave most of them idle in the last round; then whole rounds of a large tile and a
// second launch of smaller ones over the rest take less (us, one launch | two): 4096 x 4100 x 5000 123 | 108, 5231 x 4096 x 6386
// 168 | 146, 7275 x 2048 x 5251 120 | 114; of 30 shapes nine are split and none of them loses.
LinearPlan linear_plan(int M, int N, int K) {
  LinearPlan plan{};
  plan.tile = best_tile(M, N, K, &plan.us);
  plan.M1 = M, plan.N1 = N;
  for (int i = 0; i < 3; ++i) {
    const Tile &t = TILES[i];
    const int slots = 256 * t.per_cu, tm = (M + t.bm - 1) / t.bm, tn = (N + t.bn - 1) / t.bn;
    // whole rounds over the first channels, or over the first tokens
    const int n1 = tm <= slots ? tn / (slots / tm) * (slots / tm) * t.bn : 0, m1 = tn <= slots ? tm / (slots / tn) * (slots / tn) * t.bm : 0;
    float rest;
    if (n1 > 0 && n1 < N) {
      const int tile2 = best_tile(M, N - n1, K, &rest);
      const float us = tile_us(t, M, n1, K) + rest + 2.0f;
      if (us < 0.95f * plan.us) plan = LinearPlan{i, M, n1, tile2, us, 0};
    }
    if (m1 > 0 && m1 < M) {
      const int tile2 = best_tile(M - m1, N, K, &rest);
      const float us = tile_us(t, m1, N, K) + rest + 2.0f;
      if (us < 0.95f * plan.us) plan = LinearPlan{i, m1, N, tile2, us, 0};
    }
  }
  const Tile &t = TILES[plan.tile];
  plan.wgs = (int64_t)((plan.M1 + t.bm - 1) / t.bm) * ((plan.N1 + t.bn - 1) / t.bn);
  return plan;
}

}  // namespace f8
