// Attention of one new token per request over a paged cache of 8 or 16 bits:
//
//   s_t = scale * q . k_t,   p = softmax of s over the tokens of the request,   o = sum_t p_t v_t   (0 without tokens),
//
// query head h reads cache head h / G.  A workgroup's unit of work is 128 tokens of a request (or 64, of two heads), a cache head and
// up to 16 of the query heads that share it; the units of all requests are dealt out evenly (see Runs), and a second launch joins the pairs that came
// apart.
//
// Inside, a wave walks over tiles of 32 tokens on its own and keeps the running maximum, sum and output of its heads.  Both
// products run on the matrix cores with 16 heads as columns, S^T = K Q^T and O^T = V^T P^T: a lane then owns one head, its
// maximum and sum are plain numbers, and the scores that it holds of S^T (tokens 4 g + i of two blocks of 16, g = lane / 16) are,
// as they lie, its operand of the second product.  The tokens are summed over, so their order inside an operand is free: V is
// read with lane (c, g) taking dimensions c E .. c E + E - 1 of its own 8 tokens, E = dim / 16, whole rows at a time, and the
// operand of the n-th product is element n of each, which is a byte permutation inside the lane.  Nothing of K or V passes
// through LDS; what does is where a tile's rows lie (64 bits each: a cache may be larger than 4 GiB) and their scales.
//
// Codes are exact in 16-bit floating point.  A key's scale multiplies its score; a value's scale counts in the maximum,
// m = max(s_t + max(log2 scale_t, SMALL)) (scores as powers of two), so that exp2(s_t - m) scale_t, the weight of a row of codes, is at
// most 1 whatever the scales are.  The sum of the softmax takes exp2(s_t - m) itself, which a row with a small scale brings up to 2^-SMALL: rows
// of zeros, whose scale is 2^-126 or 0, are the ones that come.
//
// The second product takes weights of 16 bits.  Under 16-bit caches a weight goes in as two of them, its front and the rest: one
// alone would be as coarse as the result (8 requests of up to 300 tokens, off the exact result: bf16 1.84e-3 with one, 1.66e-3 with two, which
// is the rounding of the result alone; f16 2.18e-4 and 2.02e-4; 6.3 and 6.5 us, 16 requests of up to 8192 tokens 45.2 and 45.9).  Under 8-bit
// caches it is rounded once, to f16, relative 2^-11: an eighth of the half unit that 8 bits leave a row's largest element.
// In f16 all weights and sums are 2^15 times what is written here, the largest that f16 holds: the relative error then holds down to 2^-29 of
// the largest weight, and what lies below is off by 2^-40 of it at most, 2^-23 of it over 131072 tokens
// (in two parts 2^-39 above that line: a rest is never 0).  Scores, maxima, sums and outputs are 32 bits.
//
// Bound by HBM: every cached byte is read once, in whole rows, one tile ahead per wave (131072 tokens of 8 heads, 277 MB: 58 us, 4.8 TB/s, and
// 7 of the second launch; 64 requests of up to 8192 tokens, 491 MB: 103 us, 4.75 TB/s, and 8; a large copy reaches 5.5).  The vector units
// are a third busy (350 instructions a tile, most of them codes into f16).  Without the tile ahead the two took 97 and 239 us with their
// second launch; with the requests' lengths cut into equal stretches, a workgroup each, instead of units dealt out evenly, 68 and 167.
#include <math.h>

#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

typedef f16 h8 __attribute__((ext_vector_type(8)));
typedef bf16 b8 __attribute__((ext_vector_type(8)));
typedef f16 h2 __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef long long v2l __attribute__((ext_vector_type(2)));

constexpr int WAVES = 4, TILE = 32, HEADS = 16;
constexpr float LOG2E = 1.4426950408889634f;
// The least that a value's scale counts for in the maximum, as a power of two: 2^31 tokens of 2^(15 - SMALL) each stay below the largest
// 32-bit number.  Values whose scales all lie below it (1e-24) only lose bits below 2^-109, where their weights leave f16's normal range.
constexpr float SMALL = -80.0f;

struct AttendParams {
  const void *q, *k, *v;
  const float *k_scale, *v_scale;
  const int32_t *table, *lens;
  void *out;
  float *part_o, *part_ml;                 // [2 wgs][rows][dim] and [2 wgs][rows][2], rows = min(group, HEADS)
  int64_t qt, qh, ot, oh, page, token, head, spage, stoken, shead, table_ld;
  int batch, hp, kv_groups, group, chunks, dim, pages, max_len;   // kv_groups: of hp heads of the cache
  int unit_shift;                          // log2 of the tokens of a unit
  int wgs;                                 // 0: a workgroup to each pair
  FastDiv page_size;
  float scale;                             // of the scores, times log2 e
};

// How the work is dealt out.  A pair is a request and a cache head (or HP of them) with up to 16 of its query heads; its units are
// rounds of a workgroup's four waves over the request's tokens.  All pairs' units lie in a row, request by request, and each workgroup takes
// an equal run of them, whatever the lengths are: a pair that a run does not hold whole is left in pieces for join_kernel, at most
// two to a workgroup (slot 0 its first pair, slot 1 its last).  The lengths are only known on the device, so every workgroup adds
// them up itself.
constexpr int UNIT = WAVES * TILE;
__device__ __forceinline__ int len_of(const AttendParams &p, int b) { return min(max(p.lens[b], 0), p.max_len); }
__device__ __forceinline__ int units_of(const AttendParams &p, int b) { return (len_of(p, b) + (1 << p.unit_shift) - 1) >> p.unit_shift; }
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

// What a wave keeps in LDS of a tile: where its 32 rows begin, in elements, and (8-bit caches) the scales of its keys, those of its
// values and their logarithms, SMALL at least.
struct TileRows {
  int64_t at[TILE];
  float scale[3 * TILE];
};

// (two waves to a SIMD where the registers allow it: the second workgroup of a CU works while the first one looks up its pair or joins its
// waves.  128 dimensions of 16 bits held to that spill 14 words a lane, and their reloads wait for the tile ahead: 57.7 us against 51.1)
template <typename C, typename Q, int DP, int HP>
__global__ __launch_bounds__(64 * WAVES, DP * sizeof(C) > 128 ? 1 : 2) void attend_kernel(AttendParams p) {
  typedef Operand<C> Op;
  typedef typename Op::t H;
  constexpr bool S8 = sizeof(C) == 1;
  constexpr int E = DP / 16, VB = E * (int)sizeof(C);     // elements and bytes of a value row per lane
  constexpr int KL = DP * (int)sizeof(C) / 64;            // 16-byte loads of a key row per lane
  constexpr int KS = DP / 32;                             // products per block of 16 scores
  constexpr int SHARE = WAVES / HP;                       // waves of a head
  __shared__ TileRows rows[WAVES][2];
  __shared__ float part[WAVES][HEADS][DP + 1], ml[WAVES][HEADS][2];
  __shared__ int64_t scan[WAVES][2], before;
  __shared__ int from;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c16 = lane & 15, g = lane >> 4;
  const int per_b = p.kv_groups * p.chunks, group_rows = min(p.group, HEADS), mine = wave % HP;
  // Runs that follow one another lie on one XCD, so that the heads of a request, whose scales share lines, share an L2 (64 requests of
  // up to 8192 tokens, 491 MB, one head at a time: 592 MB fetched otherwise and 122 us, 563 and 117 with it).  With few requests a head
  // is many runs, and those of the same tokens meet on an XCD by themselves.
  const uint32_t run = p.batch >= 8 ? xcd_remap(blockIdx.x, gridDim.x) : blockIdx.x;
  int b, hc, unit, units, slot = 0;
  int64_t left;                               // units of this workgroup's run
  if (p.wgs == 0) {
    b = (int)run / per_b, hc = (int)run % per_b, unit = 0, units = units_of(p, b), left = units;
  } else {
    // The request that holds the run's first unit: the units of 256 requests at a time, added up from the front.  (The sum of all
    // of them comes with it where there are no more requests than that.)
    int64_t total = -1, start = 0, done = 0;
    if (p.batch > 64 * WAVES) {
      int64_t sum[2] = {0, 0};
      for (int i = threadIdx.x; i < p.batch; i += 64 * WAVES) sum[0] += units_of(p, i);
      wg_sum<WAVES>(sum, scan);
      total = sum[0] * per_b;
    }
    for (int i0 = 0;; i0 += 64 * WAVES) {
      const int i = i0 + (int)threadIdx.x;
      const int64_t mine = i < p.batch ? (int64_t)units_of(p, i) * per_b : 0;
      int64_t upto = mine;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int64_t o = __shfl_up((long long)upto, d);
        if (lane >= d) upto += o;
      }
      if (lane == 63) scan[wave][0] = upto;
      __syncthreads();
      int64_t at = done, all = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        if (w < wave) at += scan[w][0];
        all += scan[w][0];
      }
      at += upto - mine;
      if (i0 == 0) {
        const Runs runs(uniform64(total < 0 ? all : total), p.wgs);
        start = runs.start(run);
        left = runs.start((int64_t)run + 1) - start;
        if (left == 0) return;
      }
      if (mine > 0 && at <= start && start < at + mine) from = i, before = at;
      __syncthreads();
      done += all;
      if (start < done) break;
    }
    b = from;
    units = units_of(p, b);
    const int64_t in = start - before;
    hc = (int)(in / units), unit = (int)(in - (int64_t)hc * units);
  }
  b = __builtin_amdgcn_readfirstlane(b), hc = __builtin_amdgcn_readfirstlane(hc);
  unit = __builtin_amdgcn_readfirstlane(unit), units = __builtin_amdgcn_readfirstlane(units), left = uniform64(left);
  for (bool more = true; more;) {
    const int kv0 = hc / p.chunks * HP, kvh = kv0 + mine, qc = hc % p.chunks, len = len_of(p, b);
    const int last = (int)min((int64_t)units, unit + left), first = unit * (UNIT / HP), end = min(len, last * (UNIT / HP));
    const int heads = min(HEADS, p.group - qc * HEADS), hq0 = kvh * p.group + qc * HEADS;
    const int32_t *table = p.table + b * p.table_ld;

    // Q^T as the right operand: the lane's head, the dimensions that its loads of K bring
    v4i q[KS];
    float q_scale = p.scale;
    {
      const Q *src = static_cast<const Q *>(p.q) + b * p.qt + (hq0 + min(c16, heads - 1)) * p.qh;
      float f[KS][8];
      v4i raw[KS];
      uint32_t top = 0;
      // (8 neighbours at a time, all loads in flight; dimensions past the head's and heads past the group's become 0 afterwards)
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int d = S8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
        __builtin_memcpy(&raw[s], src + (d < p.dim ? d : 0), 16);
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int d = S8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
        unpack8<Q>(&raw[s], f[s]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f[s][j] = c16 < heads && d < p.dim ? f[s][j] : 0.0f;
          top = max(top, magnitude(f[s][j]));
        }
      }
      if (S8) {
        // a power of two brings the largest element of the head to [2^14, 2^15): f16 then holds what the 16-bit q had, elements
        // 2^-28 below the largest excepted
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const int ex = max((int)(top >> 23), 15);             // (the two factors are then normal numbers, for an infinity's exponent too)
        q_scale *= __int_as_float((ex - 14) << 23);
        const float inv = __int_as_float((268 - ex) << 23);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int j = 0; j < 8; ++j) f[s][j] *= inv;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        typedef H t8 __attribute__((ext_vector_type(8)));
        t8 o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = (H)f[s][j];
        q[s] = __builtin_bit_cast(v4i, o);
      }
    }

    v4f o[E];
#pragma unroll
    for (int n = 0; n < E; ++n) o[n] = v4f{0, 0, 0, 0};
    float m = -INFINITY, l = 0.0f;

    // A tile on its way: while one is attended to, the next one's rows are in flight, and the table entries of the one after.
    struct Tile {
      Raw<16> k[2][KL];
      Raw<VB> v[8];
      float scale;                            // lanes 0..31: of the key of token `lane`, 32..63: of the value of token `lane - 32`
      uint32_t there;                         // its tokens that exist
    };
    const C *const kbase = static_cast<const C *>(p.k) + kvh * p.head, *const vbase = static_cast<const C *>(p.v) + kvh * p.head;
    const int dv = c16 * E < p.dim ? c16 * E : 0;
    auto look_up = [&](int t0) {              // page of token lane % 32 of the tile at t0
      const int tok = t0 + (lane & 31);
      return tok < end ? table[p.page_size.div((uint32_t)tok)] : -1;
    };
    auto fetch = [&](int t0, int page, int64_t (&at_lds)[TILE], Tile &x) {
      const uint32_t tok = (uint32_t)(t0 + (lane & 31)), place = tok - p.page_size.div(tok) * p.page_size.d;
      const bool there = (uint32_t)page < (uint32_t)p.pages;
      x.there = (uint32_t)__ballot(there);
      const int64_t at = there ? page * p.page + place * p.token : 0;
      if (lane < 32) at_lds[lane] = at;
      lanes_meet();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const C *row = kbase + at_lds[16 * h + c16];
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          const int d = (i * 4 + g) * (16 / (int)sizeof(C));
          x.k[h][i] = load_raw<16>(row + (d < p.dim ? d : 0));
        }
      }
      if constexpr (S8) {
        const float *src = lane < 32 ? p.k_scale : p.v_scale;
        x.scale = there ? src[page * p.spage + place * p.stoken + kvh * p.shead] : 1.0f;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) x.v[4 * h + j] = load_raw<VB>(vbase + at_lds[16 * h + 4 * g + j] + dv);
    };

    auto attend = [&](Tile &x, float *scale_lds) {
      v4f ks[2], vs[2], vl[2];
      if constexpr (S8) {
        scale_lds[lane] = x.scale;
        if (lane >= 32) scale_lds[32 + lane] = fmaxf(__log2f(x.scale), SMALL);
        lanes_meet();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          ks[h] = *reinterpret_cast<const v4f *>(scale_lds + 16 * h + 4 * g);
          vs[h] = *reinterpret_cast<const v4f *>(scale_lds + 32 + 16 * h + 4 * g);
          vl[h] = *reinterpret_cast<const v4f *>(scale_lds + 64 + 16 * h + 4 * g);
        }
      }
      // scores of the lane's head at its 8 tokens
      float s[8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        v4f acc{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          const bool real = (i * 4 + g) * (16 / (int)sizeof(C)) < p.dim;
          uint32_t d[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) d[j] = real ? x.k[h][i].d[j] : 0u;
          if constexpr (S8) {
            h8 lo, hi;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t u = d[j] ^ 0x80808080u;
              const h2 a = codes_lo(u), e = codes_hi(u);
              h8 &to = j < 2 ? lo : hi;
              to[4 * (j & 1)] = a[0], to[4 * (j & 1) + 1] = a[1], to[4 * (j & 1) + 2] = e[0], to[4 * (j & 1) + 3] = e[1];
            }
            acc = Op::mfma(__builtin_bit_cast(v4i, lo), q[2 * i], acc);
            acc = Op::mfma(__builtin_bit_cast(v4i, hi), q[2 * i + 1], acc);
          } else {
            acc = Op::mfma(v4i{(int)d[0], (int)d[1], (int)d[2], (int)d[3]}, q[i], acc);
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) s[4 * h + j] = acc[j] * (S8 ? q_scale * ks[h][j] : q_scale);
      }
      if (x.there != 0xffffffffu) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const bool there = x.there >> (16 * h + 4 * g + j) & 1;
            if (!there) s[4 * h + j] = -INFINITY;
#pragma unroll
            for (int n = 0; n < VB / 4; ++n) x.v[4 * h + j].d[n] = there ? x.v[4 * h + j].d[n] : 0u;   // (0 * NaN is NaN)
          }
      }
      float top = m;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, S8 ? s[j] + vl[j >> 2][j & 3] : s[j]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float base = top == -INFINITY ? 0.0f : top;
      if (__any(top > m)) {                   // (seldom in a long context)
        const float shrink = __builtin_amdgcn_exp2f(m - base);
        l *= shrink;
#pragma unroll
        for (int n = 0; n < E; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) o[n][j] *= shrink;
        m = top;
      }
      typedef H t8 __attribute__((ext_vector_type(8)));
      float w[8];
      v4i pt, rest;
      const float below = base - Op::UP;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] = __builtin_amdgcn_exp2f(s[j] - below);
        l += w[j];
      }
      if constexpr (S8) {
        t8 wh;
#pragma unroll
        for (int j = 0; j < 8; ++j) wh[j] = (H)(w[j] * vs[j >> 2][j & 3]);
        pt = __builtin_bit_cast(v4i, wh);
      } else {
        t8 wl;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
          const uint32_t pair = Op::cut(w[j], w[j + 1]);
          pt[j / 2] = (int)pair;
          wl[j] = Op::rest(w[j], pair, 0), wl[j + 1] = Op::rest(w[j + 1], pair, 1);
        }
        rest = __builtin_bit_cast(v4i, wl);
      }
#pragma unroll
      for (int n = 0; n < E; ++n) {
        v4i a;
        if constexpr (S8) {
          const uint32_t sel = 0x0c000c00u | (uint32_t)(n & 3) | (uint32_t)(4 + (n & 3)) << 16;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t u = __builtin_amdgcn_perm(x.v[2 * j + 1].d[n >> 2], x.v[2 * j].d[n >> 2], sel) ^ 0x64806480u;
            a[j] = __builtin_bit_cast(int, __builtin_bit_cast(h2, u) - h2{(f16)1152, (f16)1152});
          }
        } else {
          const uint32_t sel = n & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
          for (int j = 0; j < 4; ++j) a[j] = (int)__builtin_amdgcn_perm(x.v[2 * j + 1].d[n >> 1], x.v[2 * j].d[n >> 1], sel);
        }
        o[n] = Op::mfma(a, pt, o[n]);
        if constexpr (!S8) o[n] = Op::mfma(a, rest, o[n]);
      }
    };

    constexpr int NEXT = SHARE * TILE;
    int t0 = first + wave / HP * TILE;
    if (t0 < end) {
      Tile x, y;
      fetch(t0, look_up(t0), rows[wave][0].at, x);
      int page = look_up(t0 + NEXT);
      auto turn = [&](Tile &now, Tile &then, int buf) {
        if (t0 + NEXT < end) {
          const int ahead = look_up(t0 + 2 * NEXT);
          fetch(t0 + NEXT, page, rows[wave][buf ^ 1].at, then);
          page = ahead;
        }
        attend(now, rows[wave][buf].scale);
        t0 += NEXT;
        return t0 < end;
      };
      while (turn(x, y, 0) && turn(y, x, 1)) {
      }
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // the waves of a head join in LDS
    if (g == 0) ml[wave][c16][0] = m, ml[wave][c16][1] = l;
    __syncthreads();
    float top = ml[mine][c16][0];
#pragma unroll
    for (int w = 1; w < SHARE; ++w) top = fmaxf(top, ml[mine + w * HP][c16][0]);
    const float shrink = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
#pragma unroll
    for (int n = 0; n < E; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) part[wave][c16][(4 * g + j) * E + n] = o[n][j] * shrink;
    __syncthreads();
    for (int i = threadIdx.x; i < HP * heads * DP; i += 64 * WAVES) {
      const int row = i / DP, d = i % DP, k = row / heads, h = row - k * heads;      // cache head kv0 + k, its query head h
      float mh = ml[k][h][0], sum = 0.0f, of = 0.0f;
#pragma unroll
      for (int w = 1; w < SHARE; ++w) mh = fmaxf(mh, ml[k + w * HP][h][0]);
      const float base = mh == -INFINITY ? 0.0f : mh;
#pragma unroll
      for (int w = 0; w < SHARE; ++w) {
        sum += ml[k + w * HP][h][1] * __builtin_amdgcn_exp2f(ml[k + w * HP][h][0] - base);
        of += part[k + w * HP][h][d];
      }
      if (d >= p.dim) continue;
      if (unit == 0 && last == units) {
        static_cast<Q *>(p.out)[b * p.ot + ((kv0 + k) * p.group + qc * HEADS + h) * p.oh + d] = (Q)(sum == 0.0f ? 0.0f : of / sum);
      } else {
        const int64_t at = ((2 * (int64_t)run + slot) * HP + k) * group_rows + h;
        p.part_o[at * p.dim + d] = of;
        if (d == 0) p.part_ml[2 * at] = mh, p.part_ml[2 * at + 1] = sum;
      }
    }
    left -= last - unit;
    more = left > 0;
    if (more) {                                 // the next pair that has tokens
      __syncthreads();
      slot = 1, unit = 0;
      if (++hc == per_b) {
        hc = 0;
        do units = __builtin_amdgcn_readfirstlane(units_of(p, ++b));
        while (units == 0);
      }
    }
  }
}

// The pairs that lie in pieces, and the requests without tokens.  A workgroup takes JOIN_PART elements (heads by dimensions) of a
// pair, 4 neighbours a thread and as many pieces at a time as threads are left; the pieces are added up in a fixed order.
constexpr int JOINERS = 8, JOIN_PART = 256, JOIN_VECS = JOIN_PART / 4, JOIN_AT_ONCE = 64 * JOINERS / JOIN_VECS;

template <typename Q>
__global__ __launch_bounds__(64 * JOINERS) void join_kernel(AttendParams p) {
  __shared__ v4f part[JOIN_AT_ONCE][JOIN_VECS];
  __shared__ float sums[JOIN_AT_ONCE][JOIN_VECS];
  __shared__ int64_t scan[JOINERS][2];
  const int per_b = p.kv_groups * p.chunks, b = blockIdx.x / per_b, hc = blockIdx.x % per_b, kv0 = hc / p.chunks * p.hp, qc = hc % p.chunks;
  const int heads = min(HEADS, p.group - qc * HEADS), group_rows = min(p.group, HEADS), rows = p.hp * group_rows, units = units_of(p, b);
  const int vec = (int)threadIdx.x % JOIN_VECS, mine = (int)threadIdx.x / JOIN_VECS;
  // (dim is a multiple of 16: four neighbours belong to one head)
  const int e = blockIdx.y * JOIN_PART + vec * 4, row = e / p.dim, d = e - row * p.dim, k = row / group_rows, h = row - k * group_rows;
  const bool real = k < p.hp && h < heads;
  Q *out = static_cast<Q *>(p.out) + b * p.ot + ((kv0 + k) * p.group + qc * HEADS + h) * p.oh + d;
  if (units == 0) {
    if (mine == 0 && real)
      for (int j = 0; j < 4; ++j) out[j] = (Q)0.0f;
    return;
  }
  int64_t all[2] = {0, 0};                    // units of all requests, and of those in front of this one
  for (int i = threadIdx.x; i < p.batch; i += 64 * JOINERS) {
    const int u = units_of(p, i);
    all[0] += u;
    if (i < b) all[1] += u;
  }
  wg_sum<JOINERS>(all, scan);
  const Runs runs(uniform64(all[0] * per_b), p.wgs);
  const int64_t at = uniform64(all[1] * per_b + (int64_t)hc * units), i0 = runs.of(at), i1 = runs.of(at + units - 1);
  if (i0 == i1) return;                       // whole in one run
  // piece i lies in slot 0 of workgroup i, but the pair may begin behind others in the first one (runs in between are not empty:
  // with fewer units than workgroups the first ones have one each)
  const int64_t row0 = (2 * i0 + (runs.start(i0) < at ? 1 : 0)) * rows, step = 2 * rows;
  const int n = (int)(i1 - i0) + 1, hr = real ? row : 0;
  const float2 *ml = reinterpret_cast<const float2 *>(p.part_ml) + hr;
  const float *po = p.part_o + hr * p.dim + (real ? d : 0);
  auto row_of = [&](int i) { return i == 0 ? row0 : (2 * i0) * rows + i * step; };
  // running maximum, as in the kernel above; four pieces on their way at a time
  float top = -INFINITY, sum = 0.0f;
  v4f o{0, 0, 0, 0};
  for (int i = mine; i < n; i += 4 * JOIN_AT_ONCE) {
    float2 s[4];
    v4f v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t r = row_of(min(i + u * JOIN_AT_ONCE, n - 1));
      s[u] = ml[r];
      v[u] = *reinterpret_cast<const v4f *>(po + r * p.dim);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i + u * JOIN_AT_ONCE >= n) break;
      const float now = fmaxf(top, s[u].x), base = now == -INFINITY ? 0.0f : now;
      const float was = __builtin_amdgcn_exp2f(top - base), is = __builtin_amdgcn_exp2f(s[u].x - base);
      top = now;
      sum = sum * was + s[u].y * is;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = o[k] * was + v[u][k] * is;
    }
  }
  __shared__ float tops[JOIN_AT_ONCE][JOIN_VECS];
  part[mine][vec] = o, sums[mine][vec] = sum, tops[mine][vec] = top;
  __syncthreads();
  if (mine != 0 || !real) return;
  for (int w = 1; w < JOIN_AT_ONCE; ++w) top = fmaxf(top, tops[w][vec]);
  const float base = top == -INFINITY ? 0.0f : top;
  sum = 0.0f, o = v4f{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < JOIN_AT_ONCE; ++w) {
    const float f = __builtin_amdgcn_exp2f(tops[w][vec] - base);
    sum += sums[w][vec] * f;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] += part[w][vec][k] * f;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) out[k] = (Q)(sum == 0.0f ? 0.0f : o[k] / sum);
}

template <typename C, typename Q>
f8_status launch(const AttendParams &p, hipStream_t s) {
  const int pairs = p.batch * p.kv_groups * p.chunks;
  const dim3 grid(p.wgs ? p.wgs : pairs);
  const dim3 block(64 * WAVES);
  if (sizeof(C) == 1 && p.hp == 2) {
    if (p.dim <= 64) hipLaunchKernelGGL((attend_kernel<int8_t, Q, 64, 2>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((attend_kernel<int8_t, Q, 128, 2>), grid, block, 0, s, p);
  } else if (p.dim <= 64) {
    hipLaunchKernelGGL((attend_kernel<C, Q, 64, 1>), grid, block, 0, s, p);
  } else if (p.dim <= 128) {
    hipLaunchKernelGGL((attend_kernel<C, Q, 128, 1>), grid, block, 0, s, p);
  } else {
    hipLaunchKernelGGL((attend_kernel<C, Q, 256, 1>), grid, block, 0, s, p);
  }
  f8_status st = launch_status();
  if (st != F8_OK || p.wgs == 0) return st;
  const int elements = p.hp * (p.group < HEADS ? p.group : HEADS) * p.dim;
  hipLaunchKernelGGL(join_kernel<Q>, dim3(pairs, (elements + JOIN_PART - 1) / JOIN_PART), dim3(64 * JOINERS), 0, s, p);
  return launch_status();
}

// How a call's work is dealt out.
// wgs: workgroups among which the units are, or 0: a workgroup to each pair and no second launch, up to 4 units (300 tokens, 32 pairs:
// 5.7 us against 7.1).  Otherwise as many as are resident at once, two to a CU, or one where a row is more than 128 bytes (of the
// kernel's 64, 128 or 256 dimensions): a workgroup's way to its first rows is 5 us that only its neighbour hides (131072 tokens, 8
// pairs: 67 us with 512, 72 with 1024, 81 with 256; 256 dimensions, 16 pairs of up to 16384 tokens: 39 us with 256, 45 with 512), and
// at most 256 to a pair, whose pieces the second launch adds up (one pair of 131072 tokens: 26 us with 256, 33 with 512).
// hp: heads of the cache that a workgroup reads side by side, half of the waves each.  Two, where rows of 8 bits are at most 128 bytes
// and there are many requests: their rows are neighbours in a token's memory, and so are their scales (us with one | two: 16 requests of
// 8192 tokens 73 | 66, 64 of up to 8192 117 | 113, 64 of up to 4096 with 64 dimensions 53 | 48, but 8 of up to 4096 23 | 25 and 2 of up to
// 65536 30 | 33; 16 of up to 8192 in 16 bits 52 | 53).
struct Deal {
  int hp, wgs;
  size_t rows;                             // of the pieces that the workgroups may leave
};
Deal deal_of(int64_t batch, int kv_heads, int group, int dim, int bytes, int max_len) {
  const int row = (dim <= 64 ? 64 : dim <= 128 ? 128 : 256) * bytes, chunks = (group + HEADS - 1) / HEADS;
  Deal d{1, 0, 0};
  if (max_len <= 4 * UNIT) return d;
  const int64_t rounds = batch * kv_heads * chunks * (((int64_t)max_len + UNIT - 1) / UNIT);
  if (bytes == 1 && row <= 128 && kv_heads % 2 == 0 && batch >= 16 && rounds >= 2048) d.hp = 2;
  const int64_t pairs = batch * (kv_heads / d.hp) * chunks, units = ((int64_t)max_len + UNIT / d.hp - 1) / (UNIT / d.hp);
  const int64_t most = row > 128 || pairs == 1 ? 256 : 512;
  d.wgs = (int)(pairs * units < most ? pairs * units : most);
  d.rows = (size_t)2 * d.wgs * d.hp * (group < HEADS ? group : HEADS);
  return d;
}

}  // namespace
}  // namespace f8

using namespace f8;

extern "C" {

// (for any type of cache)
size_t f8_attend_workspace_bytes(int batch, int q_heads, int kv_heads, int dim, int max_len) {
  if (batch < 1 || q_heads < 1 || kv_heads < 1 || dim < 1 || max_len < 1 || q_heads % kv_heads != 0) return 0;
  const size_t a = deal_of(batch, kv_heads, q_heads / kv_heads, dim, 1, max_len).rows, b = deal_of(batch, kv_heads, q_heads / kv_heads, dim, 2, max_len).rows;
  return (a > b ? a : b) * (dim + 2) * sizeof(float);
}

f8_status f8_attend_paged(const void *q, const void *k_cache, const void *v_cache, const float *k_scale, const float *v_scale,
                          const int32_t *table, const int32_t *lens, void *out, const f8_kv_layout *c, const f8_attend_desc *d,
                          void *workspace, size_t workspace_bytes, void *stream) {
  if (!c || !d) return F8_ERR_NULL;
  f8_status st = check_kv_layout(*c);
  if (st != F8_OK) return st;
  if ((d->type != F8_F16 && d->type != F8_BF16) || (c->type != F8_S8 && c->type != d->type)) return F8_ERR_DTYPE;
  if (d->batch < 0 || d->batch > 65535 || d->q_heads < 1 || d->q_heads % c->heads != 0 || d->table_cols < 0 || d->max_len < 0) return F8_ERR_SHAPE;
  if ((int64_t)d->max_len > (int64_t)d->table_cols * c->page_size || d->max_len > 0x7fff0000) return F8_ERR_SHAPE;
  if (d->table_ld < d->table_cols || isnan(d->scale)) return F8_ERR_SHAPE;
  if (d->batch == 0) return F8_OK;
  const bool codes = c->type == F8_S8;
  if (!q || !k_cache || !v_cache || (!table && d->max_len > 0) || !lens || !out || (codes && (!k_scale || !v_scale))) return F8_ERR_NULL;
  const size_t e = bytes_of(c->type);
  if (!aligned_to(q, 2) || !aligned_to(out, 2) || !aligned_to(table, 4) || !aligned_to(lens, 4) || !aligned_to(k_scale, 4) || !aligned_to(v_scale, 4) ||
      !aligned_to(k_cache, 16) || !aligned_to(v_cache, 16) || c->page_stride * e % 16 || c->token_stride * e % 16 || c->head_stride * e % 16)
    return F8_ERR_ALIGN;
  const int group = d->q_heads / c->heads, chunks = (group + HEADS - 1) / HEADS;
  if ((int64_t)d->batch * c->heads * chunks > 1 << 22) return F8_ERR_UNSUPPORTED;          // (workgroups of a launch)
  const Deal deal = deal_of(d->batch, c->heads, group, c->dim, (int)bytes_of(c->type), d->max_len);
  if (deal.wgs) {
    if (!workspace) return F8_ERR_NULL;
    if (!aligned_to(workspace, 16)) return F8_ERR_ALIGN;
    if (workspace_bytes < f8_attend_workspace_bytes(d->batch, d->q_heads, c->heads, c->dim, d->max_len)) return F8_ERR_SHAPE;
  }
  float *ws = static_cast<float *>(workspace);
  const AttendParams p{q, k_cache, v_cache, k_scale, v_scale, table, lens, out, ws, deal.wgs ? ws + deal.rows * c->dim : nullptr,
                       d->q_token, d->q_head, d->o_token, d->o_head, c->page_stride, c->token_stride, c->head_stride,
                       c->scale_page, c->scale_token, c->scale_head, d->table_ld, d->batch, deal.hp, c->heads / deal.hp, group, chunks, c->dim, c->pages, d->max_len,
                       deal.hp == 1 ? 7 : 6, deal.wgs, FastDiv((uint32_t)c->page_size), d->scale * LOG2E};
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (codes) return d->type == F8_F16 ? launch<int8_t, f16>(p, hs) : launch<int8_t, bf16>(p, hs);
  return d->type == F8_F16 ? launch<f16, f16>(p, hs) : launch<bf16, bf16>(p, hs);
}

}  // extern "C"
