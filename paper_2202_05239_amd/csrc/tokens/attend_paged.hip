// Attention of one new token per request over a paged cache of 8 or 16 bits:
//
//   s_t = scale * q . k_t,   p = softmax of s over the tokens of the request,   o = sum_t p_t v_t   (0 without tokens),
//
// query head h reads cache head h / G.  One workgroup takes a request, a cache head, up to 16 of the query heads that share it
// and a stretch of its tokens; a second launch joins the stretches where there are several.
//
// Inside, a wave walks over tiles of 32 tokens on its own and keeps the running maximum, sum and output of its heads.  Both
// products run on the matrix cores with 16 heads as columns, S^T = K Q^T and O^T = V^T P^T: a lane then owns one head, its
// maximum and sum are plain numbers, and the scores that it holds of S^T (tokens 4 g + i of two blocks of 16, g = lane / 16) are,
// as they lie, its operand of the second product.  The tokens are summed over, so their order inside an operand is free: V is
// read with lane (c, g) taking dimensions c E .. c E + E - 1 of its own 8 tokens, E = dim / 16, whole rows at a time, and the
// operand of the n-th product is element n of each, which is a byte permutation inside the lane.  Nothing of K or V passes
// through LDS; what does is where a tile's rows lie (64 bits each: a cache may be larger than 4 GiB) and their scales.
//
// Codes are exact in 16-bit floating point.  A key's scale multiplies its score; a value's scale joins the exponent,
// w_t = exp(s_t + log scale_t - m) with m the maximum of that sum, so that w is in [0, 1] whatever the scales are.  w is rounded
// to 16 bits for the second product (as P is for 16-bit caches): relative 2^-12 (f16) or 2^-9 (bf16) of each weight, at random,
// below the rounding of the 16-bit result.  Scores, maxima, sums and outputs are 32 bits.
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

struct AttendParams {
  const void *q, *k, *v;
  const float *k_scale, *v_scale;
  const int32_t *table, *lens;
  void *out;
  float *part_o, *part_ml;                 // [batch][q_heads][splits][dim] and [..][2]
  int64_t qt, qh, ot, oh, page, token, head, spage, stoken, shead, table_ld;
  int q_heads, group, dim, pages, max_len, splits, chunk;
  FastDiv page_size;
  float scale;                             // of the scores, times log2 e
};

// Codes of four neighbouring bytes as f16, exactly: byte + 128 under the exponent of 1024, minus 1152.
__device__ __forceinline__ h2 codes_lo(uint32_t u) { return __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - h2{(f16)1152, (f16)1152}; }
__device__ __forceinline__ h2 codes_hi(uint32_t u) { return __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - h2{(f16)1152, (f16)1152}; }

template <typename C>
struct Operand {                            // 16-bit type of the products
  typedef f16 t;
  static __device__ __forceinline__ v4f mfma(v4i a, v4i b, v4f c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
};
template <>
struct Operand<bf16> {
  typedef bf16 t;
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

// What a wave keeps in LDS of a tile: where its 32 rows begin, in elements, and (8-bit caches) the scales of its keys and the
// logarithms of its values'.
struct TileRows {
  int64_t at[TILE];
  float scale[2 * TILE];
};

template <typename C, typename Q, int DP>
__global__ __launch_bounds__(64 * WAVES) void attend_kernel(AttendParams p) {
  typedef Operand<C> Op;
  typedef typename Op::t H;
  constexpr bool S8 = sizeof(C) == 1;
  constexpr int E = DP / 16, VB = E * (int)sizeof(C);     // elements and bytes of a value row per lane
  constexpr int KL = DP * (int)sizeof(C) / 64;            // 16-byte loads of a key row per lane
  constexpr int KS = DP / 32;                             // products per block of 16 scores
  __shared__ TileRows rows[WAVES][2];
  __shared__ float part[WAVES][HEADS][DP + 1], ml[WAVES][HEADS][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c16 = lane & 15, g = lane >> 4;
  const int chunks = (p.group + HEADS - 1) / HEADS;
  const int kvh = blockIdx.x / chunks, qc = blockIdx.x % chunks, split = blockIdx.y, b = blockIdx.z;
  const int len = min(max(p.lens[b], 0), p.max_len), first = split * p.chunk, end = min(len, first + p.chunk);
  if (split > 0 && first >= len) return;
  const int heads = min(HEADS, p.group - qc * HEADS), hq0 = kvh * p.group + qc * HEADS;
  const int32_t *table = p.table + b * p.table_ld;

  // Q^T as the right operand: the lane's head, the dimensions that its loads of K bring
  v4i q[KS];
  float q_scale = p.scale;
  {
    const Q *src = static_cast<const Q *>(p.q) + b * p.qt + (hq0 + min(c16, heads - 1)) * p.qh;
    float f[KS][8];
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int d = S8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 + j : s * 32 + g * 8 + j;
        f[s][j] = c16 < heads && d < p.dim ? (float)src[d] : 0.0f;
        top = max(top, magnitude(f[s][j]));
      }
    if (S8) {
      // a power of two brings the largest element of the head into [1, 2): f16 then holds what the 16-bit q had, elements
      // 2^-14 below the largest excepted
      top = max(top, (uint32_t)__shfl_xor((int)top, 16));
      top = max(top, (uint32_t)__shfl_xor((int)top, 32));
      const int ex = (int)(top >> 23);
      const bool plain = ex > 0 && ex < 254;
      q_scale *= plain ? __int_as_float(ex << 23) : 1.0f;
      const float inv = plain ? __int_as_float((254 - ex) << 23) : 1.0f;
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

  struct Tile {
    Raw<16> k[2][KL];
    Raw<VB> v[8];
    v4f ks[2], vs[2];
    uint32_t there;
  };
  // The rows of the tile at `t0`: lane l looks up token l % 32, and everybody fetches what is theirs.
  auto fetch = [&](int t0, int buf, Tile &x) {
    TileRows &r = rows[wave][buf];
    const int tok = t0 + (lane & 31);
    const uint32_t pg = p.page_size.div((uint32_t)tok), place = (uint32_t)tok - pg * p.page_size.d;
    const int page = tok < end ? table[pg] : -1;
    const bool there = (uint32_t)page < (uint32_t)p.pages;
    x.there = (uint32_t)__ballot(there);
    const int64_t at = there ? page * p.page + place * p.token : 0;
    if (lane < 32) r.at[lane] = at;
    if constexpr (S8) {
      const float *src = lane < 32 ? p.k_scale : p.v_scale;
      const float s = there ? src[page * p.spage + place * p.stoken + kvh * p.shead] : 1.0f;
      r.scale[lane] = lane < 32 ? s : __log2f(s);
    }
    lanes_meet();
    const C *k = static_cast<const C *>(p.k) + kvh * p.head, *v = static_cast<const C *>(p.v) + kvh * p.head;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const C *row = k + r.at[16 * h + c16];
#pragma unroll
      for (int i = 0; i < KL; ++i) {
        const int d = (i * 4 + g) * (16 / (int)sizeof(C));
        x.k[h][i] = load_raw<16>(row + (d < p.dim ? d : 0));
      }
    }
    const int dv = c16 * E < p.dim ? c16 * E : 0;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) x.v[4 * h + j] = load_raw<VB>(v + r.at[16 * h + 4 * g + j] + dv);
    if constexpr (S8) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        x.ks[h] = *reinterpret_cast<const v4f *>(&r.scale[16 * h + 4 * g]);
        x.vs[h] = *reinterpret_cast<const v4f *>(&r.scale[32 + 16 * h + 4 * g]);
      }
    }
  };

  auto attend = [&](Tile &x) {
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
      for (int j = 0; j < 4; ++j) s[4 * h + j] = acc[j] * (S8 ? q_scale * x.ks[h][j] : q_scale);
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
    float w[8], top = m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = S8 ? s[j] + x.vs[j >> 2][j & 3] : s[j];
      top = fmaxf(top, w[j]);
    }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float base = top == -INFINITY ? 0.0f : top, shrink = __builtin_amdgcn_exp2f(m - base);
    m = top;
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sum += __builtin_amdgcn_exp2f(s[j] - base);
      w[j] = __builtin_amdgcn_exp2f(w[j] - base);
    }
    l = l * shrink + sum;
    typedef H t8 __attribute__((ext_vector_type(8)));
    t8 wh;
#pragma unroll
    for (int j = 0; j < 8; ++j) wh[j] = (H)w[j];
    const v4i pt = __builtin_bit_cast(v4i, wh);
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
#pragma unroll
      for (int j = 0; j < 4; ++j) o[n][j] *= shrink;
      o[n] = Op::mfma(a, pt, o[n]);
    }
  };

  for (int t0 = first + wave * TILE; t0 < end; t0 += WAVES * TILE) {
    Tile x;
    fetch(t0, 0, x);
    attend(x);
  }
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);

  // the four waves join in LDS
  if (g == 0) ml[wave][c16][0] = m, ml[wave][c16][1] = l;
  __syncthreads();
  float top = ml[0][c16][0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) top = fmaxf(top, ml[w][c16][0]);
  const float shrink = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
#pragma unroll
  for (int n = 0; n < E; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) part[wave][c16][(4 * g + j) * E + n] = o[n][j] * shrink;
  __syncthreads();
  for (int i = threadIdx.x; i < heads * DP; i += 64 * WAVES) {
    const int h = i / DP, d = i % DP;
    float mh = ml[0][h][0], sum = 0.0f, of = 0.0f;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) mh = fmaxf(mh, ml[w][h][0]);
    const float base = mh == -INFINITY ? 0.0f : mh;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      sum += ml[w][h][1] * __builtin_amdgcn_exp2f(ml[w][h][0] - base);
      of += part[w][h][d];
    }
    if (d >= p.dim) continue;
    if (p.splits == 1) {
      static_cast<Q *>(p.out)[b * p.ot + (hq0 + h) * p.oh + d] = (Q)(sum == 0.0f ? 0.0f : of / sum);
    } else {
      const int64_t at = ((int64_t)b * p.q_heads + hq0 + h) * p.splits + split;
      p.part_o[at * p.dim + d] = of;
      if (d == 0) p.part_ml[2 * at] = mh, p.part_ml[2 * at + 1] = sum;
    }
  }
}

// The stretches of a request and head, in their order: 4 groups of 64 lanes take every fourth.
template <typename Q>
__global__ __launch_bounds__(256) void join_kernel(AttendParams p) {
  __shared__ float part[4][256], sums[4];
  const int hq = blockIdx.x, b = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int len = min(max(p.lens[b], 0), p.max_len), n = (len + p.chunk - 1) / p.chunk;
  const int64_t at = ((int64_t)b * p.q_heads + hq) * p.splits;
  float top = -INFINITY;
  for (int i = lane; i < n; i += 64) top = fmaxf(top, p.part_ml[2 * (at + i)]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float base = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f, o[4] = {0, 0, 0, 0};
#pragma unroll 4
  for (int i = wave; i < n; i += 4) {
    const float f = __builtin_amdgcn_exp2f(p.part_ml[2 * (at + i)] - base);
    sum += f * p.part_ml[2 * (at + i) + 1];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane + 64 * k < p.dim) o[k] = __builtin_fmaf(f, p.part_o[(at + i) * p.dim + lane + 64 * k], o[k]);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) part[wave][lane + 64 * k] = o[k];
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  const int d = threadIdx.x;
  if (d >= p.dim) return;
  const float total = sums[0] + sums[1] + sums[2] + sums[3], of = part[0][d] + part[1][d] + part[2][d] + part[3][d];
  static_cast<Q *>(p.out)[b * p.ot + hq * p.oh + d] = (Q)(total == 0.0f ? 0.0f : of / total);
}

template <typename C, typename Q>
f8_status launch(const AttendParams &p, int batch, int kv_heads, hipStream_t s) {
  const int chunks = (p.group + HEADS - 1) / HEADS;
  const dim3 grid(kv_heads * chunks, p.splits, batch), block(64 * WAVES);
  if (p.dim <= 64) hipLaunchKernelGGL((attend_kernel<C, Q, 64>), grid, block, 0, s, p);
  else if (p.dim <= 128) hipLaunchKernelGGL((attend_kernel<C, Q, 128>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((attend_kernel<C, Q, 256>), grid, block, 0, s, p);
  f8_status st = launch_status();
  if (st != F8_OK || p.splits == 1) return st;
  hipLaunchKernelGGL(join_kernel<Q>, dim3(p.q_heads, batch), dim3(256), 0, s, p);
  return launch_status();
}

struct Split {
  int splits, chunk;
};
// Stretches of whole rounds of the four waves (128 tokens), as many as give the chip some workgroups per CU.
Split split_of(int batch, int kv_heads, int group, int max_len) {
  const int64_t wgs = (int64_t)batch * kv_heads * ((group + HEADS - 1) / HEADS);
  const int64_t rounds = (max_len + WAVES * TILE - 1) / (WAVES * TILE);
  int64_t want = wgs > 0 ? (2048 + wgs - 1) / wgs : 1;
  want = want < rounds ? want : rounds;
  if (want < 1) want = 1;
  const int64_t per = rounds ? (rounds + want - 1) / want : 1;
  return Split{(int)(rounds ? (rounds + per - 1) / per : 1), (int)per * WAVES * TILE};
}

}  // namespace
}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_attend_workspace_bytes(int batch, int q_heads, int kv_heads, int dim, int max_len) {
  if (batch < 1 || q_heads < 1 || kv_heads < 1 || dim < 1 || max_len < 1 || q_heads % kv_heads != 0) return 0;
  const Split s = split_of(batch, kv_heads, q_heads / kv_heads, max_len);
  return s.splits == 1 ? 0 : (size_t)batch * q_heads * s.splits * (dim + 2) * sizeof(float);
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
  if (!q || !k_cache || !v_cache || !table || !lens || !out || (codes && (!k_scale || !v_scale))) return F8_ERR_NULL;
  const size_t e = bytes_of(c->type);
  if (!aligned_to(q, 2) || !aligned_to(out, 2) || !aligned_to(table, 4) || !aligned_to(lens, 4) || !aligned_to(k_scale, 4) || !aligned_to(v_scale, 4) ||
      !aligned_to(k_cache, 16) || !aligned_to(v_cache, 16) || c->page_stride * e % 16 || c->token_stride * e % 16 || c->head_stride * e % 16)
    return F8_ERR_ALIGN;
  const int group = d->q_heads / c->heads;
  const Split s = split_of(d->batch, c->heads, group, d->max_len);
  if (s.splits > 65535) return F8_ERR_UNSUPPORTED;
  const size_t rows = (size_t)d->batch * d->q_heads * s.splits;
  if (s.splits > 1) {
    if (!workspace) return F8_ERR_NULL;
    if (!aligned_to(workspace, 16)) return F8_ERR_ALIGN;
    if (workspace_bytes < rows * (c->dim + 2) * sizeof(float)) return F8_ERR_SHAPE;
  }
  float *ws = static_cast<float *>(workspace);
  const AttendParams p{q, k_cache, v_cache, k_scale, v_scale, table, lens, out, ws, ws ? ws + rows * c->dim : nullptr,
                       d->q_token, d->q_head, d->o_token, d->o_head, c->page_stride, c->token_stride, c->head_stride,
                       c->scale_page, c->scale_token, c->scale_head, d->table_ld, d->q_heads, group, c->dim, c->pages, d->max_len,
                       s.splits, s.chunk, FastDiv((uint32_t)c->page_size), d->scale * LOG2E};
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (codes) return d->type == F8_F16 ? launch<int8_t, f16>(p, d->batch, c->heads, hs) : launch<int8_t, bf16>(p, d->batch, c->heads, hs);
  return d->type == F8_F16 ? launch<f16, f16>(p, d->batch, c->heads, hs) : launch<bf16, bf16>(p, d->batch, c->heads, hs);
}

}  // extern "C"
