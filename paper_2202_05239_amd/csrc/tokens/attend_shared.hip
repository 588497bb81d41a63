// Attention of one new token per request over a paged cache whose requests begin alike: groups of neighbouring requests have their first
// tokens in common (the prompt of a beam search, the instructions in front of a batch's questions), which are read once for all of a group.
//
//   o = sum_t exp(s_t) v_t / sum_t exp(s_t)   over the prefix and the request's own tokens:
//
// both parts leave a maximum, a sum and a sum of values, which a second launch joins.  The prefix's part is a product with many rows, the query heads of
// all the group's requests; as in f8_attend_paged both of its products run on the matrix cores with query heads as columns, S^T = K Q^T and
// O^T = V^T P^T, the scores leaving the first one as the second one's operand, and K and V go from memory into registers: there by a tile for 16
// columns, here for up to NB times 16 at once, so that what a tile costs to load, to bring into the products' form and, for 8 bits, to
// convert, is shared among them.
#include <math.h>

#include <type_traits>

#include "attend_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

constexpr int WAVES = 4, TILE = 32, COLS = 16, UNIT = WAVES * TILE, THREADS = 64 * WAVES;
constexpr int GROUPS_LDS = 1024;             // groups whose bounds a workgroup keeps in LDS
constexpr int WGS = 256;
// The maximum that weights are taken against follows the scores only where they pass it by more than this, as a power of two: the
// lanes of a column then seldom have to agree on a new one.
constexpr float SLACK = 4.0f;

struct SharedParams {
  const void *q, *k, *v;
  const float *k_scale, *v_scale;
  const int32_t *table, *lens, *first, *shared;
  void *out;
  float *part_o, *part_ml;                   // [pieces][dim] and [pieces][2]
  int64_t qt, qh, ot, oh, page, token, head, spage, stoken, shead, table_ld;
  int batch, groups, heads, group, chunks, per_block, dim, pages, max_len, wgs;
  int rows;                                  // of a block: query heads of per_block requests, or some of one request's
  FastDiv page_size, by_group;
  float scale;                               // of the scores, times log2 e
};

// How the work is dealt out.  An item is a group (its prefix) or a request (its own tokens).  A pair is an item, a cache head and a block
// of up to `rows` query heads that read it; its units are rounds of a workgroup's waves over its tokens.  All units lie in a row, groups first, and
// every workgroup takes an equal run of them.  A pair that lies in one run leaves its piece at its own place; one that is cut leaves a piece in each
// run, at slot 1 of the run that it begins in and at slot 0 of the others.
struct Prefix {
  int b0, n, tokens;                         // requests b0 .. b0 + n - 1
};
struct Work {
  const SharedParams &p;
  const int32_t *first;                      // (in LDS where it fits)
  __device__ __forceinline__ int len(int b) const { return min(max(p.lens[b], 0), p.max_len); }
  __device__ __forceinline__ Prefix prefix(int g) const {
    const int b0 = min(max(first[g], 0), p.batch), n = min(max(first[g + 1], 0), p.batch) - b0;
    return Prefix{b0, n, n > 1 ? min(max(p.shared[g], 0), p.max_len) : 0};
  }
  // The group that request b belongs to, or -1
  __device__ __forceinline__ int group_of(int b) const {
    int lo = 0, hi = p.groups;               // the last group that begins at b or before it: in lo .. hi - 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= b) lo = mid;
      else hi = mid;
    }
    return first[lo] <= b && b < first[lo + 1] ? lo : -1;
  }
  // Tokens of request b that its group reads for it: all of the prefix, or nothing where it ends inside it
  __device__ __forceinline__ int prefix_of(int b) const {
    const int g = group_of(b), n = g < 0 ? 0 : prefix(g).tokens;
    return n <= len(b) ? n : 0;
  }
  static __device__ __forceinline__ int units(int tokens) { return (tokens + UNIT - 1) / UNIT; }
  __device__ __forceinline__ int blocks(int requests) const { return (requests + p.per_block - 1) / p.per_block * p.chunks; }
  __device__ __forceinline__ int64_t units_of(int item) const {
    if (item < p.groups) {
      const Prefix x = prefix(item);
      return x.tokens > 0 ? (int64_t)units(x.tokens) * p.heads * blocks(x.n) : 0;
    }
    const int b = item - p.groups;
    return (int64_t)units(len(b) - prefix_of(b)) * p.heads * p.chunks;
  }
};
// Pieces: of pairs in one run [2][batch][query heads] (the prefix's part, the own part), then [workgroups][2][rows].
__device__ __forceinline__ int64_t whole_at(const SharedParams &p, bool own, int b, int hq) {
  return ((int64_t)(own ? p.batch : 0) + b) * p.heads * p.group + hq;
}
__device__ __forceinline__ int64_t cut_at(const SharedParams &p, int64_t run, int slot, int row) {
  return (int64_t)2 * p.batch * p.heads * p.group + (2 * run + slot) * p.rows + row;
}

__device__ __forceinline__ const int32_t *bounds(const SharedParams &p, int32_t *lds, int threads) {
  if (p.groups > GROUPS_LDS) return p.first;
  for (int i = threadIdx.x; i <= p.groups; i += threads) lds[i] = p.first[i];
  __syncthreads();
  return lds;
}

struct TileRows {
  int64_t at[TILE];
  float scale[3 * TILE];
};

// Powers of two: the weight of the largest score, which leaves room for SLACK above it.
template <typename C>
constexpr float up() { return Operand<C>::UP > SLACK ? Operand<C>::UP - SLACK : 0.0f; }

// What a weight has at least, so that it counts against an infinite value whatever its type holds: f16's smallest number, 2^-35 of the
// largest weight.
template <typename C>
constexpr float floor_of() { return __is_same(C, f16) ? 0x1p-24f : 0.0f; }

template <typename C, typename Q, int DP, int NB>
__global__ __launch_bounds__(THREADS, 1) void attend_shared_kernel(SharedParams p) {
  typedef Operand<C> Op;
  typedef typename Op::t H;
  typedef H t8 __attribute__((ext_vector_type(8)));
  constexpr bool S8 = sizeof(C) == 1;
  constexpr int E = DP / 16, VB = E * (int)sizeof(C);     // elements and bytes of a value row per lane
  constexpr int KL = DP * (int)sizeof(C) / 64;            // 16-byte loads of a key row per lane
  constexpr int KS = DP / 32;                             // products per block of 16 scores
  __shared__ TileRows rows[WAVES][2];
  __shared__ float part[WAVES][COLS][DP + 1], ml[WAVES][NB * COLS][2];
  __shared__ int64_t scan[WAVES][2], before;
  __shared__ int from, found[WAVES];
  __shared__ int32_t first_lds[GROUPS_LDS + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c16 = lane & 15, g = lane >> 4;
  const Work work{p, bounds(p, first_lds, THREADS)};
  // (runs that follow one another lie on one XCD: the blocks of a head meet in its L2)
  const uint32_t run = xcd_remap(blockIdx.x, gridDim.x);
  const int items = p.groups + p.batch;

  // the item that holds the run's first unit
  int64_t left, start, done = 0;
  {
    int64_t sum[2] = {0, 0};
    for (int i = threadIdx.x; i < items; i += THREADS) sum[0] += work.units_of(i);
    wg_sum<WAVES>(sum, scan);
    const Runs runs(uniform64(sum[0]), p.wgs);
    start = runs.start(run);
    left = runs.start((int64_t)run + 1) - start;
    if (left == 0) return;
  }
  for (int i0 = 0;; i0 += THREADS) {
    const int i = i0 + (int)threadIdx.x;
    const int64_t mine = i < items ? work.units_of(i) : 0;
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
    if (mine > 0 && at <= start && start < at + mine) from = i, before = at;
    __syncthreads();
    done += all;
    if (start < done) break;
  }
  int item = __builtin_amdgcn_readfirstlane(from);
  left = uniform64(left);
  int64_t in = uniform64(start - before);       // units of the item in front of this run

  for (bool more = true; more;) {
    // the pair: requests b0 .. b0 + n - 1, `heads` query heads of cache head kvh from hq0 on, tokens t_begin .. t_end - 1 of row `leader` of the table
    const bool own = item >= p.groups;
    int b0, n, t_begin, t_end, leader, pairs;
    if (own) {
      b0 = item - p.groups, n = 1, t_begin = work.prefix_of(b0), t_end = work.len(b0), leader = b0, pairs = p.heads * p.chunks;
    } else {
      const Prefix x = work.prefix(item);
      b0 = x.b0, n = x.n, t_begin = 0, t_end = x.tokens, leader = b0, pairs = p.heads * work.blocks(n);
    }
    b0 = __builtin_amdgcn_readfirstlane(b0), n = __builtin_amdgcn_readfirstlane(n), leader = b0;
    t_begin = __builtin_amdgcn_readfirstlane(t_begin), t_end = __builtin_amdgcn_readfirstlane(t_end);
    pairs = __builtin_amdgcn_readfirstlane(pairs);
    if (!own && work.len(leader) < t_end) {
      // (an empty place in front) the first member that has all of the prefix; without any nobody reads what comes out
      int have = 0x7fffffff;
      for (int i = b0 + (int)threadIdx.x; i < b0 + n && have == 0x7fffffff; i += THREADS)
        if (work.len(i) >= t_end) have = i;
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) have = min(have, __shfl_xor(have, d));
      if (lane == 0) found[wave] = have;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < WAVES; ++w) have = min(have, found[w]);
      __syncthreads();
      leader = __builtin_amdgcn_readfirstlane(have);
      if (leader == 0x7fffffff) leader = b0, t_end = 0;
    }
    const int units = work.units(own ? t_end - t_begin : work.prefix(item).tokens);
    const int pair = __builtin_amdgcn_readfirstlane((int)(in / units));
    int unit = __builtin_amdgcn_readfirstlane((int)(in - (int64_t)pair * units));
    const int blocks = pairs / p.heads, kvh = pair / blocks, block = pair - kvh * blocks;
    const int chunk = block % p.chunks, req0 = block / p.chunks * p.per_block;
    const int h0 = chunk * p.rows, heads = p.chunks > 1 ? min(p.rows, p.group - h0) : p.group;
    const int real_rows = min(n - req0, p.per_block) * heads, nb_used = (real_rows + COLS - 1) / COLS;
    const int last = (int)min((int64_t)units, unit + left), begin = t_begin + unit * UNIT, end = min(t_end, t_begin + last * UNIT);
    const int32_t *table = p.table + leader * p.table_ld;
    auto place = [&](int row, int &b, int &hq) {             // of a row of the block
      const int r = p.chunks > 1 ? 0 : (int)p.by_group.div((uint32_t)row);
      b = b0 + req0 + r, hq = kvh * p.group + h0 + row - r * heads;
    };

    // Q^T as the right operand: the lane's column, the dimensions that its loads of K bring
    v4i q[NB][KS];
    float q_scale[NB];
    const bool negative = p.scale < 0;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      q_scale[nb] = fabsf(p.scale);
      if (nb >= nb_used) continue;
      const int row = nb * COLS + c16;
      int b, hq;
      place(min(row, real_rows - 1), b, hq);
      const Q *src = static_cast<const Q *>(p.q) + b * p.qt + hq * p.qh;
      v4i raw[KS];
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int d = S8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
        __builtin_memcpy(&raw[s], src + (d < p.dim ? d : 0), 16);
      }
      float f[KS][8];
      uint32_t top = 0;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int d = S8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
        unpack8<Q>(&raw[s], f[s]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          f[s][j] = row < real_rows && d < p.dim ? (negative ? -f[s][j] : f[s][j]) : 0.0f;
          top = max(top, magnitude(f[s][j]));
        }
      }
      if constexpr (S8) {
        // a power of two brings the largest element of the row to [2^14, 2^15): f16 then holds what the 16-bit q had, elements
        // 2^-28 below the largest excepted
        top = max(top, (uint32_t)__shfl_xor((int)top, 16));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32));
        const int ex = max((int)(top >> 23), 15);             // (the two factors are then normal numbers, for an infinity's exponent too)
        q_scale[nb] *= __int_as_float((ex - 14) << 23);
        const float inv = __int_as_float((268 - ex) << 23);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
          for (int j = 0; j < 8; ++j) f[s][j] *= inv;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        t8 o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = (H)f[s][j];
        q[nb][s] = __builtin_bit_cast(v4i, o);
      }
    }

    v4f o[NB][E];
    float m[NB], l[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      m[nb] = -INFINITY, l[nb] = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[nb][e] = v4f{0, 0, 0, 0};
    }

    const C *const kbase = static_cast<const C *>(p.k) + kvh * p.head, *const vbase = static_cast<const C *>(p.v) + kvh * p.head;
    const int dv = c16 * E < p.dim ? c16 * E : 0;
    // The rows of a tile in registers.  The next one's keys are loaded when this one's scores are there, its values when this one's have been summed
    // up: every load has half a tile's time on its way and no register waits twice.
    Raw<16> k[2][KL];
    Raw<VB> v[8];
    float tile_scale;                         // lanes 0..31: of the key of token `lane`, 32..63: of the value of token `lane - 32`
    uint32_t there;                           // its tokens that exist
    auto look_up = [&](int t0) {              // page of token lane % 32 of the tile at t0
      const int tok = t0 + (lane & 31);
      return tok < end ? table[p.page_size.div((uint32_t)tok)] : -1;
    };
    auto locate = [&](int t0, int page, int64_t (&at_lds)[TILE]) {
      const uint32_t tok = (uint32_t)(t0 + (lane & 31)), place = tok - p.page_size.div(tok) * p.page_size.d;
      const bool real = (uint32_t)page < (uint32_t)p.pages;
      const int64_t at = real ? page * p.page + place * p.token : 0;
      if (lane < 32) at_lds[lane] = at;
      lanes_meet();
      if constexpr (S8) {
        const float *src = lane < 32 ? p.k_scale : p.v_scale;
        tile_scale = real ? src[page * p.spage + place * p.stoken + kvh * p.shead] : 1.0f;
      }
      return (uint32_t)__ballot(real);
    };
    auto load_keys = [&](const int64_t (&at_lds)[TILE]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const C *row = kbase + at_lds[16 * h + c16];
#pragma unroll
        for (int i = 0; i < KL; ++i) {
          const int d = (i * 4 + g) * (16 / (int)sizeof(C));
          k[h][i] = load_raw<16>(row + (d < p.dim ? d : 0));
        }
      }
    };
    auto load_values = [&](const int64_t (&at_lds)[TILE]) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * h + j] = load_raw<VB>(vbase + at_lds[16 * h + 4 * g + j] + dv);
    };

    // All tiles of this wave, for N blocks of columns: no branch between a tile's products
    auto walk = [&](auto blocks_used) {
      constexpr int N = decltype(blocks_used)::value;
      int t0 = begin + wave * TILE, buf = 0;
      if (t0 >= end) return;
      there = locate(t0, look_up(t0), rows[wave][0].at);
      load_keys(rows[wave][0].at);
      load_values(rows[wave][0].at);
      int page = look_up(t0 + UNIT);
      for (;;) {
        const bool next = t0 + UNIT < end;
        const uint32_t now = there;
        v4f ks[2], vs[2], vl[2];
        if constexpr (S8) {
          float *const scale_lds = rows[wave][buf].scale;
          scale_lds[lane] = tile_scale;
          if (lane >= 32) scale_lds[32 + lane] = fmaxf(__log2f(tile_scale), SMALL);
          lanes_meet();
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            ks[h] = *reinterpret_cast<const v4f *>(scale_lds + 16 * h + 4 * g);
            vs[h] = *reinterpret_cast<const v4f *>(scale_lds + 32 + 16 * h + 4 * g);
            vl[h] = *reinterpret_cast<const v4f *>(scale_lds + 64 + 16 * h + 4 * g);
          }
        }
        v4f acc[N][2];
#pragma unroll
        for (int nb = 0; nb < N; ++nb) acc[nb][0] = acc[nb][1] = v4f{0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < KL; ++i) {
            const bool real = (i * 4 + g) * (16 / (int)sizeof(C)) < p.dim;
            uint32_t d[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) d[j] = real ? k[h][i].d[j] : 0u;
            if constexpr (S8) {
              h8 lo, hi;
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t u = d[j] ^ 0x80808080u;
                const h2 a = codes_lo(u), e = codes_hi(u);
                h8 &to = j < 2 ? lo : hi;
                to[4 * (j & 1)] = a[0], to[4 * (j & 1) + 1] = a[1], to[4 * (j & 1) + 2] = e[0], to[4 * (j & 1) + 3] = e[1];
              }
#pragma unroll
              for (int nb = 0; nb < N; ++nb) acc[nb][h] = Op::mfma(__builtin_bit_cast(v4i, lo), q[nb][2 * i], acc[nb][h]);
#pragma unroll
              for (int nb = 0; nb < N; ++nb) acc[nb][h] = Op::mfma(__builtin_bit_cast(v4i, hi), q[nb][2 * i + 1], acc[nb][h]);
            } else {
#pragma unroll
              for (int nb = 0; nb < N; ++nb) acc[nb][h] = Op::mfma(v4i{(int)d[0], (int)d[1], (int)d[2], (int)d[3]}, q[nb][i], acc[nb][h]);
            }
          }
        if (next) {
          const int ahead = look_up(t0 + 2 * UNIT);
          there = locate(t0 + UNIT, page, rows[wave][buf ^ 1].at);
          load_keys(rows[wave][buf ^ 1].at);
          page = ahead;
        }
#pragma unroll
        for (int nb = 0; nb < N; ++nb)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[nb][h][j] *= S8 ? q_scale[nb] * ks[h][j] : q_scale[nb];
        if (now != 0xffffffffu) {
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const bool real = now >> (16 * h + 4 * g + j) & 1;
#pragma unroll
              for (int nb = 0; nb < N; ++nb) acc[nb][h][j] = real ? acc[nb][h][j] : -INFINITY;
#pragma unroll
              for (int w = 0; w < VB / 4; ++w) v[4 * h + j].d[w] = real ? v[4 * h + j].d[w] : 0u;   // (0 * NaN is NaN)
            }
        }
        // the maximum of the scores (of what the values weigh, for 8 bits)
        float top[N];
        bool rises = false;
#pragma unroll
        for (int nb = 0; nb < N; ++nb) {
          top[nb] = -INFINITY;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) top[nb] = fmaxf(top[nb], S8 ? acc[nb][h][j] + vl[h][j] : acc[nb][h][j]);
          rises = rises || top[nb] > m[nb] + SLACK;
        }
        if (__any(rises)) {                   // (seldom in a long context)
#pragma unroll
          for (int nb = 0; nb < N; ++nb) {
            float to = fmaxf(top[nb], m[nb]);
            to = fmaxf(to, __shfl_xor(to, 16));
            to = fmaxf(to, __shfl_xor(to, 32));
            const float shrink = __builtin_amdgcn_exp2f(m[nb] - (to == -INFINITY ? 0.0f : to));
            l[nb] *= shrink;
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll
              for (int j = 0; j < 4; ++j) o[nb][e][j] *= shrink;
            m[nb] = to;
          }
        }
        v4i pt[N];
#pragma unroll
        for (int nb = 0; nb < N; ++nb) {
          const float below = (m[nb] == -INFINITY ? 0.0f : m[nb]) - up<C>();
          t8 wh;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float w = __builtin_amdgcn_exp2f(acc[nb][j >> 2][j & 3] - below);
            l[nb] += w;
            wh[j] = (H)(S8 ? w * vs[j >> 2][j & 3] : w + floor_of<C>());
          }
          pt[nb] = __builtin_bit_cast(v4i, wh);
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
          v4i a;
          if constexpr (S8) {
            const uint32_t sel = 0x0c000c00u | (uint32_t)(e & 3) | (uint32_t)(4 + (e & 3)) << 16;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t u = __builtin_amdgcn_perm(v[2 * j + 1].d[e >> 2], v[2 * j].d[e >> 2], sel) ^ 0x64806480u;
              a[j] = __builtin_bit_cast(int, __builtin_bit_cast(h2, u) - h2{(f16)1152, (f16)1152});
            }
          } else {
            const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
            for (int j = 0; j < 4; ++j) a[j] = (int)__builtin_amdgcn_perm(v[2 * j + 1].d[e >> 1], v[2 * j].d[e >> 1], sel);
          }
#pragma unroll
          for (int nb = 0; nb < N; ++nb) o[nb][e] = Op::mfma(a, pt[nb], o[nb][e]);
        }
        // The results of the last products are there before any branch: behind one the compiler (ROCm 7.2) has read an
        // accumulator without the wait that a matrix instruction's result needs.
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 15" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if (!next) break;
        load_values(rows[wave][buf ^ 1].at);
        buf ^= 1, t0 += UNIT;
      }
    };
    if constexpr (NB >= 4) {
      if (nb_used > 2) walk(std::integral_constant<int, 4>());
      else if (nb_used > 1) walk(std::integral_constant<int, 2>());
      else walk(std::integral_constant<int, 1>());
    } else {
      if (nb_used > 1) walk(std::integral_constant<int, 2>());
      else walk(std::integral_constant<int, 1>());
    }

    // the waves join in LDS, 16 columns at a time, and leave the piece
    const bool whole = unit == 0 && last == units;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (nb >= nb_used) continue;
      l[nb] += __shfl_xor(l[nb], 16);
      l[nb] += __shfl_xor(l[nb], 32);
      if (g == 0) ml[wave][nb * COLS + c16][0] = m[nb], ml[wave][nb * COLS + c16][1] = l[nb];
    }
    __syncthreads();
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if (nb >= nb_used) continue;
      float top = ml[0][nb * COLS + c16][0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) top = fmaxf(top, ml[w][nb * COLS + c16][0]);
      const float shrink = __builtin_amdgcn_exp2f(m[nb] - (top == -INFINITY ? 0.0f : top));
#pragma unroll
      for (int e = 0; e < E; ++e)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[wave][c16][(4 * g + j) * E + e] = o[nb][e][j] * shrink;
      __syncthreads();
      for (int i = threadIdx.x; i < COLS * DP; i += THREADS) {
        const int c = i / DP, d = i % DP, row = nb * COLS + c;
        if (row >= real_rows || d >= p.dim) continue;
        float mh = ml[0][row][0], sum = 0.0f, of = 0.0f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) mh = fmaxf(mh, ml[w][row][0]);
        const float base = mh == -INFINITY ? 0.0f : mh;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          sum += ml[w][row][1] * __builtin_amdgcn_exp2f(ml[w][row][0] - base);
          of += part[w][c][d];
        }
        int b, hq;
        place(row, b, hq);
        const int64_t at = whole ? whole_at(p, own, b, hq) : cut_at(p, run, unit == 0, row);
        p.part_o[at * p.dim + d] = of;
        if (d == 0) p.part_ml[2 * at] = mh, p.part_ml[2 * at + 1] = sum;
      }
      __syncthreads();
    }
    left -= last - unit;
    more = left > 0;
    in += last - unit;
    if (more && in == (int64_t)units * pairs) {               // the next item that has units
      in = 0;
      do ++item;
      while (work.units_of(item) == 0);
      item = __builtin_amdgcn_readfirstlane(item);
    }
  }
}

// Both parts of a request's heads together.  A workgroup takes JOIN_PART elements (heads by dimensions) of a request, a cache head and a chunk of
// its query heads, 4 neighbours a thread and as many pieces at a time as threads are left; the pieces are added up in a fixed order.
constexpr int JOINERS = 4, JOIN_PART = 256, JOIN_VECS = JOIN_PART / 4, JOIN_AT_ONCE = 64 * JOINERS / JOIN_VECS;

template <typename Q>
__global__ __launch_bounds__(64 * JOINERS) void join_shared_kernel(SharedParams p) {
  __shared__ v4f part[JOIN_AT_ONCE][JOIN_VECS];
  __shared__ float sums[JOIN_AT_ONCE][JOIN_VECS], tops[JOIN_AT_ONCE][JOIN_VECS];
  __shared__ int64_t scan[JOINERS][2];
  __shared__ int32_t first_lds[GROUPS_LDS + 1];
  const Work work{p, bounds(p, first_lds, 64 * JOINERS)};
  const int per_b = p.heads * p.chunks, b = blockIdx.x / per_b, hc = blockIdx.x % per_b, kvh = hc / p.chunks, chunk = hc % p.chunks;
  const int h0 = chunk * p.rows, heads = p.chunks > 1 ? min(p.rows, p.group - h0) : p.group;
  const int vec = (int)threadIdx.x % JOIN_VECS, mine = (int)threadIdx.x / JOIN_VECS;
  // (dim is a multiple of 16: four neighbours belong to one head)
  const int e = blockIdx.y * JOIN_PART + vec * 4, h = e / p.dim, d = e - h * p.dim;
  const bool real = h < heads;
  const int hq = kvh * p.group + h0 + (real ? h : 0), col = real ? d : 0;
  // units in front of the group and of the request, and all of them
  const int g = work.group_of(b), own = p.groups + b, prefix = work.prefix_of(b);
  const Prefix x = g < 0 ? Prefix{0, 0, 0} : work.prefix(g);
  int64_t sum[2] = {0, 0}, front[2] = {0, 0};
  for (int i = threadIdx.x; i < p.groups + p.batch; i += 64 * JOINERS) {
    const int64_t u = work.units_of(i);
    sum[0] += u;
    if (i < own) front[0] += u;
    if (i < g) front[1] += u;
  }
  wg_sum<JOINERS>(sum, scan);
  wg_sum<JOINERS>(front, scan);
  const Runs runs(uniform64(sum[0]), p.wgs);
  // pieces of the prefix's pair and of the own one: places i0 .. i0 + n - 1
  struct Pieces {
    int64_t first, rest;                      // rows of piece 0 and 1; the others follow 2 * rows apart
    int n;
  };
  auto pieces = [&](int64_t at, int units, bool is_own, int row) {
    if (units == 0) return Pieces{0, 0, 0};
    const int64_t i0 = runs.of(at), i1 = runs.of(at + units - 1);
    if (i0 == i1) return Pieces{whole_at(p, is_own, b, hq), 0, 1};
    return Pieces{cut_at(p, i0, 1, row), cut_at(p, i0 + 1, 0, row), (int)(i1 - i0) + 1};
  };
  const int pu = prefix > 0 ? work.units(prefix) : 0, ou = work.units(work.len(b) - prefix);
  const int blocks = work.blocks(x.n), block = (b - x.b0) / p.per_block * p.chunks + chunk;
  const Pieces a = pieces(uniform64(front[1] + ((int64_t)kvh * blocks + block) * pu), pu, false, (b - x.b0) % p.per_block * heads + (real ? h : 0));
  const Pieces c = pieces(uniform64(front[0] + (int64_t)hc * ou), ou, true, real ? h : 0);
  const int n = a.n + c.n;
  auto row_of = [&](int i) {
    const Pieces &k = i < a.n ? a : c;
    const int j = i < a.n ? i : i - a.n;
    return j == 0 ? k.first : k.rest + (int64_t)(j - 1) * 2 * p.rows;
  };
  Q *out = static_cast<Q *>(p.out) + b * p.ot + hq * p.oh + col;
  const float2 *ml = reinterpret_cast<const float2 *>(p.part_ml);
  // running maximum, as in the kernel above; four pieces on their way at a time
  float top = -INFINITY, total = 0.0f;
  v4f o{0, 0, 0, 0};
  for (int i = mine; i < n; i += 4 * JOIN_AT_ONCE) {
    float2 s[4];
    v4f v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t r = row_of(min(i + u * JOIN_AT_ONCE, n - 1));
      s[u] = ml[r];
      v[u] = *reinterpret_cast<const v4f *>(p.part_o + r * p.dim + col);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i + u * JOIN_AT_ONCE >= n) break;
      const float now = fmaxf(top, s[u].x), base = now == -INFINITY ? 0.0f : now;
      const float was = __builtin_amdgcn_exp2f(top - base), is = __builtin_amdgcn_exp2f(s[u].x - base);
      top = now;
      total = total * was + s[u].y * is;
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = o[k] * was + v[u][k] * is;
    }
  }
  part[mine][vec] = o, sums[mine][vec] = total, tops[mine][vec] = top;
  __syncthreads();
  if (mine != 0 || !real) return;
  for (int w = 1; w < JOIN_AT_ONCE; ++w) top = fmaxf(top, tops[w][vec]);
  const float base = top == -INFINITY ? 0.0f : top;
  total = 0.0f, o = v4f{0, 0, 0, 0};
#pragma unroll
  for (int w = 0; w < JOIN_AT_ONCE; ++w) {
    const float f = __builtin_amdgcn_exp2f(tops[w][vec] - base);
    total += sums[w][vec] * f;
#pragma unroll
    for (int k = 0; k < 4; ++k) o[k] += part[w][vec][k] * f;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) out[k] = (Q)(total == 0.0f ? 0.0f : o[k] / total);
}

// Blocks of columns of a workgroup, by the registers that a column's output takes.
constexpr int blocks_of(int dim) { return dim <= 128 ? 4 : 2; }

template <typename C, typename Q>
f8_status launch(const SharedParams &p, hipStream_t s) {
  const dim3 grid(p.wgs), block(THREADS);
  if (p.dim <= 64) hipLaunchKernelGGL((attend_shared_kernel<C, Q, 64, blocks_of(64)>), grid, block, 0, s, p);
  else if (p.dim <= 128) hipLaunchKernelGGL((attend_shared_kernel<C, Q, 128, blocks_of(128)>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((attend_shared_kernel<C, Q, 256, blocks_of(256)>), grid, block, 0, s, p);
  const f8_status st = launch_status();
  if (st != F8_OK) return st;
  const int elements = (p.chunks > 1 ? p.rows : p.group) * p.dim;
  hipLaunchKernelGGL(join_shared_kernel<Q>, dim3(p.batch * p.heads * p.chunks, (elements + JOIN_PART - 1) / JOIN_PART), dim3(64 * JOINERS), 0, s, p);
  return launch_status();
}

// Where a request's tokens fit one launch of f8_attend_paged, that is the faster way.
bool alone(int groups, int max_len) { return groups == 0 || max_len <= 4 * UNIT; }
size_t pieces_of(int64_t batch, int q_heads, int dim) { return (size_t)2 * batch * q_heads + (size_t)2 * WGS * blocks_of(dim) * COLS; }

}  // namespace
}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_attend_shared_workspace_bytes(int batch, int groups, int q_heads, int kv_heads, int dim, int max_len) {
  if (batch < 1 || groups < 0 || q_heads < 1 || kv_heads < 1 || dim < 1 || max_len < 1 || q_heads % kv_heads != 0) return 0;
  if (alone(groups, max_len)) return f8_attend_workspace_bytes(batch, q_heads, kv_heads, dim, max_len);
  return pieces_of(batch, q_heads, dim) * (dim + 2) * sizeof(float);
}

f8_status f8_attend_shared(const void *q, const void *k_cache, const void *v_cache, const float *k_scale, const float *v_scale,
                           const int32_t *table, const int32_t *lens, const int32_t *first, const int32_t *shared, void *out,
                           const f8_kv_layout *c, const f8_attend_desc *d, int groups, void *workspace, size_t workspace_bytes, void *stream) {
  if (!c || !d) return F8_ERR_NULL;
  if (groups < 0 || groups > 65535) return F8_ERR_SHAPE;
  f8_status st = check_attend(*c, *d);
  if (st != F8_OK) return st;
  if (d->batch > 0 && groups > 0 && (!first || !shared)) return F8_ERR_NULL;
  if (!aligned_to(first, 4) || !aligned_to(shared, 4)) return F8_ERR_ALIGN;
  if (d->batch == 0 || alone(groups, d->max_len))
    return f8_attend_paged(q, k_cache, v_cache, k_scale, v_scale, table, lens, out, c, d, workspace, workspace_bytes, stream);
  st = check_attend_pointers(q, k_cache, v_cache, k_scale, v_scale, table, lens, out, *c, *d);
  if (st != F8_OK) return st;
  const int group = d->q_heads / c->heads, most = blocks_of(c->dim) * COLS, chunks = (group + most - 1) / most;
  if ((int64_t)d->batch * c->heads * chunks > 1 << 22) return F8_ERR_UNSUPPORTED;          // (workgroups of a launch)
  if (!workspace) return F8_ERR_NULL;
  if (!aligned_to(workspace, 16)) return F8_ERR_ALIGN;
  if (workspace_bytes < f8_attend_shared_workspace_bytes(d->batch, groups, d->q_heads, c->heads, c->dim, d->max_len)) return F8_ERR_SHAPE;
  float *ws = static_cast<float *>(workspace);
  const SharedParams p{q, k_cache, v_cache, k_scale, v_scale, table, lens, first, shared, out, ws, ws + pieces_of(d->batch, d->q_heads, c->dim) * c->dim,
                       d->q_token, d->q_head, d->o_token, d->o_head, c->page_stride, c->token_stride, c->head_stride,
                       c->scale_page, c->scale_token, c->scale_head, d->table_ld, d->batch, groups, c->heads, group, chunks,
                       chunks > 1 ? 1 : most / group, c->dim, c->pages, d->max_len, WGS, most, FastDiv((uint32_t)c->page_size), FastDiv((uint32_t)group),
                       d->scale * LOG2E};
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (c->type == F8_S8) return d->type == F8_F16 ? launch<int8_t, f16>(p, hs) : launch<int8_t, bf16>(p, hs);
  return d->type == F8_F16 ? launch<f16, f16>(p, hs) : launch<bf16, bf16>(p, hs);
}

}  // extern "C"
