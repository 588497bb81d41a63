// Attention of one new token per request over a paged cache whose requests begin alike: groups of neighbouring requests have their first
// tokens in common (the prompt of a beam search, the instructions in front of a batch's questions), which are read once for all of a group.
//
//   o = sum_t exp(s_t) v_t / sum_t exp(s_t)   over the prefix and the request's own tokens:
//
// both parts leave a maximum, a sum and a sum of values, which a second launch joins.  The prefix's part is a product with many rows, the query heads of
// all the group's requests; as in f8_attend_paged both of its products run on the matrix cores with query heads as columns, S^T = K Q^T and
// O^T = V^T P^T, the scores leaving the first one as the second one's operand: there by a tile for 16 columns, here for up to NB times 16 at
// once, so that what a tile costs to load, to bring into the products' form and, for 8 bits, to convert, is shared among them.
//
// What bounds it: few rows behind a prefix, HBM; many rows (16 to 64 columns to a byte), the vector instructions around the products
// (of 64 columns: 330 to a tile's 64 products, exponentials of 16 cycles among them) and the waits of a wave that stands alone on its SIMD.  bf16, dim 128, 8 heads
// of 4 query heads each: 64 requests behind 32768 tokens with 512 of their own 93 us, with one of their own 74 (455 TFLOP/s; a twentieth
// less where every page is in the second-level cache).  8 bits, 16 groups of 4 behind 4096 tokens, 128 of their own: 38 us for 90 MB.
// The way to the first rows (bounds, lengths, places, rows: four latencies one after the other), the join and the second
// launch are 16 us, however little there is to read.
#include <math.h>

#include <type_traits>

#include "attend_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

constexpr int WAVES = 4, TILE = 32, COLS = 16, UNIT = WAVES * TILE, THREADS = 64 * WAVES;
constexpr int ITEMS_LDS = 512;               // groups, and requests, that a workgroup keeps in LDS
constexpr int CUS = 256;
// Workgroups and blocks of columns of a workgroup.  Two to a CU hide one another's waits, one has registers for twice the columns, or for the next
// tile's values and operands ahead of time.  One to a CU, two to a CU, us: 16 bits, dim 128 (64 and 32 columns), 64 requests behind 32768 tokens, 512
// of their own 93, 98; 3 groups of 17 behind 9001 tokens, dim 80 40, 49; 64 requests of 600 tokens of their own alone 35, 33.  16 bits, dim 64 (64
// columns each) 64, 54.  8 bits, dim 128 (64 and 32 columns) 108, 100, dim 64 77, 76; 16 groups of 4 behind 4096 tokens 44, 38.
// Larger heads' accumulators leave one.
constexpr int wgs_of(int dim, int bytes) { return dim <= 64 || (dim <= 128 && bytes == 1) ? 2 * CUS : CUS; }
constexpr int blocks_of(int dim, int bytes) { return dim <= 128 && bytes == 2 ? 4 : 2; }

// What the first launch leaves of a request for the second one: units in front of its group, tiles in front of it, its tokens and those of them that
// its group reads, the group.  One more behind the last: the units and tiles of all.
struct __align__(16) Record {
  int units, tiles, len, prefix, b0, n, unused[2];
};

struct SharedParams {
  const void *q, *k, *v;
  const float *k_scale, *v_scale;
  const int32_t *table, *lens, *first, *shared;
  void *out;
  float *part_o, *part_ml;                   // [pieces][dim] and [pieces][2]
  Record *records;                           // [batch + 1]
  int32_t *group_units;                      // [groups]: units in front of it
  int64_t qt, qh, ot, oh, page, token, head, spage, stoken, shead, table_ld;
  int batch, groups, heads, group, chunks, per_block, dim, pages, max_len, wgs;
  int rows;                                  // of a block: query heads of per_block requests, or some of one request's
  FastDiv page_size, by_group;
  float scale;                               // of the scores, times log2 e
};

// How the work is dealt out, first the prefixes and then the requests' own tokens.
// A pair of the first kind is a group, a cache head and a block of up to `rows` query heads that read it; its units are rounds of a workgroup's
// four waves over the prefix.  All units lie in a row and every workgroup takes an equal run of them.  A pair of the second kind is a request, a cache
// head and up to 16 of its query heads; its units are tiles, and every wave takes an equal run on its own: these pairs are many and
// short, and a pair's way to its first rows is 3 us (64 requests of 600 tokens, 8 heads, bf16: 35 us so, 107 with a workgroup to such a pair).
// A pair that lies in one run leaves its piece at its own place; one that is cut leaves a piece in each run, at slot 1 of the run that it begins in and at
// slot 0 of the others.
struct Prefix {
  int b0, n, tokens;                         // requests b0 .. b0 + n - 1
};
__device__ __forceinline__ int units(int tokens) { return (int)((uint32_t)(tokens + UNIT - 1) / UNIT); }
__device__ __forceinline__ int tiles(int tokens) { return (int)((uint32_t)(tokens + TILE - 1) / TILE); }
__device__ __forceinline__ int blocks_of(const SharedParams &p, int requests) { return (requests + p.per_block - 1) / p.per_block * p.chunks; }
__device__ __forceinline__ int own_chunks(const SharedParams &p) { return (p.group + COLS - 1) / COLS; }
struct Items {                               // (in LDS)
  int32_t first[ITEMS_LDS + 1], shared[ITEMS_LDS], lens[ITEMS_LDS], units[ITEMS_LDS];
};
struct Work {
  const SharedParams &p;
  Items &lds;
  __device__ __forceinline__ Work(const SharedParams &p, Items &lds) : p(p), lds(lds) {
    if (p.groups <= ITEMS_LDS)
      for (int i = threadIdx.x; i <= p.groups; i += THREADS) {
        lds.first[i] = p.first[i];
        if (i < p.groups) lds.shared[i] = p.shared[i];
      }
    if (p.batch <= ITEMS_LDS)
      for (int i = threadIdx.x; i < p.batch; i += THREADS) lds.lens[i] = p.lens[i];
    __syncthreads();
  }
  // (as an atomic, so that the compiler keeps the two kinds of memory apart: one load of either is a flat one, which all others wait for)
  static __device__ __forceinline__ int far(const int32_t *at) { return __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
  __device__ __forceinline__ int first(int g) const { return p.groups <= ITEMS_LDS ? lds.first[g] : far(p.first + g); }
  __device__ __forceinline__ int len(int b) const { return min(max(p.batch <= ITEMS_LDS ? lds.lens[b] : far(p.lens + b), 0), p.max_len); }
  __device__ __forceinline__ Prefix prefix(int g) const {
    const int b0 = min(max(first(g), 0), p.batch), n = min(max(first(g + 1), 0), p.batch) - b0;
    return Prefix{b0, n, n > 1 ? min(max(p.groups <= ITEMS_LDS ? lds.shared[g] : far(p.shared + g), 0), p.max_len) : 0};
  }
  // The group that request b belongs to, or -1
  __device__ __forceinline__ int group_of(int b) const {
    int lo = 0, hi = p.groups;               // the last group that begins at b or before it: in lo .. hi - 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first(mid) <= b) lo = mid;
      else hi = mid;
    }
    return first(lo) <= b && b < first(lo + 1) ? lo : -1;
  }
  // Tokens of request b that its group reads for it: all of the prefix, or nothing where it ends inside it
  __device__ __forceinline__ int prefix_of(int b) const {
    const int g = group_of(b), n = g < 0 ? 0 : prefix(g).tokens;
    return n <= len(b) ? n : 0;
  }
  __device__ __forceinline__ int blocks(int requests) const { return blocks_of(p, requests); }
  __device__ __forceinline__ int64_t units_of(int g) const {
    const Prefix x = prefix(g);
    return x.tokens > 0 ? (int64_t)units(x.tokens) * p.heads * blocks(x.n) : 0;
  }
  __device__ __forceinline__ int64_t tiles_of(int b) const { return (int64_t)tiles(len(b) - prefix_of(b)) * p.heads * own_chunks(p); }
};
// Pieces: of pairs in one run [2][batch][query heads] (the prefix's part, the own part), then [workgroups][2][rows] and [waves][2][COLS].
__device__ __forceinline__ int64_t whole_at(const SharedParams &p, bool own, int b, int hq) {
  return ((int64_t)(own ? p.batch : 0) + b) * p.heads * p.group + hq;
}
__device__ __forceinline__ int64_t cut_at(const SharedParams &p, bool own, int64_t run, int slot, int row) {
  return (int64_t)2 * p.batch * p.heads * p.group + (own ? (int64_t)2 * p.wgs * p.rows + (2 * run + slot) * COLS : (2 * run + slot) * p.rows) + row;
}

// `total` units in N equal runs, N a power of two, the first `more` of them one longer.
template <int N>
struct Equal {
  int per, more;
  __device__ __forceinline__ explicit Equal(int total) : per(total / N), more(total % N) {}
  __device__ __forceinline__ int start(int i) const { return i * per + min(i, more); }
  __device__ __forceinline__ int of(int unit) const {
    const int longer = more * (per + 1);
    return (int)(unit < longer ? (uint32_t)unit / (uint32_t)(per + 1) : (uint32_t)more + (uint32_t)(unit - longer) / (uint32_t)per);
  }
};

// What a wave keeps in LDS of a tile: where its 32 rows begin, in bytes, and (8-bit caches) the scales of its keys and values and the logarithms
// of both, SMALL at least.
struct TileRows {
  int64_t at[TILE];
  float scale[4 * TILE];
};

// The maximum that weights are taken against follows the scores only where they pass it by more than SLACK, as a power of two, and the largest
// weight of a tile is at most 2^TOP: an accumulator is seldom touched by anything but products.  bf16 has the range of 32 bits.
// A weight is rounded once, to 16 bits (the sum of the weights takes them in 32): a second product with what is left of it, as in f8_attend_paged,
// would be half as many matrix instructions again and four vector instructions a weight.  Relative error of the results: 64 requests behind 32768
// tokens, bf16 0.0022, where their own rounding alone is 0.0017; 3 groups of 17 behind 9001, f16 0.00022 and 0.00021.
// f16 weights keep their relative error down to 2^-21 of the largest one; what lies below is off by 2^-32 of it at most.  Under f16 values those below
// 2^-31 of it are also raised, 256-fold or to f16's smallest number, whichever is less (the sum of the weights takes them unraised): an infinite value
// then shows under every weight from 2^-40 of the largest one up, as in f8_attend_paged, a weight below 2^-48 is 0, and one between is off by
// 2^-31 at most.
template <typename C>
struct Weights {
  static constexpr float SLACK = 8.0f, TOP = 15.0f;
  static __device__ __forceinline__ float raised(float w) {
    return sizeof(C) == 1 ? w : __builtin_amdgcn_fmed3f(w, w * 0x1p8f, 0x1p-24f);
  }
};
template <>
struct Weights<bf16> {
  static constexpr float SLACK = 40.0f, TOP = 0.0f;
  static __device__ __forceinline__ float raised(float w) { return w; }
};

__device__ const v4i zeros[1] = {v4i{0, 0, 0, 0}};          // keys' dimensions beyond the head's

// Two values of each thread: their sums over the threads in front, with `done` of those before them; `done` then has this round's too.
__device__ __forceinline__ void scan_step(const int64_t (&mine)[2], int64_t (&at)[2], int64_t (&done)[2], int64_t (*lds)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t upto[2] = {mine[0], mine[1]};
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t a = __shfl_up((long long)upto[0], d), b = __shfl_up((long long)upto[1], d);
    upto[0] += lane >= d ? a : 0, upto[1] += lane >= d ? b : 0;
  }
  if (lane == 63) lds[wave][0] = upto[0], lds[wave][1] = upto[1];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    at[k] = done[k] + upto[k] - mine[k];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int64_t o = lds[w][k];
      at[k] += w < wave ? o : 0, done[k] += o;
    }
    done[k] = uniform64(done[k]);
  }
  __syncthreads();
}

template <typename C, typename Q, int DP, int NB>
__global__ __launch_bounds__(THREADS, wgs_of(DP, sizeof(C)) / CUS) void attend_shared_kernel(SharedParams p) {
  typedef Operand<C> Op;
  typedef Weights<C> Wt;
  typedef typename Op::t H;
  typedef H t8 __attribute__((ext_vector_type(8)));
  constexpr bool S8 = sizeof(C) == 1;
  constexpr int E = DP / 16, VB = E * (int)sizeof(C);     // elements and bytes of a value row per lane
  constexpr int KL = DP * (int)sizeof(C) / 64;            // 16-byte loads of a key row per lane
  constexpr int KS = DP / 32;                             // products per block of 16 scores
  constexpr int BLOCKS = NB > WAVES ? NB : WAVES;
  constexpr bool EARLY = wgs_of(DP, sizeof(C)) == CUS;    // there are registers for what comes next
  constexpr int PIECES = DP * (int)sizeof(C) / 16;        // 16-byte pieces of a key row, and loads of a tile's keys
  constexpr int KI = TILE * PIECES / 64;
  // A wave's keys, and its part of a piece when its run is over.
  union Stage {
    v4i keys[TILE * PIECES];
    float part[COLS][DP + 4];
  };
  __shared__ Stage stage[WAVES];
  __shared__ TileRows rows[WAVES][2];
  __shared__ int64_t no_rows[TILE];                       // for dimensions beyond the head's: where `zeros` lies
  __shared__ float ml[WAVES][NB * COLS][2];
  __shared__ int64_t scan[WAVES][2];
  __shared__ int from[1 + WAVES], before[1 + WAVES], found[WAVES];
  __shared__ v4i q_lds[BLOCKS][KS][64];
  __shared__ float q_scale_lds[BLOCKS][COLS];
  __shared__ Items items;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c16 = lane & 15, g = lane >> 4;
  if (threadIdx.x < TILE) no_rows[threadIdx.x] = reinterpret_cast<int64_t>(zeros);
  const Work work(p, items);

  // Units and tiles of all, and in front of each; this workgroup's and its waves' runs of them, and the items that these begin in
  constexpr int WGS = wgs_of(DP, sizeof(C));
  const int most = max(p.groups, p.batch);
  int64_t mine[2], at[2], done[2] = {0, 0};
  auto scan_from = [&](int i0) {
    const int i = i0 + (int)threadIdx.x;
    mine[0] = i < p.groups ? work.units_of(i) : 0, mine[1] = i < p.batch ? work.tiles_of(i) : 0;
    scan_step(mine, at, done, scan);
  };
  for (int i0 = 0; i0 < most; i0 += THREADS) {
    scan_from(i0);
    if (blockIdx.x == 0) {
      const int i = i0 + (int)threadIdx.x;
      if (i < p.groups) {
        if (p.groups <= ITEMS_LDS) items.units[i] = (int)at[0];
        else __hip_atomic_store(p.group_units + i, (int)at[0], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      if (i < p.batch) p.records[i].tiles = (int)at[1];
    }
  }
  // (more than fits 31 bits: groups that overlap, which nothing is computed for)
  const int all_units = done[0] <= 0x7fffffff ? (int)done[0] : 0, all_tiles = (int)done[1];
  const Equal<WGS> runs(all_units);
  const Equal<WGS * WAVES> own_runs(all_tiles);
  // (a wave's runs follow those of the same wave of the workgroups in front: with few tiles every workgroup has some)
  const int run = blockIdx.x, own_run = wave * WGS + (int)blockIdx.x;
  int left = runs.start(run + 1) - runs.start(run), own_left = own_runs.start(own_run + 1) - own_runs.start(own_run);
  auto find = [&](int i0) {
    const int i = i0 + (int)threadIdx.x, start = runs.start(run);
    if (at[0] <= start && start < at[0] + mine[0]) from[0] = i, before[0] = (int)at[0];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int start = own_runs.start(w * WGS + (int)blockIdx.x);
      if (at[1] <= start && start < at[1] + mine[1]) from[1 + w] = i, before[1 + w] = (int)at[1];
    }
  };
  if (most <= THREADS) {
    find(0);
  } else {
    done[0] = done[1] = 0;
    for (int i0 = 0; i0 < most; i0 += THREADS) scan_from(i0), find(i0);
  }
  __syncthreads();
  if (blockIdx.x == 0) {
    for (int b = threadIdx.x; b < p.batch; b += THREADS) {
      const int g = work.group_of(b), len = work.len(b);
      const Prefix x = g < 0 ? Prefix{b, 1, 0} : work.prefix(g);
      Record &r = p.records[b];
      r.units = g < 0 ? 0 : p.groups <= ITEMS_LDS ? items.units[g] : work.far(p.group_units + g);
      r.len = len, r.prefix = x.tokens <= len ? x.tokens : 0, r.b0 = x.b0, r.n = x.n;
    }
    if (threadIdx.x == 0) p.records[p.batch].units = all_units, p.records[p.batch].tiles = all_tiles;
  }

  v4f o[NB][E];
  float m[NB], l[NB], q_scale[NB];
  auto clear = [&]() {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      m[nb] = -INFINITY, l[nb] = 0.0f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[nb][e] = v4f{0, 0, 0, 0};
    }
  };
  // 16 query heads as columns, on their way and then into block nb of LDS (`real`: the lane's column is one)
  v4i raw[KS];
  auto load_queries = [&](const Q *src) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = S8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
      __builtin_memcpy(&raw[s], src + (d < p.dim ? d : 0), 16);
    }
  };
  auto put_queries = [&](int nb, bool real) __attribute__((always_inline)) {
    float f[KS][8], scale = fabsf(p.scale);
    uint32_t top = 0;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = S8 ? (s >> 1) * 64 + g * 16 + (s & 1) * 8 : s * 32 + g * 8;
      unpack8<Q>(&raw[s], f[s]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        f[s][j] = real && d < p.dim ? (p.scale < 0 ? -f[s][j] : f[s][j]) : 0.0f;
        top = max(top, magnitude(f[s][j]));
      }
    }
    if constexpr (S8) {
      // a power of two brings the largest element of the row to [2^14, 2^15): f16 then holds what the 16-bit q had, elements
      // 2^-28 below the largest excepted
      top = max(top, (uint32_t)__shfl_xor((int)top, 16));
      top = max(top, (uint32_t)__shfl_xor((int)top, 32));
      const int ex = max((int)(top >> 23), 15);               // (the two factors are then normal numbers, for an infinity's exponent too)
      scale *= __int_as_float((ex - 14) << 23);
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
      q_lds[nb][s][lane] = __builtin_bit_cast(v4i, o);
    }
    // (never 0, which -infinity in a place that a mask leaves out must not meet)
    if (g == 0) q_scale_lds[nb][c16] = fmaxf(scale, 1.17549435e-38f);
  };

  // The tiles at t0, t0 + step .. below `end` of a row of the table, for N blocks of columns from block q0 of LDS on (all of these the same for a
  // wave).  No branch between a tile's products, and none over lanes: the compiler (ROCm 7.2) has put copies of what lives across the loop
  // into the block behind such a branch before that block had all its lanes back.
  // `ready` is called when the first rows are on their way: it waits for the queries.
  auto walk = [&](auto blocks_used, const int32_t *table, int kvh, int t0, int step, int end, int q0, auto ready) {
    constexpr int N = decltype(blocks_used)::value;
    if (t0 >= end) {
      ready();
      return;
    }
    const C *const kbase = static_cast<const C *>(p.k) + kvh * p.head, *const vbase = static_cast<const C *>(p.v) + kvh * p.head;
    const char *const value_base = reinterpret_cast<const char *>(vbase + (c16 * E < p.dim ? c16 * E : 0));
    // Keys come as they lie in memory, rows of neighbouring lanes, and become the product's left operand in LDS: its lanes hold 16 bytes of
    // 16 rows each, which the load unit would take a row at a time (a quarter of the rate).  A row's pieces are permuted by its number: no 16
    // rows' pieces share banks.
    auto turned = [](int row) { return PIECES >= 16 ? row & 15 : PIECES == 8 ? row & 7 : row >> 1 & 3; };
    const int key_row = lane / PIECES, key_piece = lane % PIECES;             // of load 0; load n is n * 64 / PIECES rows further
    const bool key_real = key_piece * (16 / (int)sizeof(C)) < p.dim;
    // (a lane of such dimensions takes its places from no_rows)
    const int64_t key_base = key_real ? reinterpret_cast<int64_t>(kbase) + key_piece * 16 : 0;
    v4i *const keys = stage[wave].keys;
    // The next tile's keys are on their way from when this one's are in LDS, its values from when this one's have been summed up, or before
    // that where there are registers for both.  All loads are issued whether there is a next tile or not (a token that does not exist reads
    // row 0 of the cache): behind a branch around a load nobody knows how many are on their way, and the wait is for all.
    v4i k[KI];
    Raw<VB> v[8];
    float tile_scale = 1.0f;                  // lanes 0..31: of the key of token `lane`, 32..63: of the value of token `lane - 32`
    int64_t scale_at = 0;                     // where the next tile's lies
    uint32_t there, then;                     // tokens of this tile and of the next one that exist
    auto look_up = [&](int t0) {              // page of token lane % 32 of the tile at t0, where there is one
      return table[p.page_size.div((uint32_t)min(t0 + (lane & 31), end - 1))];
    };
    auto locate = [&](int t0, int page, int64_t (&at_lds)[TILE]) {
      const uint32_t tok = (uint32_t)(t0 + (lane & 31)), place = tok - p.page_size.div(tok) * p.page_size.d;
      const bool real = (int)tok < end && (uint32_t)page < (uint32_t)p.pages;
      // (selected, not branched to, and written by both halves of the wave: see above)
      const int64_t pg = real ? page : 0, pl = real ? (int)place : 0;
      at_lds[lane & 31] = (pg * p.page + pl * p.token) * (int64_t)sizeof(C);
      if constexpr (S8) scale_at = pg * p.spage + pl * p.stoken + kvh * p.shead;
      return (uint32_t)__ballot(real);
    };
    auto load_keys = [&](const int64_t (&at_lds)[TILE]) {
      if constexpr (S8) tile_scale = (lane < 32 ? p.k_scale : p.v_scale)[scale_at];
      const int64_t *const at = key_real ? at_lds : no_rows;
      int64_t from[KI];                       // (all read before the first is used)
#pragma unroll
      for (int n = 0; n < KI; ++n) from[n] = at[n * (64 / PIECES) + key_row];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int n = 0; n < KI; ++n) k[n] = *(const __attribute__((address_space(1))) v4i *)(key_base + from[n]);
    };
    auto stage_keys = [&]() {
      lanes_meet();
#pragma unroll
      for (int n = 0; n < KI; ++n) {
        const int row = n * (64 / PIECES) + key_row;
        keys[row * PIECES + (key_piece ^ turned(row))] = k[n];
      }
    };
    auto key = [&](int h, int i) { return keys[(16 * h + c16) * PIECES + ((i * 4 + g) ^ turned(c16))]; };
    auto load_values = [&](const int64_t (&at_lds)[TILE]) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * h + j] = load_raw<VB>(value_base + at_lds[16 * h + 4 * g + j]);
    };

    // Element e of the lane's of its 8 rows: a column of V^T's block e
    auto turn_values = [&](int e) {
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
      return a;
    };

    // A tile's places are looked up two tiles ahead and worked out one ahead, while the first product runs.
    int buf = 0;
    there = locate(t0, look_up(t0), rows[wave][0].at);
    lanes_meet();
    load_keys(rows[wave][0].at);
    int page = look_up(t0 + step);          // (in the order of the loop below)
    load_values(rows[wave][0].at);
    ready();
    then = locate(t0 + step, page, rows[wave][1].at);
    page = look_up(t0 + 2 * step);
    for (;;) {
      const uint32_t now = there;
      there = then;
      const float now_scale = tile_scale;
      stage_keys();
      load_keys(rows[wave][buf ^ 1].at);
      lanes_meet();
      v4f ks[2], vs[2], vl[2];
      if constexpr (S8) {
        float *const scale_lds = rows[wave][buf].scale;
        const float scale = now >> (lane & 31) & 1 ? now_scale : 1.0f;
        scale_lds[lane] = scale;
        scale_lds[64 + lane] = fmaxf(__log2f(scale), SMALL);
        lanes_meet();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          ks[h] = *reinterpret_cast<const v4f *>(scale_lds + 16 * h + 4 * g);
          vs[h] = *reinterpret_cast<const v4f *>(scale_lds + 32 + 16 * h + 4 * g);
          vl[h] = *reinterpret_cast<const v4f *>(scale_lds + 96 + 16 * h + 4 * g);
        }
      }
      v4f acc[N][2];
#pragma unroll
      for (int nb = 0; nb < N; ++nb) acc[nb][0] = acc[nb][1] = v4f{0, 0, 0, 0};
      // A step of the product needs two pieces of keys and N of queries (twice as many of the converted ones); the next step's are read from LDS
      // before this one's products, which hide the way, where there are registers for both.
      constexpr int QS = S8 ? 2 : 1, AHEAD = EARLY ? 2 : 1;
      v4i kd[AHEAD][2], qd[AHEAD][QS][N];
      auto read_step = [&](int i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) kd[i % AHEAD][h] = key(h, i);
#pragma unroll
        for (int s = 0; s < QS; ++s)
#pragma unroll
          for (int nb = 0; nb < N; ++nb) qd[i % AHEAD][s][nb] = q_lds[q0 + nb][QS * i + s][lane];
      };
      if constexpr (EARLY) read_step(0);
#pragma unroll
      for (int i = 0; i < KL; ++i) {
        if constexpr (EARLY) {
          if (i + 1 < KL) read_step(i + 1);
          __builtin_amdgcn_sched_barrier(0);
        } else {
          read_step(i);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const v4i d = kd[i % AHEAD][h];
          if constexpr (S8) {
            h8 lo, hi;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t u = (uint32_t)d[j] ^ 0x80808080u;
              const h2 a = codes_lo(u), e = codes_hi(u);
              h8 &to = j < 2 ? lo : hi;
              to[4 * (j & 1)] = a[0], to[4 * (j & 1) + 1] = a[1], to[4 * (j & 1) + 2] = e[0], to[4 * (j & 1) + 3] = e[1];
            }
#pragma unroll
            for (int nb = 0; nb < N; ++nb) acc[nb][h] = Op::mfma(__builtin_bit_cast(v4i, lo), qd[i % AHEAD][0][nb], acc[nb][h]);
#pragma unroll
            for (int nb = 0; nb < N; ++nb) acc[nb][h] = Op::mfma(__builtin_bit_cast(v4i, hi), qd[i % AHEAD][QS - 1][nb], acc[nb][h]);
          } else {
#pragma unroll
            for (int nb = 0; nb < N; ++nb) acc[nb][h] = Op::mfma(d, qd[i % AHEAD][0][nb], acc[nb][h]);
          }
        }
        if constexpr (EARLY) __builtin_amdgcn_sched_barrier(0);
      }
      then = locate(t0 + 2 * step, page, rows[wave][buf].at);
      page = look_up(t0 + 3 * step);
      __builtin_amdgcn_sched_barrier(0);    // (ahead of the values' loads, which a wait for it must not wait for)
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
      v4i turned_values[EARLY ? E : 1];
      if constexpr (EARLY) {
#pragma unroll
        for (int e = 0; e < E; ++e) turned_values[e] = turn_values(e);
        load_values(rows[wave][buf ^ 1].at);
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
          for (int j = 0; j < 4; ++j)
            top[nb] = fmaxf(top[nb], S8 ? __builtin_fmaf(acc[nb][h][j], q_scale[nb] * ks[h][j], vl[h][j]) : acc[nb][h][j]);
        if (!S8) top[nb] *= q_scale[nb];
        rises = rises || top[nb] > m[nb] + Wt::SLACK;
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
        const float below = (m[nb] == -INFINITY ? 0.0f : m[nb]) - (Wt::TOP - Wt::SLACK);
        t8 wh;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[nb][j >> 2][j & 3], S8 ? q_scale[nb] * ks[j >> 2][j & 3] : q_scale[nb], -below));
          l[nb] += w;
          wh[j] = (H)(S8 ? w * vs[j >> 2][j & 3] : Wt::raised(w));
        }
        pt[nb] = __builtin_bit_cast(v4i, wh);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const v4i a = EARLY ? turned_values[EARLY ? e : 0] : turn_values(e);
#pragma unroll
        for (int nb = 0; nb < N; ++nb) o[nb][e] = Op::mfma(a, pt[nb], o[nb][e]);
      }
      // The results of the last products are there before any branch: behind one the compiler (ROCm 7.2) has read an
      // accumulator without the wait that a matrix instruction's result needs.
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_nop 15" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (!EARLY) load_values(rows[wave][buf ^ 1].at);
      buf ^= 1, t0 += step;
      if (t0 >= end) break;
    }
  };

  // ---- prefixes ----
  int item = left > 0 ? __builtin_amdgcn_readfirstlane(from[0]) : 0;
  int in = left > 0 ? __builtin_amdgcn_readfirstlane(runs.start(run) - before[0]) : 0;        // units of the item in front of this run
  while (left > 0) {
    // requests b0 + req0 .., `heads` query heads of cache head kvh each, over tokens of the row `leader` of the table
    const Prefix x = work.prefix(item);
    const int b0 = __builtin_amdgcn_readfirstlane(x.b0), n = __builtin_amdgcn_readfirstlane(x.n), tokens = __builtin_amdgcn_readfirstlane(x.tokens);
    const int item_units = units(tokens), blocks = work.blocks(n);
    int leader = b0, t_end = tokens;
    if (work.len(leader) < tokens) {
      // (an empty place in front) the first member that has all of the prefix; without any nobody reads what comes out
      int have = 0x7fffffff;
      for (int i = b0 + (int)threadIdx.x; i < b0 + n && have == 0x7fffffff; i += THREADS)
        if (work.len(i) >= tokens) have = i;
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
    const int pair = __builtin_amdgcn_readfirstlane((int)((uint32_t)in / (uint32_t)item_units)), unit = in - pair * item_units;
    const int kvh = pair / blocks, block = pair - kvh * blocks, chunk = block % p.chunks, req0 = block / p.chunks * p.per_block;
    const int h0 = chunk * p.rows, heads = p.chunks > 1 ? min(p.rows, p.group - h0) : p.group;
    const int real_rows = __builtin_amdgcn_readfirstlane(min(n - req0, p.per_block) * heads), nb_used = (real_rows + COLS - 1) / COLS;
    const int last = min(item_units, unit + left), end = min(t_end, last * UNIT);
    auto place = [&](int row, int &b, int &hq) {             // of a row of the block
      const int r = p.chunks > 1 ? 0 : (int)p.by_group.div((uint32_t)row);
      b = b0 + req0 + r, hq = kvh * p.group + h0 + row - r * heads;
    };
    // blocks of columns that a walk takes: three are taken as four, and the fourth one's zeros are put down like any other column that is none
    // (its maximum counts where the walk asks whether any rises)
    const int walked = nb_used == 3 ? 4 : nb_used;
    const int row0 = wave * COLS + c16;
    {
      int b, hq;
      place(min(row0, real_rows - 1), b, hq);
      load_queries(static_cast<const Q *>(p.q) + b * p.qt + hq * p.qh);
    }
    auto ready = [&]() {
      if (wave < walked) put_queries(wave, row0 < real_rows);
      __syncthreads();
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) q_scale[nb] = q_scale_lds[nb][c16];
      clear();
    };
    const int32_t *table = p.table + leader * p.table_ld;
    const int t0 = unit * UNIT + wave * TILE;
    if constexpr (NB >= 4) {
      if (walked == 4) walk(std::integral_constant<int, 4>(), table, kvh, t0, UNIT, end, 0, ready);
      else if (walked == 2) walk(std::integral_constant<int, 2>(), table, kvh, t0, UNIT, end, 0, ready);
      else walk(std::integral_constant<int, 1>(), table, kvh, t0, UNIT, end, 0, ready);
    } else {
      if (walked == 2) walk(std::integral_constant<int, 2>(), table, kvh, t0, UNIT, end, 0, ready);
      else walk(std::integral_constant<int, 1>(), table, kvh, t0, UNIT, end, 0, ready);
    }

    // the waves join in LDS, 16 columns at a time, and leave the piece
    const bool whole = unit == 0 && last == item_units;
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
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < E; e += 4)
          *reinterpret_cast<v4f *>(&stage[wave].part[c16][(4 * g + j) * E + e]) =
              v4f{o[nb][e][j] * shrink, o[nb][e + 1][j] * shrink, o[nb][e + 2][j] * shrink, o[nb][e + 3][j] * shrink};
      __syncthreads();
#pragma unroll
      for (int i = threadIdx.x; i < COLS * DP / 4; i += THREADS) {
        const int c = i / (DP / 4), d = i % (DP / 4) * 4, row = nb * COLS + c;
        if (row >= real_rows || d >= p.dim) continue;
        v4f of{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
          const v4f x = *reinterpret_cast<const v4f *>(&stage[w].part[c][d]);
#pragma unroll
          for (int k = 0; k < 4; ++k) of[k] += x[k];
        }
        int b, hq;
        place(row, b, hq);
        const int64_t at = whole ? whole_at(p, false, b, hq) : cut_at(p, false, run, unit == 0, row);
        *reinterpret_cast<v4f *>(p.part_o + at * p.dim + d) = of;
        if (d == 0) {
          float mh = ml[0][row][0], sum = 0.0f;
#pragma unroll
          for (int w = 1; w < WAVES; ++w) mh = fmaxf(mh, ml[w][row][0]);
          const float base = mh == -INFINITY ? 0.0f : mh;
#pragma unroll
          for (int w = 0; w < WAVES; ++w) sum += ml[w][row][1] * __builtin_amdgcn_exp2f(ml[w][row][0] - base);
          p.part_ml[2 * at] = mh, p.part_ml[2 * at + 1] = sum;
        }
      }
      __syncthreads();
    }
    left -= last - unit, in += last - unit;
    if (left > 0 && in == item_units * blocks * p.heads) {                // the next group that has units
      in = 0;
      do ++item;
      while (work.units_of(item) == 0);
      item = __builtin_amdgcn_readfirstlane(item);
    }
  }

  // ---- own tokens, every wave for itself ----
  int b = own_left > 0 ? __builtin_amdgcn_readfirstlane(from[1 + wave]) : 0;
  in = own_left > 0 ? __builtin_amdgcn_readfirstlane(own_runs.start(own_run) - before[1 + wave]) : 0;
  const int chunks = own_chunks(p);
  while (own_left > 0) {
    const int t_begin = __builtin_amdgcn_readfirstlane(work.prefix_of(b)), len = __builtin_amdgcn_readfirstlane(work.len(b));
    const int own_tiles = tiles(len - t_begin);
    const int pair = __builtin_amdgcn_readfirstlane((int)((uint32_t)in / (uint32_t)own_tiles)), tile = in - pair * own_tiles;
    const int kvh = pair / chunks, h0 = (pair - kvh * chunks) * COLS, heads = min(COLS, p.group - h0), hq = kvh * p.group + h0 + min(c16, heads - 1);
    const int last = min(own_tiles, tile + own_left);
    load_queries(static_cast<const Q *>(p.q) + b * p.qt + hq * p.qh);
    auto ready = [&]() {
      lanes_meet();
      put_queries(wave, c16 < heads);
      lanes_meet();
      q_scale[0] = q_scale_lds[wave][c16];
      clear();
    };
    walk(std::integral_constant<int, 1>(), p.table + b * p.table_ld, kvh, t_begin + tile * TILE, TILE, min(len, t_begin + last * TILE), wave, ready);
    l[0] += __shfl_xor(l[0], 16);
    l[0] += __shfl_xor(l[0], 32);
    if (c16 < heads) {
      const int64_t at = tile == 0 && last == own_tiles ? whole_at(p, true, b, hq) : cut_at(p, true, own_run, tile == 0, c16);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = (4 * g + j) * E;          // (dim is a multiple of 16 and so of E)
        if (d < p.dim) {
#pragma unroll
          for (int e = 0; e < E; e += 4)
            *reinterpret_cast<v4f *>(p.part_o + at * p.dim + d + e) = v4f{o[0][e][j], o[0][e + 1][j], o[0][e + 2][j], o[0][e + 3][j]};
        }
      }
      if (g == 0) p.part_ml[2 * at] = m[0], p.part_ml[2 * at + 1] = l[0];
    }
    own_left -= last - tile, in += last - tile;
    if (own_left > 0 && in == own_tiles * chunks * p.heads) {         // the next request that has tiles
      in = 0;
      do ++b;
      while (work.tiles_of(b) == 0);
      b = __builtin_amdgcn_readfirstlane(b);
    }
  }
}

// Both parts of a request's heads together: 5 us, a launch and three latencies (the record, the pieces, the store).  A workgroup takes
// JOIN_PART elements (heads by dimensions) of a request, a cache head and a chunk of
// its query heads, 4 neighbours a thread and as many pieces at a time as threads are left; the pieces are added up in a fixed order.
constexpr int JOINERS = 4, JOIN_PART = 256, JOIN_VECS = JOIN_PART / 4, JOIN_AT_ONCE = 64 * JOINERS / JOIN_VECS;

template <typename Q, int WGS>
__global__ __launch_bounds__(64 * JOINERS) void join_shared_kernel(SharedParams p) {
  __shared__ v4f part[JOIN_AT_ONCE][JOIN_VECS];
  __shared__ float sums[JOIN_AT_ONCE][JOIN_VECS], tops[JOIN_AT_ONCE][JOIN_VECS];
  const int per_b = p.heads * p.chunks, b = blockIdx.x / per_b, hc = blockIdx.x % per_b, kvh = hc / p.chunks, chunk = hc % p.chunks;
  const int h0 = chunk * p.rows, heads = p.chunks > 1 ? min(p.rows, p.group - h0) : p.group;
  const int vec = (int)threadIdx.x % JOIN_VECS, mine = (int)threadIdx.x / JOIN_VECS;
  // (dim is a multiple of 16: four neighbours belong to one head)
  const int e = blockIdx.y * JOIN_PART + vec * 4, h = e / p.dim, d = e - h * p.dim;
  const bool real = h < heads;
  const int hq = kvh * p.group + h0 + (real ? h : 0), col = real ? d : 0;
  const Record x = p.records[b], all = p.records[p.batch];
  // pieces of the prefix's pair and of the own one
  struct Pieces {
    int64_t first, rest, step;                // rows of piece 0 and 1, and from there to the next
    int n;
  };
  auto pieces = [&](const auto &runs, int at, int units, bool own, int row) {
    if (units == 0) return Pieces{0, 0, 0, 0};
    const int i0 = runs.of(at), i1 = runs.of(at + units - 1);
    if (i0 == i1) return Pieces{whole_at(p, own, b, hq), 0, 0, 1};
    return Pieces{cut_at(p, own, i0, 1, row), cut_at(p, own, i0 + 1, 0, row), 2 * (own ? COLS : p.rows), i1 - i0 + 1};
  };
  const int pu = x.prefix > 0 && all.units > 0 ? units(x.prefix) : 0, ot = tiles(x.len - x.prefix), in_group = h0 + (real ? h : 0);
  const int blocks = blocks_of(p, x.n), block = (b - x.b0) / p.per_block * p.chunks + chunk;
  const Pieces a = pieces(Equal<WGS>(all.units), x.units + (kvh * blocks + block) * pu, pu, false, (b - x.b0) % p.per_block * heads + (real ? h : 0));
  const Pieces c = pieces(Equal<WGS * WAVES>(all.tiles), x.tiles + (kvh * own_chunks(p) + in_group / COLS) * ot, ot, true, in_group % COLS);
  const int n = a.n + c.n;
  auto row_of = [&](int i) {
    const Pieces &k = i < a.n ? a : c;
    const int j = i < a.n ? i : i - a.n;
    return j == 0 ? k.first : k.rest + (j - 1) * k.step;
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

template <typename C, typename Q, int DP>
f8_status launch_dim(const SharedParams &p, hipStream_t s) {
  hipLaunchKernelGGL((attend_shared_kernel<C, Q, DP, blocks_of(DP, sizeof(C))>), dim3(p.wgs), dim3(THREADS), 0, s, p);
  const f8_status st = launch_status();
  if (st != F8_OK) return st;
  const int elements = (p.chunks > 1 ? p.rows : p.group) * p.dim;
  hipLaunchKernelGGL((join_shared_kernel<Q, wgs_of(DP, sizeof(C))>), dim3(p.batch * p.heads * p.chunks, (elements + JOIN_PART - 1) / JOIN_PART),
                     dim3(64 * JOINERS), 0, s, p);
  return launch_status();
}
template <typename C, typename Q>
f8_status launch(const SharedParams &p, hipStream_t s) {
  return p.dim <= 64 ? launch_dim<C, Q, 64>(p, s) : p.dim <= 128 ? launch_dim<C, Q, 128>(p, s) : launch_dim<C, Q, 256>(p, s);
}

// Up to 512 tokens to a request the call goes to f8_attend_paged, and past 2^31 tiles in all, which only that counts in 64 bits.  One group behind 256
// common tokens, 32 of each request's own, 8 heads of 4 query heads, dim 128, us there and here: bf16 8 requests 9 and 18, 64 17 and 23, 256 60 and 35;
// 8 bits 8.5 and 18, 11 and 20, 35 and 31.  Behind 480: bf16 11 and 18, 21 and 24, 74 and 37; 8 bits 10 and 19, 15 and 21, 45 and 33.  So for
// some 200 requests and more it is the slower way, which this rule, on the length alone, does not see.
bool alone(int batch, int groups, int q_heads, int max_len) {
  return groups == 0 || max_len <= 4 * UNIT || ((int64_t)max_len + TILE - 1) / TILE * batch * q_heads > 0x7fffffff;
}
size_t pieces_of(int64_t batch, int q_heads, int dim) {
  const int a = wgs_of(dim, 1) * (blocks_of(dim, 1) + WAVES), b = wgs_of(dim, 2) * (blocks_of(dim, 2) + WAVES);
  return (size_t)2 * batch * q_heads + (size_t)2 * (a > b ? a : b) * COLS;
}

}  // namespace
}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_attend_shared_workspace_bytes(int batch, int groups, int q_heads, int kv_heads, int dim, int max_len) {
  if (batch < 1 || groups < 0 || q_heads < 1 || kv_heads < 1 || dim < 1 || max_len < 1 || q_heads % kv_heads != 0) return 0;
  if (alone(batch, groups, q_heads, max_len)) return f8_attend_workspace_bytes(batch, q_heads, kv_heads, dim, max_len);
  return ((size_t)batch + 1) * sizeof(Record) + pieces_of(batch, q_heads, dim) * (dim + 2) * sizeof(float) + groups * sizeof(int32_t);
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
  if (d->batch == 0 || alone(d->batch, groups, d->q_heads, d->max_len))
    return f8_attend_paged(q, k_cache, v_cache, k_scale, v_scale, table, lens, out, c, d, workspace, workspace_bytes, stream);
  st = check_attend_pointers(q, k_cache, v_cache, k_scale, v_scale, table, lens, out, *c, *d);
  if (st != F8_OK) return st;
  const int group = d->q_heads / c->heads, most = blocks_of(c->dim, (int)bytes_of(c->type)) * COLS, chunks = (group + most - 1) / most;
  if ((int64_t)d->batch * c->heads * chunks > 1 << 22) return F8_ERR_UNSUPPORTED;          // (workgroups of a launch)
  if (!workspace) return F8_ERR_NULL;
  if (!aligned_to(workspace, 16)) return F8_ERR_ALIGN;
  if (workspace_bytes < f8_attend_shared_workspace_bytes(d->batch, groups, d->q_heads, c->heads, c->dim, d->max_len)) return F8_ERR_SHAPE;
  Record *records = static_cast<Record *>(workspace);
  const size_t pieces = pieces_of(d->batch, d->q_heads, c->dim);
  float *ws = reinterpret_cast<float *>(records + d->batch + 1);
  const SharedParams p{q, k_cache, v_cache, k_scale, v_scale, table, lens, first, shared, out, ws, ws + pieces * c->dim,
                       records, reinterpret_cast<int32_t *>(ws + pieces * (c->dim + 2)),
                       d->q_token, d->q_head, d->o_token, d->o_head, c->page_stride, c->token_stride, c->head_stride,
                       c->scale_page, c->scale_token, c->scale_head, d->table_ld, d->batch, groups, c->heads, group, chunks,
                       chunks > 1 ? 1 : most / group, c->dim, c->pages, d->max_len, wgs_of(c->dim, (int)bytes_of(c->type)), most,
                       FastDiv((uint32_t)c->page_size), FastDiv((uint32_t)group),
                       d->scale * LOG2E};
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (c->type == F8_S8) return d->type == F8_F16 ? launch<int8_t, f16>(p, hs) : launch<int8_t, bf16>(p, hs);
  return d->type == F8_F16 ? launch<f16, f16>(p, hs) : launch<bf16, bf16>(p, hs);
}

}  // extern "C"
