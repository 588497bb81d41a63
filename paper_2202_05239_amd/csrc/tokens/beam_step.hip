// Beam search's selection: the `keep` largest of S[i][t] = score_i + x_it - lse_i over a prompt's beams i and tokens t.
//
// Within a beam S falls with x, so a first launch needs no scores: a workgroup takes up to 16384 logits of a row into its registers and leaves
// their maximum m, sum exp(x - m) and `keep` largest, and a second launch (a workgroup to a prompt) adds up the sums, forms S of what
// is left in 64 bits and takes the `keep` largest of that.  Bound by HBM: the logits are read once.
//
// The largest of a set.  Elements are keys (value, then lowest index: no two alike).  Threads form at least `keep` groups; every group's
// largest key is one of the elements, so the least of these maxima is a lower bound of the keep-th largest key, which few elements pass (16 of 16384
// random ones: about 45).  Those go to a list in LDS, and each one's place is the number of keys above it.  Where more pass than
// the list holds, the bound is the keep-th largest of the threads' own maxima: what passes then are elements of `keep` threads.
#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int CHUNK = 16384;                                // logits of a workgroup at most
constexpr int CANDIDATES = 8192;                            // of a prompt in the second launch at most
constexpr int BEAMS = 1024;
__host__ __device__ inline int each_of(uint32_t candidates) { return (int)((candidates + THREADS - 1) / THREADS); }   // of a thread there

struct Stat {
  double sum;                               // of exp(x - top)
  float top;
};

struct BeamParams {
  const void *logits;
  const float *scores;
  const uint8_t *done;
  float *score;
  int32_t *parent, *token;
  uint64_t *best;                           // [rows][splits][keep]: order of the value, ~token; 0: none
  Stat *stat;                               // [rows][splits]
  int64_t ld;
  int beams, vocab, keep, splits, eos, groups;              // groups of threads: a power of two, at least `keep`
  int64_t blocks;
  FastDiv by_splits;
};

// Numbers as unsigned integers of the same order, all above 0; -0 is 0 and NaN lies above all.
__device__ __forceinline__ uint32_t order_of(float v) {
  if (v != v) return 0xffffffffu;
  const uint32_t u = __float_as_uint(v + 0.0f);
  return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t o) { return __uint_as_float(o >> 31 ? (o == 0xffffffffu ? o : o & 0x7fffffffu) : ~o); }
__device__ __forceinline__ uint64_t order_of(double v) {
  if (v != v) return ~0ull;
  const uint64_t u = (uint64_t)__double_as_longlong(v + 0.0);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ __forceinline__ double of_order(uint64_t o) {
  return __longlong_as_double((long long)(o >> 63 ? (o == ~0ull ? o : o & ~(1ull << 63)) : ~o));
}

// Keys: a logit and its token; S, its beam, its logit and token (a score may be so large that 64 bits give two logits of a beam the same
// S: the larger one's is larger).  Key{} is no element.
struct Key64 {
  uint64_t k;
  __device__ __forceinline__ bool operator<(const Key64 &o) const { return k < o.k; }
  __device__ __forceinline__ bool real() const { return k != 0; }
  __device__ __forceinline__ Key64 from(int d) const { return Key64{(uint64_t)__shfl_xor((unsigned long long)k, d)}; }
};
struct KeyS {
  uint64_t s, beam, logit;                  // beam: ~i, logit: its order, ~token
  __device__ __forceinline__ bool operator<(const KeyS &o) const {
    return s < o.s || (s == o.s && (beam < o.beam || (beam == o.beam && logit < o.logit)));
  }
  __device__ __forceinline__ bool real() const { return s != 0; }
  __device__ __forceinline__ KeyS from(int d) const {
    return KeyS{(uint64_t)__shfl_xor((unsigned long long)s, d), (uint64_t)__shfl_xor((unsigned long long)beam, d),
                (uint64_t)__shfl_xor((unsigned long long)logit, d)};
  }
};

template <typename K>
struct Pick {
  K top[THREADS], bound;
  int n;
};

// The `keep` largest of all threads' elements: mine is the largest of this thread's, each(bound, f) calls f for those of them that are not below
// `bound` (and may for others).  out(place, key) is called for each, places from 0 in descending order; returns how many there are.
// list: `most` keys, keep times a thread's elements.  Every thread of the workgroup comes here.
template <typename K, typename Each, typename Out>
__device__ __forceinline__ int pick(Pick<K> &l, K *list, int most, int keep, int groups, K mine, Each each, Out out) {
  const int t = threadIdx.x, lane = t & 63;
  // thread t belongs to group t mod `groups`: neighbours, which hold neighbouring elements, to different ones
  K bound = mine;
  for (int d = 32; d >= groups; d >>= 1) {
    const K o = bound.from(d);
    if (bound < o) bound = o;
  }
  l.top[t] = bound;
  if (t == 0) l.n = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w)
    if (bound < l.top[w * 64 + lane]) bound = l.top[w * 64 + lane];
  for (int d = min(groups, 64) >> 1; d > 0; d >>= 1) {
    const K o = bound.from(d);
    if (o < bound) bound = o;
  }
  auto collect = [&](K key) {
    if (key.real() && !(key < bound)) {
      const int i = atomicAdd(&l.n, 1);
      if (i < most) list[i] = key;
    }
  };
  each(bound, collect);
  __syncthreads();
  int n = l.n;
  if (n > most) {
    __syncthreads();
    l.top[t] = mine;
    if (t == 0) l.n = 0, l.bound = K{};
    __syncthreads();
    int above = 0;
    for (int i = 0; i < THREADS; ++i) above += mine < l.top[i];
    if (above == keep - 1 && mine.real()) l.bound = mine;
    __syncthreads();
    bound = l.bound;
    each(bound, collect);
    __syncthreads();
    n = min(l.n, most);
  }
  for (int i = t; i < n; i += THREADS) {
    const K key = list[i];
    int above = 0;
    for (int j = 0; j < n; ++j) above += key < list[j];
    if (above < keep) out(above, key);
  }
  return min(n, keep);
}

// exp(t) for t <= 0 to the last place of the hardware's exponential: the product with log2 e in two parts.
__device__ __forceinline__ float exp_of(float t) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(t, 1.44269502162933349609375f, t * 1.92596299e-8f));
}

template <typename T, int NV>
__global__ __launch_bounds__(THREADS) void beam_rows_kernel(BeamParams p) {
  typedef RowMap<THREADS, NV> Map;
  extern __shared__ __align__(16) uint8_t dynamic[];
  __shared__ Pick<Key64> l;
  __shared__ float tops[WAVES];
  __shared__ double sums[WAVES];
  const int64_t block = row_block();
  if (block >= p.blocks) return;
  const int row = (int)p.by_splits.div((uint32_t)block), split = (int)block - row * p.splits;
  if (p.done && p.done[row]) return;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int base = split * Map::most, cols = min(Map::most, p.vocab - base);
  const T *x = static_cast<const T *>(p.logits) + row * p.ld + base;
  float v[NV][8], piece[NV], top = -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i) load_piece<T, Map>(x, i, t, cols, v[i]);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int here = cols - Map::col(i, 0, t);              // elements from the piece's first one on
    if (here < 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = j < here ? v[i][j] : -INFINITY;
    }
    piece[i] = fmaxf(fmaxf(fmaxf(v[i][0], v[i][1]), fmaxf(v[i][2], v[i][3])), fmaxf(fmaxf(v[i][4], v[i][5]), fmaxf(v[i][6], v[i][7])));
    top = fmaxf(top, piece[i]);
  }
  // the thread's largest: the first of its value
  int at = 0x7fffffff;
#pragma unroll
  for (int i = NV - 1; i >= 0; --i) {
    if (piece[i] == top) {
#pragma unroll
      for (int j = 7; j >= 0; --j)
        if (v[i][j] == top && Map::col(i, j, t) < cols) at = Map::col(i, j, t);
    }
  }
  const Key64 mine{at < cols ? (uint64_t)order_of(top) << 32 | (uint32_t)~(base + at) : 0};
  float m = top;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  if (lane == 0) tops[wave] = m;
  const int n = pick<Key64>(
      l, reinterpret_cast<Key64 *>(dynamic), p.keep * NV * 8, p.keep, p.groups, mine,
      [&](Key64 bound, auto f) {
        const float least = bound.real() ? of_order((uint32_t)(bound.k >> 32)) : -INFINITY;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          if (piece[i] >= least) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
              if (v[i][j] >= least && Map::col(i, j, t) < cols)
                f(Key64{(uint64_t)order_of(v[i][j]) << 32 | (uint32_t)~(base + Map::col(i, j, t))});
          }
        }
      },
      [&](int place, Key64 key) { p.best[(block * p.keep) + place] = key.k; });
  if (t >= n && t < p.keep) p.best[block * p.keep + t] = 0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) m = fmaxf(m, tops[w]);
  // (NaN and +infinity come out as a sum that is NaN: fmaxf passes over a NaN, the differences do not)
  float part[2] = {0, 0};
  if (m != -INFINITY) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) part[j & 1] += exp_of(v[i][j] - m);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) part[0] += v[i][j] != v[i][j] ? v[i][j] : 0.0f;
  }
  double sum = (double)part[0] + (double)part[1];
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  if (t == 0) {
    for (int w = 1; w < WAVES; ++w) sum += sums[w];
    p.stat[block] = Stat{sum, m};
  }
}

__global__ __launch_bounds__(THREADS) void beam_join_kernel(BeamParams p) {
  extern __shared__ __align__(16) uint8_t dynamic[];
  __shared__ Pick<KeyS> l;
  __shared__ double lse[BEAMS];             // NaN or -infinity: S of the beam is that throughout; 0: it is done
  const int b = blockIdx.x, t = threadIdx.x;
  const int64_t row0 = (int64_t)b * p.beams;
  for (int i = t; i < p.beams; i += THREADS) {
    const float score = p.scores[row0 + i];
    double of = 0;
    if (!(score < INFINITY)) {
      of = (double)__builtin_nanf("");
    } else if (score == -INFINITY) {
      of = score;
    } else if (!(p.done && p.done[row0 + i])) {
      const Stat *s = p.stat + (row0 + i) * p.splits;
      float top = -INFINITY;
      for (int j = 0; j < p.splits; ++j) top = fmaxf(top, s[j].top);
      double sum = 0;
      for (int j = 0; j < p.splits; ++j) sum += s[j].top == -INFINITY ? s[j].sum : s[j].sum * exp((double)s[j].top - (double)top);
      of = sum == 0 ? -(double)INFINITY : (double)top + log(sum);
    }
    lse[i] = of;
  }
  __syncthreads();
  const uint32_t per_row = (uint32_t)p.splits * p.keep, all = per_row * p.beams;
  auto key_of = [&](uint32_t c) -> KeyS {
    const uint32_t i = c / per_row, in = c - i * per_row;
    const float score = p.scores[row0 + i];
    const double of = lse[i];
    uint64_t logit;                          // (all the same where S is the same throughout: tokens in their order)
    double s;
    if (of != of || of == -(double)INFINITY) {
      if (in >= (uint32_t)min(p.keep, p.vocab)) return KeyS{};
      logit = (uint32_t)~in, s = of;
    } else if (p.done && p.done[row0 + i]) {
      if (in >= (uint32_t)min(p.keep, p.vocab)) return KeyS{};
      logit = (uint32_t)~(in == 0 ? p.eos : in - (in <= (uint32_t)p.eos)), s = in == 0 ? (double)score : -(double)INFINITY;
    } else {
      logit = p.best[(row0 + i) * per_row + in];
      if (logit == 0) return KeyS{};
      s = (double)score + ((double)of_order((uint32_t)(logit >> 32)) - of);
    }
    return KeyS{order_of(s), ~(uint64_t)i, logit};
  };
  KeyS mine{};
  for (uint32_t c = t; c < all; c += THREADS) {
    const KeyS k = key_of(c);
    if (mine < k) mine = k;
  }
  const int64_t out = (int64_t)b * p.keep;
  pick<KeyS>(
      l, reinterpret_cast<KeyS *>(dynamic), p.keep * each_of(all), p.keep, p.groups, mine,
      [&](KeyS bound, auto f) {
        if (bound.real() && mine < bound) return;
        for (uint32_t c = t; c < all; c += THREADS) f(key_of(c));
      },
      [&](int place, KeyS key) {
        p.score[out + place] = (float)of_order(key.s);
        p.parent[out + place] = (int32_t)(row0 + (int64_t)~key.beam);
        p.token[out + place] = (int32_t)~(uint32_t)key.logit;
      });
}

// Pieces of 8 logits to a thread of the first launch.  The second one's work grows with the number of workgroups to a row, so a row is cut as
// little as fills the chip.
int pieces_of(int64_t rows, int vocab, int beams, int keep) {
  int nv = 1;
  while (nv < 8) {
    const int64_t splits = ((int64_t)vocab + THREADS * 8 * nv - 1) / (THREADS * 8 * nv);
    if (splits == 1 || (rows * splits <= 1024 && splits * beams * keep <= CANDIDATES)) break;
    nv *= 2;
  }
  return nv;
}
int splits_of(int64_t rows, int vocab, int beams, int keep) {
  const int chunk = THREADS * 8 * pieces_of(rows, vocab, beams, keep);
  return (int)(((int64_t)vocab + chunk - 1) / chunk);
}

template <typename T>
void launch_rows(const BeamParams &p, int nv, hipStream_t s) {
  const dim3 grid = block_grid(p.blocks), block(THREADS);
  const size_t lds = (size_t)p.keep * nv * 8 * sizeof(Key64);
  switch (nv) {
    case 1: hipLaunchKernelGGL((beam_rows_kernel<T, 1>), grid, block, lds, s, p); break;
    case 2: hipLaunchKernelGGL((beam_rows_kernel<T, 2>), grid, block, lds, s, p); break;
    case 4: hipLaunchKernelGGL((beam_rows_kernel<T, 4>), grid, block, lds, s, p); break;
    default: hipLaunchKernelGGL((beam_rows_kernel<T, 8>), grid, block, lds, s, p);
  }
}

}  // namespace
}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_beam_workspace_bytes(int batch, int beams, int vocab, int keep) {
  if (batch < 1 || beams < 1 || vocab < 1 || keep < 1 || beams > BEAMS || keep > F8_BEAM_MAX_KEEP) return 0;
  const size_t parts = (size_t)batch * beams * splits_of((int64_t)batch * beams, vocab, beams, keep);
  return parts * (sizeof(Stat) + keep * sizeof(uint64_t));
}

f8_status f8_beam_step(const void *logits, const float *scores, const uint8_t *done, float *score, int32_t *parent, int32_t *token,
                       const f8_beam_desc *d, void *workspace, size_t workspace_bytes, void *stream) {
  if (!d) return F8_ERR_NULL;
  if (!real_type(d->type)) return F8_ERR_DTYPE;
  if (d->batch < 0 || d->beams < 1 || d->vocab < 1 || d->keep < 1 || (int64_t)d->keep > (int64_t)d->beams * d->vocab || d->ld < d->vocab) return F8_ERR_SHAPE;
  if (done && (d->eos < 0 || d->eos >= d->vocab)) return F8_ERR_SHAPE;
  if (d->beams > BEAMS || d->keep > F8_BEAM_MAX_KEEP || d->vocab > 0x3fffffff || (int64_t)d->beams * d->keep * (((int64_t)d->vocab + CHUNK - 1) / CHUNK) > CANDIDATES)
    return F8_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)d->batch * d->beams;
  if (rows > 0x7fffffff) return F8_ERR_SHAPE;
  const int nv = pieces_of(rows, d->vocab, d->beams, d->keep), splits = splits_of(rows, d->vocab, d->beams, d->keep);
  if (rows * splits > 0x7fffffff) return F8_ERR_UNSUPPORTED;
  if (d->batch == 0) return F8_OK;
  if (!logits || !scores || !score || !parent || !token || !workspace) return F8_ERR_NULL;
  if (!aligned_to(logits, bytes_of(d->type)) || !aligned_to(scores, 4) || !aligned_to(score, 4) || !aligned_to(parent, 4) || !aligned_to(token, 4) ||
      !aligned_to(workspace, 16))
    return F8_ERR_ALIGN;
  if (workspace_bytes < f8_beam_workspace_bytes(d->batch, d->beams, d->vocab, d->keep)) return F8_ERR_SHAPE;
  int groups = 1;
  while (groups < d->keep) groups *= 2;
  const int64_t parts = rows * splits;
  Stat *stat = static_cast<Stat *>(workspace);
  const BeamParams p{logits, scores, done, score, parent, token, reinterpret_cast<uint64_t *>(stat + parts), stat, d->ld, d->beams, d->vocab, d->keep, splits,
                     d->eos, groups, parts, FastDiv((uint32_t)splits)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d->type == F8_F32) launch_rows<float>(p, nv, s);
  else if (d->type == F8_F16) launch_rows<f16>(p, nv, s);
  else launch_rows<bf16>(p, nv, s);
  const f8_status st = launch_status();
  if (st != F8_OK) return st;
  hipLaunchKernelGGL(beam_join_kernel, dim3(d->batch), dim3(THREADS), (size_t)d->keep * each_of((uint32_t)(d->beams * splits * d->keep)) * sizeof(KeyS), s, p);
  return launch_status();
}

}  // extern "C"
