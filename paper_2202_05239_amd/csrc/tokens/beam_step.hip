// Beam search's selection: the `keep` largest of S[i][t] = score_i + x_it - lse_i over a prompt's beams i and tokens t.
//
// Within a beam S falls with x, so a first launch needs no scores: a workgroup takes up to 16384 logits of a row into its registers and leaves
// their maximum m, sum exp(x - m) and `keep` largest, and a second launch (a workgroup to a prompt) adds up the sums, forms S of what
// is left in 64 bits and takes the `keep` largest of that.  Bound by HBM: the logits are read once (64 prompts of 8 beams, a fifth of them done,
// 131072 bf16 logits, keep 16: 36.6 us for 107 MB, 2.9 TB/s: a wave waits for its piece and then has about 25 instructions to 8 logits; the second
// launch 11.4).  A single prompt of 4 beams and 5001 logits takes 5 + 8 us, a chain of barriers each.
//
// The largest of a set.  Threads form at least `keep` groups; every group's largest element is one of the set's, so the least of these maxima is a
// lower bound of the keep-th largest, which few elements reach (16 of 16384 random ones: about 45).  Those go to a list in LDS, as keys of which no
// two are alike (value, then lowest index), and each one's place is the number of keys above it.  Where more reach it than
// the list holds (many alike), the bound is the keep-th largest of the threads' own largest keys: what passes then are elements of `keep` threads.
// (A vocabulary that a mask leaves a thousandth of takes that way, because a group without any other element has the mask's value as its largest:
// 64 prompts of 8 beams, none done, 131072 bf16 logits, keep 16 then take 219 us instead of 52; with half of it masked 52.)  Placing the list
// compares 64 bits for every two elements of it: with keep 64 the same prompts take 124 us, a single one 58 (keep 16: 27, 8: 20).
//
// The exponentials are taken in 32 bits and 16 of them added there, then on in 64: the log sum is good to 2^-17, and S no better.
#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int CHUNK = 16384;                                // logits of a workgroup at most
constexpr int CANDIDATES = 8192;                            // of a prompt in the second launch at most
constexpr int BEAMS = 1024;
// Keys that the list has room for: those of `keep` threads, or as many as reach a bound that fits loosely
__host__ __device__ inline int list_of(int keep, int each) { return keep * each < 512 ? 512 : keep * each; }
inline int each_of(uint32_t candidates) { return (int)((candidates + THREADS - 1) / THREADS); }   // of a thread there

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
  int batch, beams, vocab, keep, splits, eos, groups;       // groups of threads: a power of two, at least `keep`
  int64_t blocks;
  FastDiv by_splits, by_row;                // by_row: candidates of a row in the second launch
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

constexpr float LOG2E = 1.4426950408889634f;

// Keys: a logit and its token; S, its beam, its logit and token (a score may be so large that 64 bits give two logits of a beam the same
// S: the larger one's is larger).  Key{} is no element.
struct Key64 {
  uint64_t k;
  __device__ __forceinline__ bool operator<(const Key64 &o) const { return k < o.k; }
  __device__ __forceinline__ bool real() const { return k != 0; }
};
struct KeyS {
  uint64_t s, beam, logit;                  // beam: ~i, logit: its order, ~token
  __device__ __forceinline__ bool operator<(const KeyS &o) const {
    return s < o.s || (s == o.s && (beam < o.beam || (beam == o.beam && logit < o.logit)));
  }
  __device__ __forceinline__ bool real() const { return s != 0; }
};

// One instruction for two maxima (fmaxf costs two for one, where it does not know that its operands are no signalling NaN).
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

// The `keep` largest of a list of n keys, none alike: out(place, key) is called for each, places from 0 in descending order.
template <typename K, typename Out>
__device__ __forceinline__ void rank(const K *list, int n, int keep, Out out) {
  for (int i = threadIdx.x; i < n; i += THREADS) {
    const K key = list[i];
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) above += key < list[j];               // (several readings on their way at a time)
    if (above < keep) out(above, key);
  }
}

// The keep-th largest of the threads' keys (Key{} where fewer are real), for all threads.  `top`: a key to a thread, and one more.
template <typename K>
__device__ __forceinline__ K kth(K mine, int keep, K *top) {
  const int t = threadIdx.x;
  __syncthreads();
  top[t] = mine;
  if (t == 0) top[THREADS] = K{};
  __syncthreads();
  int above = 0;
  for (int i = 0; i < THREADS; ++i) above += mine < top[i];
  if (above == keep - 1 && mine.real()) top[THREADS] = mine;
  __syncthreads();
  return top[THREADS];
}

// The least of the groups' largest values, for all threads.  Thread t belongs to group t mod `groups`: neighbours, which hold neighbouring
// elements, to different ones.  wave_top: [THREADS].
__device__ __forceinline__ float least_of_groups(float v, int groups, float *wave_top) {
  const int lane = threadIdx.x & 63;
  for (int d = 32; d >= groups; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
  wave_top[threadIdx.x] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < WAVES; ++w) v = fmaxf(v, wave_top[w * 64 + lane]);
  for (int d = min(groups, 64) >> 1; d > 0; d >>= 1) v = fminf(v, __shfl_xor(v, d));
  return v;
}

template <typename T, int NV>
__global__ __launch_bounds__(THREADS, NV < 8 ? 6 : 4) void beam_rows_kernel(BeamParams p) {
  typedef RowMap<THREADS, NV> Map;
  constexpr int AT_ONCE = 4;
  extern __shared__ __align__(16) uint8_t dynamic[];
  Key64 *const list = reinterpret_cast<Key64 *>(dynamic);             // list_of(keep, NV * 8)
  __shared__ Key64 top_keys[THREADS + 1];
  __shared__ float wave_top[THREADS];
  __shared__ float tops[WAVES];
  __shared__ double sums[WAVES];
  __shared__ uint16_t pieces[THREADS * NV];
  __shared__ int count, reach;
  const int64_t block = row_block();
  if (block >= p.blocks) return;
  const int row = (int)p.by_splits.div((uint32_t)block), split = (int)block - row * p.splits;
  if (p.done && p.done[row]) return;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, most = list_of(p.keep, NV * 8);
  const int base = split * Map::most, cols = min(Map::most, p.vocab - base);
  const T *x = static_cast<const T *>(p.logits) + row * p.ld + base;
  float v[NV][8], piece[NV], top = -INFINITY;
  if (t == 0) count = 0, reach = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) load_piece<T, Map>(x, i, t, cols, v[i]);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int here = cols - Map::col(i, 0, t);              // elements from the piece's first one on
    if (here < 8) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = j < here ? v[i][j] : -INFINITY;
    }
    piece[i] = max3(max3(v[i][0], v[i][1], v[i][2]), max3(v[i][3], v[i][4], v[i][5]), v[i][6]);
    piece[i] = max3(piece[i], v[i][7], v[i][7]);
    top = max3(top, piece[i], piece[i]);
  }
  float m = top;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  if (lane == 0) tops[wave] = m;
  // (values alone: where many are alike, they all pass and the list runs over)
  const float least = least_of_groups(top, p.groups, wave_top);
  // pieces that reach the bound are put down, their elements looked at behind that by a thread each (read once more: 64 branches to 64 places
  // of registers would cost more than the few cached lines)
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (piece[i] >= least) pieces[atomicAdd(&reach, 1)] = (uint16_t)(i * THREADS + t);
  __syncthreads();
  const int elements = reach * 8;
  for (int q0 = t; q0 < elements; q0 += AT_ONCE * THREADS) {
    int col[AT_ONCE];
    T raw[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int q = min(q0 + u * THREADS, elements - 1);
      col[u] = pieces[q >> 3] * 8 + (q & 7);
      raw[u] = x[min(col[u], cols - 1)];
      if (q0 + u * THREADS >= elements) col[u] = cols;
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const float e = (float)raw[u];
      if (col[u] < cols && e >= least) {
        const int at = atomicAdd(&count, 1);
        if (at < most) list[at].k = (uint64_t)order_of(e) << 32 | (uint32_t)~(base + col[u]);
      }
    }
  }
  __syncthreads();
  int n = count;
  if (n > most) {
    // the bound is the keep-th largest of the threads' own largest keys: what passes then are elements of `keep` threads (read once more, one
    // by one: this way must not cost the other one registers)
    auto each = [&](auto f) {
#pragma unroll 1
      for (int i = 0; i < NV; ++i)
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
          const int col = Map::col(i, j, t);
          if (col < cols) f(Key64{(uint64_t)order_of((float)x[col]) << 32 | (uint32_t)~(base + col)});
        }
    };
    Key64 mine{};
    each([&](Key64 key) {
      if (mine < key) mine = key;
    });
    const Key64 bound = kth<Key64>(mine, p.keep, top_keys);
    if (t == 0) count = 0;
    __syncthreads();
    each([&](Key64 key) {
      if (!(key < bound)) {
        const int to = atomicAdd(&count, 1);
        if (to < most) list[to] = key;
      }
    });
    __syncthreads();
    n = min(count, most);
  }
  rank<Key64>(list, n, p.keep, [&](int place, Key64 key) { p.best[block * p.keep + place] = key.k; });
  if (t >= n && t < p.keep) p.best[block * p.keep + t] = 0;
  m = tops[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) m = fmaxf(m, tops[w]);
  // (NaN and +infinity come out as a sum that is NaN: fmaxf passes over a NaN, the differences do not)
  float part[4] = {0, 0, 0, 0};
  if (m != -INFINITY) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) part[j & 3] += __builtin_amdgcn_exp2f((v[i][j] - m) * LOG2E);
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) part[0] += v[i][j] != v[i][j] ? v[i][j] : 0.0f;
  }
  double sum = ((double)part[0] + (double)part[1]) + ((double)part[2] + (double)part[3]);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  if (t == 0) {
    for (int w = 1; w < WAVES; ++w) sum += sums[w];
    p.stat[block] = Stat{sum, m};
  }
}

// PER: candidates of a thread, held in registers
template <int PER>
__global__ __launch_bounds__(THREADS) void beam_join_kernel(BeamParams p) {
  extern __shared__ __align__(16) uint8_t dynamic[];
  KeyS *const list = reinterpret_cast<KeyS *>(dynamic);               // list_of(keep, PER)
  __shared__ KeyS top_keys[THREADS + 1];
  __shared__ uint64_t wave_top[THREADS], least;
  __shared__ double lse[BEAMS];             // NaN or -infinity: S of the beam is that throughout; 0: it is done
  __shared__ float score_of[BEAMS];
  __shared__ uint8_t done_of[BEAMS];
  __shared__ int count;
  if (row_block() >= p.batch) return;
  const int b = (int)row_block(), t = threadIdx.x;
  const int64_t row0 = (int64_t)b * p.beams;
  const uint32_t per_row = (uint32_t)p.splits * p.keep, all = per_row * p.beams;
  // the candidates' logits on their way, while the sums are added up (those of beams that are done were not written: not looked at)
  // A part of a row has its candidates in descending order: threads take different ranks, one of the first among them, so that their largest ones
  // bound the keep-th largest closely (with one rank each: 64 of 131072 logits of one beam took 160 us, a thousand candidates passing).
  const uint32_t turn = (p.keep + PER - 1) / PER;
  auto candidate = [&](int k) { return (uint32_t)k * THREADS + ((t + k * turn) & (THREADS - 1)); };
  uint64_t logit[PER];
#pragma unroll
  for (int k = 0; k < PER; ++k) logit[k] = p.best[row0 * per_row + min(candidate(k), all - 1)];
  if (t == 0) count = 0;
  // `width` lanes to a beam, one to a workgroup's part of the row: all beams at a time, if they fit
  int width = 1;
  while (width < p.splits && width < 64) width *= 2;
  const int in_beam = t & (width - 1);
  for (int i = t / width; i < p.beams; i += THREADS / width) {
    const float score = p.scores[row0 + i];
    const bool done = p.done && p.done[row0 + i];
    const Stat *s = p.stat + (row0 + i) * p.splits;
    float top = -INFINITY;
    double sum = 0;
    if (!done) {
      for (int j = in_beam; j < p.splits; j += width) {
        const Stat x = s[j];
        const float now = fmaxf(top, x.top);
        // (a part without a number above -infinity adds its sum as it is: 0, or NaN)
        if (top != -INFINITY && now > top) sum *= exp((double)top - (double)now);
        sum += x.top == -INFINITY || x.top == now ? x.sum : x.sum * exp((double)x.top - (double)now);
        top = now;
      }
      float all_top = top;
      for (int d = width >> 1; d > 0; d >>= 1) all_top = fmaxf(all_top, __shfl_xor(all_top, d));
      if (top != -INFINITY && top < all_top) sum *= exp((double)top - (double)all_top);
      for (int d = width >> 1; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
      top = all_top;
    }
    if (in_beam == 0) {
      score_of[i] = score, done_of[i] = done;
      const bool bad = !(score < INFINITY) || sum != sum;               // (the sum of a beam that is done is 0)
      lse[i] = bad ? (double)__builtin_nanf("") : score == -INFINITY ? (double)score : done ? 0 : sum == 0 ? -(double)INFINITY : (double)top + log(sum);
    }
  }
  __syncthreads();
  KeyS key[PER];
  uint64_t largest = 0;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const uint32_t c = candidate(k), i = min(p.by_row.div(c), (uint32_t)p.beams - 1), in = c - i * per_row;
    const float score = score_of[i];
    const double of = lse[i];
    const bool some = in < (uint32_t)min(p.keep, p.vocab);              // of a row whose tokens are not looked at
    uint64_t x = logit[k];                                              // (where S is the same throughout: tokens in their order)
    double s;
    if (of != of || of == -(double)INFINITY) {
      x = some ? (uint32_t)~in : 0, s = of;
    } else if (done_of[i]) {
      x = some ? (uint32_t)~(in == 0 ? p.eos : in - (in <= (uint32_t)p.eos)) : 0, s = in == 0 ? (double)score : -(double)INFINITY;
    } else {
      s = (double)score + ((double)of_order((uint32_t)(x >> 32)) - of);
    }
    if (c >= all) x = 0;
    key[k] = x == 0 ? KeyS{} : KeyS{order_of(s), ~(uint64_t)i, x};
    if (largest < key[k].s) largest = key[k].s;
  }
  // the keep-th largest of the threads' largest (in S alone)
  wave_top[t] = largest;
  if (t == 0) least = ~0ull;
  __syncthreads();
  int above = 0;
#pragma unroll 8
  for (int i = 0; i < THREADS; ++i) above += largest < wave_top[i];
  if (above < p.keep) atomicMin((unsigned long long *)&least, (unsigned long long)largest);
  __syncthreads();
  const int most = list_of(p.keep, PER);
  auto collect = [&](KeyS bound) {
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (key[k].real() && !(key[k] < bound)) {
        const int at = atomicAdd(&count, 1);
        if (at < most) list[at] = key[k];
      }
  };
  collect(KeyS{least, 0, 0});
  __syncthreads();
  int n = count;
  if (n > most) {
    KeyS most_of{};
#pragma unroll
    for (int k = 0; k < PER; ++k)
      if (most_of < key[k]) most_of = key[k];
    const KeyS bound = kth<KeyS>(most_of, p.keep, top_keys);
    if (t == 0) count = 0;
    __syncthreads();
    collect(bound);
    __syncthreads();
    n = min(count, most);
  }
  const int64_t out = (int64_t)b * p.keep;
  rank<KeyS>(list, n, p.keep, [&](int place, KeyS k) {
    p.score[out + place] = (float)of_order(k.s);
    p.parent[out + place] = (int32_t)(row0 + (int64_t)~k.beam);
    p.token[out + place] = (int32_t)~(uint32_t)k.logit;
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
  const size_t lds = (size_t)list_of(p.keep, nv * 8) * sizeof(Key64);
  switch (nv) {
    case 1: hipLaunchKernelGGL((beam_rows_kernel<T, 1>), grid, block, lds, s, p); break;
    case 2: hipLaunchKernelGGL((beam_rows_kernel<T, 2>), grid, block, lds, s, p); break;
    case 4: hipLaunchKernelGGL((beam_rows_kernel<T, 4>), grid, block, lds, s, p); break;
    default: hipLaunchKernelGGL((beam_rows_kernel<T, 8>), grid, block, lds, s, p);
  }
}

template <int PER>
void launch_join(const BeamParams &p, hipStream_t s) {
  static_assert(CANDIDATES <= 32 * THREADS, "candidates of a thread");
  hipLaunchKernelGGL((beam_join_kernel<PER>), block_grid(p.batch), dim3(THREADS), (size_t)list_of(p.keep, PER) * sizeof(KeyS), s, p);
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
  if (score == scores) return F8_ERR_SHAPE;                // (other prompts' workgroups read them while they are written)
  int groups = 1;
  while (groups < d->keep) groups *= 2;
  const int64_t parts = rows * splits;
  Stat *stat = static_cast<Stat *>(workspace);
  const BeamParams p{logits, scores, done, score, parent, token, reinterpret_cast<uint64_t *>(stat + parts), stat, d->ld, d->batch, d->beams, d->vocab, d->keep, splits,
                     d->eos, groups, parts, FastDiv((uint32_t)splits), FastDiv((uint32_t)(splits * d->keep))};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d->type == F8_F32) launch_rows<float>(p, nv, s);
  else if (d->type == F8_F16) launch_rows<f16>(p, nv, s);
  else launch_rows<bf16>(p, nv, s);
  const f8_status st = launch_status();
  if (st != F8_OK) return st;
  const int each = each_of((uint32_t)(d->beams * splits * d->keep));
  if (each <= 4) launch_join<4>(p, s);
  else if (each <= 16) launch_join<16>(p, s);
  else launch_join<32>(p, s);
  return launch_status();
}

}  // extern "C"
