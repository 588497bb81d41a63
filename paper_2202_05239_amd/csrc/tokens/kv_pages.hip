// The pages of a cache as its block tables and a count of holders per page see them: forking requests and compacting the pool.  Integers
// only; what has to be copied in the cache comes out as a list for f8_kv_copy.
//
// A page is free where its count is not positive.  New pages are the free ones of the lowest index, handed out in the order of the
// requests, so a result depends on its inputs alone: the only atomics add to counts or take a minimum.
//
// Bound by latencies: a few hundred kilobytes at most, in phases that wait for one another.  What fits one workgroup's LDS is one launch: 64
// requests of up to 2048 tokens fork in 14 us (49 with the counts in memory), a pool of 1001 pages is compacted in 4.4 us (three launches
// take 11).  More takes the phases as launches: 512 requests of up to 32768 tokens fork in 25 us, 262144 pages with 512 rows of 513 entries
// are compacted in 18.  The search for free pages is one workgroup's and ends where enough are found: 512 new pages out of 262144, 97 % in use,
// take 29 us where the free ones lie all over the pool and 160 where they lie at its end, as behind a compaction (of 65536: 29 and 51, of
// 20000: 27 and 26).
#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

constexpr int WAVES = 16, THREADS = 64 * WAVES;

// What this workgroup's or other ones' atomics have written is read where they wrote it, behind the first-level cache.
__device__ __forceinline__ int seen(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void put(int32_t *p, int v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void add(int32_t *p, int v) { __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Sums over the threads in front of this one, of K values; `all`: over the whole workgroup.
template <int K>
__device__ __forceinline__ void scan(const int (&v)[K], int (&before)[K], int (&all)[K], int (*lds)[K]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    upto[k] = v[k];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(upto[k], d);
      if (lane >= d) upto[k] += o;
    }
    if (lane == 63) lds[wave][k] = upto[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < K; ++k) {
    before[k] = upto[k] - v[k], all[k] = 0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
      const int o = lds[w][k];
      if (w < wave) before[k] += o;
      all[k] += o;
    }
  }
  __syncthreads();
}

// Where the counts are while new pages are dealt out: of each page its count, the lowest of the requests that write behind it, and how
// many those are; the new pages; of each request the place of its first one among them (twice that, and 1 more where it is a copy).
struct Pool {
  int32_t *refs, *lowest, *writers, *fresh, *at;
};

struct ForkParams {
  const int32_t *parent, *table, *lens, *refs;
  int32_t *table_out, *lens_out, *refs_out;
  int64_t *slots;
  int32_t *moves, *info;
  Pool pool;                                 // refs: refs_out, the others: workspace
  int32_t *found;                            // how many new pages there are
  int64_t table_ld, out_ld;
  int batch, cols, pages, grow;
  FastDiv page_size, by_cols, by_grow;       // the last two: of one workgroup's case
};

__device__ __forceinline__ int pages_of(const ForkParams &p, int tokens) { return tokens > 0 ? (int)p.page_size.div((uint32_t)tokens - 1) + 1 : 0; }
__device__ __forceinline__ int tokens_of(const ForkParams &p, int len) { return min(max(len, 0), p.cols * (int)p.page_size.d); }

struct Child {                               // what a request is to be: the parent's row (-1: it ends), its tokens and pages
  int row, tokens, pages;
};
__device__ __forceinline__ Child child_of(const ForkParams &p, int b) {
  const int row = p.parent[b];
  if ((uint32_t)row >= (uint32_t)p.batch) return Child{-1, 0, 0};
  const int tokens = tokens_of(p, p.lens[row]);
  return Child{row, tokens, pages_of(p, tokens)};
}

struct Branch {
  Child c;
  int full, tail;                            // pages that are full; the page behind them that it will write into (-1: none)
};
__device__ __forceinline__ Branch branch_of(const ForkParams &p, int b) {
  const Child c = child_of(p, b);
  const int full = (int)p.page_size.div((uint32_t)c.tokens);
  if (p.grow == 0 || full == c.pages) return Branch{c, full, -1};
  const int page = p.table[c.row * p.table_ld + full];
  return Branch{c, full, (uint32_t)page < (uint32_t)p.pages ? page : -1};
}
// Columns of the row that it is to have
__device__ __forceinline__ int columns_of(const ForkParams &p, const Child &c) {
  const int64_t upto = min((int64_t)c.tokens + p.grow, (int64_t)p.cols * (int)p.page_size.d);
  return c.row < 0 ? 0 : pages_of(p, (int)upto);
}

// Who copies, who gets which new page.  One workgroup; branch(b): of this thread's requests b.  Returns how many new pages there are, and
// the copies among them.
template <class F>
__device__ __forceinline__ int fork_assign(const ForkParams &p, const Pool &pool, F branch, int &copied_out) {
  __shared__ int lds[WAVES][2], moved;
  constexpr int EACH = 8;                    // pages of a thread at a time
  const int page_size = (int)p.page_size.d;
  // requests that will write into a page that is not full: the lowest of them keeps it, if all that hold it write
  if (threadIdx.x == 0) moved = 0;
  for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
    const int page = branch(b).tail;
    if (page >= 0) put(pool.lowest + page, 0x7fffffff), put(pool.writers + page, 0);
  }
  __syncthreads();
  for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
    const int page = branch(b).tail;
    if (page >= 0) {
      __hip_atomic_fetch_min(pool.lowest + page, b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      add(pool.writers + page, 1);
    }
  }
  __syncthreads();
  // places among the new pages, and how many of those there are
  int wanted = 0, beyond = 0;
  for (int b0 = 0; b0 < p.batch; b0 += blockDim.x) {
    const int b = b0 + (int)threadIdx.x;
    int v[2] = {0, 0}, before[2], all[2];
    bool copies = false;
    if (b < p.batch) {
      const Branch r = branch(b);
      if (r.tail >= 0) {
        const int held = seen(pool.refs + r.tail), writers = seen(pool.writers + r.tail), lowest = seen(pool.lowest + r.tail);
        copies = held != writers || lowest != b;
      }
      if (r.c.row >= 0) {
        const int64_t need = ((int64_t)r.c.tokens + p.grow + page_size - 1) / page_size;
        v[0] = (int)min(need, (int64_t)p.cols) - r.c.pages + copies, v[1] = (int)(need - min(need, (int64_t)p.cols));
      }
    }
    scan<2>(v, before, all, lds);
    if (b < p.batch) put(pool.at + b, 2 * (wanted + before[0]) + copies);
    wanted += all[0], beyond += all[1];
  }
  // (from here on a tail's `writers` is its place among the new pages, -1: none.  A count that is not positive although a row names the page
  // makes it a new one too, and what its holders give up before it is handed out is gone then)
  for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
    const int page = branch(b).tail;
    if (page >= 0) put(pool.writers + page, -1);
  }
  // the free pages of the lowest index
  int found = 0;
  for (int64_t i0 = 0; i0 < p.pages && found < wanted; i0 += EACH * blockDim.x) {
    const int64_t i = i0 + EACH * (int)threadIdx.x;
    int free[EACH], v[1] = {0}, before[1], all[1];
#pragma unroll
    for (int j = 0; j < EACH; ++j) free[j] = seen(pool.refs + min(i + j, (int64_t)p.pages - 1));
#pragma unroll
    for (int j = 0; j < EACH; ++j) free[j] = free[j] <= 0 && i + j < p.pages, v[0] += free[j];
    scan<1>(v, before, all, reinterpret_cast<int(*)[1]>(lds));
    int place = found + before[0];
#pragma unroll
    for (int j = 0; j < EACH; ++j)
      if (free[j]) {
        if (place < wanted) put(pool.fresh + place, (int)(i + j));
        ++place;
      }
    found += all[0];
  }
  found = min(found, wanted);
  __syncthreads();
  for (int i = threadIdx.x; i < found; i += blockDim.x) {
    const int page = seen(pool.fresh + i);
    put(pool.refs + page, 1), put(pool.writers + page, i);
  }
  __syncthreads();
  // the copies, one behind the other (those that no page was left for are the last)
  int copied = 0;
  for (int b0 = 0; b0 < p.batch; b0 += blockDim.x) {
    const int b = b0 + (int)threadIdx.x, at = b < p.batch ? seen(pool.at + b) : 0;
    int v[1] = {at & 1}, before[1], all[1];
    scan<1>(v, before, all, reinterpret_cast<int(*)[1]>(lds));
    if (v[0]) {
      const Branch r = branch(b);
      const int to = (at >> 1) < found ? seen(pool.fresh + (at >> 1)) : -1;
      if (seen(pool.writers + r.tail) <= (at >> 1)) add(pool.refs + r.tail, -1);
      if (to >= 0) {
        int32_t *m = p.moves + 3 * (int64_t)(copied + before[0]);
        m[0] = r.tail, m[1] = to, m[2] = r.c.tokens - r.full * page_size;
        atomicMax(&moved, copied + before[0] + 1);
      }
    }
    copied += all[0];
  }
  __syncthreads();
  if (threadIdx.x == 0) p.info[0] = moved, p.info[1] = wanted - found + beyond;
  copied_out = moved;
  return found;
}

// The entry of a request's new row in column col < columns_of, and the slot of its j-th new token.
__device__ __forceinline__ int entry_of(const ForkParams &p, const Pool &pool, const Child &c, int at, int found, int col) {
  const int kept = c.pages - (at & 1);       // (a copied page is the last one)
  if (col < kept) return p.table[c.row * p.table_ld + col];
  const int i = (at >> 1) + col - kept;
  return i < found ? seen(pool.fresh + i) : -1;
}
__device__ __forceinline__ int64_t slot_of(const ForkParams &p, const Pool &pool, const Child &c, int at, int found, int j) {
  const int page_size = (int)p.page_size.d;
  if (c.row < 0 || (int64_t)c.tokens + j >= (int64_t)p.cols * page_size) return -1;
  const int t = c.tokens + j, col = (int)p.page_size.div((uint32_t)t), page = entry_of(p, pool, c, at, found, col);
  return (uint32_t)page < (uint32_t)p.pages ? (int64_t)page * page_size + (t - col * page_size) : -1;
}

// All of it in one workgroup, with the counts in LDS: what takes time is that one reading waits for another (parent, length, tail), so each
// is done once.
// In a graph, one workgroup against the launches below, us: 4 requests, 600 pages 9.4, 14.6; 8192 pages, 64 requests of 128 columns 15.7, 20.4, 128
// of 128 20.6, 20.5, 1024 of 16 23.7, 28.9; compaction of 600 pages 4.7, 10.0, of 8192 with 64 rows of 128 7.7, 12.6, with 128 9.9, 12.2.
constexpr int SMALL_PAGES = 8192, SMALL_ENTRIES = 16384, SMALL_GROW = 4096;

__global__ __launch_bounds__(THREADS) void fork_small_kernel(ForkParams p) {
  __shared__ int32_t refs[SMALL_PAGES], lowest[SMALL_PAGES], writers[SMALL_PAGES], fresh[SMALL_PAGES], at[THREADS];
  __shared__ Child child[THREADS];
  __shared__ int used[THREADS], children[THREADS];
  constexpr int EACH = SMALL_PAGES / THREADS;
  const int t = threadIdx.x, entries = p.batch * p.cols;
  const Pool pool{refs, lowest, writers, fresh, at};
  int held[EACH];
#pragma unroll
  for (int j = 0; j < EACH; ++j) held[j] = p.refs[min(j * THREADS + t, p.pages - 1)];
  const int own = t < p.batch ? pages_of(p, tokens_of(p, p.lens[t])) : 0;
  const Branch mine = t < p.batch ? branch_of(p, t) : Branch{{-1, 0, 0}, 0, -1};
#pragma unroll
  for (int j = 0; j < EACH; ++j) refs[j * THREADS + t] = held[j];
  children[t] = 0, used[t] = own, child[t] = mine.c;
  __syncthreads();
  if (mine.c.row >= 0) atomicAdd(&children[mine.c.row], 1);
  __syncthreads();
  // a page's holders: each child holds what its parent held
#pragma unroll 4
  for (int i = t; i < entries; i += THREADS) {
    const int b = (int)p.by_cols.div((uint32_t)i), col = i - b * p.cols, page = p.table[b * p.table_ld + col], n = children[b] - 1;
    if (col < used[b] && n != 0 && (uint32_t)page < (uint32_t)p.pages) atomicAdd(&refs[page], n);
  }
  __syncthreads();
  int moved;
  const int found = fork_assign(p, pool, [&](int) { return mine; }, moved);
#pragma unroll 4
  for (int i = t; i < entries; i += THREADS) {
    const int b = (int)p.by_cols.div((uint32_t)i), col = i - b * p.cols;
    const Child c = child[b];
    p.table_out[b * p.out_ld + col] = col < columns_of(p, c) ? entry_of(p, pool, c, at[b], found, col) : -1;
  }
  for (int i = t; i < p.batch * p.grow; i += THREADS) {
    const int b = (int)p.by_grow.div((uint32_t)i);
    p.slots[i] = slot_of(p, pool, child[b], at[b], found, i - b * p.grow);
  }
  for (int i = t; i < p.pages; i += THREADS) p.refs_out[i] = refs[i];
  for (int i = 3 * moved + t; i < 3 * p.batch; i += THREADS) p.moves[i] = i % 3 == 2 ? 0 : -1;
  if (t < p.batch) p.lens_out[t] = mine.c.row < 0 ? 0 : (int)min((int64_t)mine.c.tokens + p.grow, (int64_t)p.cols * (int)p.page_size.d);
}

// The same phases as launches of many workgroups (256 threads each, but for the assignment).  Counts as they were, lists without entries.
__global__ __launch_bounds__(256) void fork_counts_kernel(ForkParams p) {
  const int64_t step = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t i = first; i < p.pages; i += step) p.refs_out[i] = p.refs[i];
  for (int64_t i = first; i < 3 * (int64_t)p.batch; i += step) p.moves[i] = i % 3 == 2 ? 0 : -1;
}
__global__ __launch_bounds__(256) void fork_hold_kernel(ForkParams p) {
  __shared__ int children;
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
    if (threadIdx.x == 0) children = 0;
    __syncthreads();
    int mine = 0;
    for (int i = threadIdx.x; i < p.batch; i += 256) mine += p.parent[i] == b;
    if (mine) atomicAdd(&children, mine);
    __syncthreads();
    const int n = children - 1;
    if (n != 0) {
      const int used = pages_of(p, tokens_of(p, p.lens[b]));
      for (int i = threadIdx.x; i < used; i += 256) {
        const int page = p.table[b * p.table_ld + i];
        if ((uint32_t)page < (uint32_t)p.pages) add(p.refs_out + page, n);
      }
    }
    __syncthreads();
  }
}
__global__ __launch_bounds__(THREADS) void fork_assign_kernel(ForkParams p) {
  const Branch mine = (int)threadIdx.x < p.batch ? branch_of(p, threadIdx.x) : Branch{{-1, 0, 0}, 0, -1};
  int moved;
  const int found = fork_assign(p, p.pool, [&](int b) { return b == (int)threadIdx.x ? mine : branch_of(p, b); }, moved);
  if (threadIdx.x == 0) *p.found = found;
}
__global__ __launch_bounds__(256) void fork_rows_kernel(ForkParams p) {
  const int found = *p.found;
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
    const Child c = child_of(p, b);
    const int at = p.pool.at[b], columns = columns_of(p, c);
    for (int i = threadIdx.x; i < p.cols; i += 256) p.table_out[b * p.out_ld + i] = i < columns ? entry_of(p, p.pool, c, at, found, i) : -1;
    for (int j = threadIdx.x; j < p.grow; j += 256) p.slots[(int64_t)b * p.grow + j] = slot_of(p, p.pool, c, at, found, j);
    if (threadIdx.x == 0) p.lens_out[b] = c.row < 0 ? 0 : (int)min((int64_t)c.tokens + p.grow, (int64_t)p.cols * (int)p.page_size.d);
  }
}

// ---- compaction ----

constexpr int PER = 4, BLOCK = 256 * PER;    // pages of a thread and of a workgroup

struct CompactParams {
  const int32_t *table, *refs;
  int32_t *table_out, *refs_out, *moves, *info;
  int32_t *counts, *rank;                   // workspace: pages in use of each block; of a page that goes, and of a hole, its place in the list
  int64_t table_ld, out_ld, entries;
  int cols, pages, page_size, blocks, page_wgs;
  FastDiv by_cols;
};

// All of it in one workgroup, with the counts in LDS.
__global__ __launch_bounds__(THREADS) void compact_small_kernel(CompactParams p) {
  constexpr int EACH = SMALL_PAGES / THREADS;
  __shared__ int32_t refs[SMALL_PAGES], to[SMALL_PAGES], holes[SMALL_PAGES / 2], gone[SMALL_PAGES / 2];
  __shared__ int lds[WAVES][1], moved_of;
  const int t = threadIdx.x;
  int held[EACH], v[1] = {0}, before[1], all[1];
#pragma unroll
  for (int j = 0; j < EACH; ++j) held[j] = p.refs[min(j * THREADS + t, p.pages - 1)];
#pragma unroll
  for (int j = 0; j < EACH; ++j) refs[j * THREADS + t] = j * THREADS + t < p.pages ? held[j] : 0;
  if (t == 0) moved_of = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < EACH; ++j) held[j] = refs[t * EACH + j] > 0, v[0] += held[j];
  scan<1>(v, before, all, lds);
  const int used = all[0];
  int rank = before[0];                     // pages in use in front of this one
#pragma unroll
  for (int j = 0; j < EACH; ++j) {
    const int i = t * EACH + j;
    if (i == used) moved_of = used - rank;
    if (held[j] && i >= used) gone[used - 1 - rank] = i;    // (the last one first)
    if (!held[j] && i < used) holes[i - rank] = i;
    rank += held[j];
  }
  __syncthreads();
  const int moved = moved_of;
  for (int k = t; k < p.pages / 2; k += THREADS) {
    int from = -1, hole = -1;
    if (k < moved) {
      from = gone[moved - 1 - k], hole = holes[k];
      to[from] = hole, refs[hole] = refs[from];
    }
    p.moves[3 * k] = from, p.moves[3 * k + 1] = hole, p.moves[3 * k + 2] = k < moved ? p.page_size : 0;
  }
  __syncthreads();
  for (int i = t; i < p.pages; i += THREADS) p.refs_out[i] = i < used ? refs[i] : 0;
#pragma unroll 4
  for (int i = t; i < (int)p.entries; i += THREADS) {
    const int row = (int)p.by_cols.div((uint32_t)i), col = i - row * p.cols;
    int e = p.table[row * p.table_ld + col];
    if (e >= used && e < p.pages && refs[e] > 0) e = to[e];
    p.table_out[row * p.out_ld + col] = e;
  }
  if (t == 0) p.info[0] = moved, p.info[1] = used;
}

__global__ __launch_bounds__(256) void compact_count_kernel(CompactParams p) {
  __shared__ int lds[4][1];
  int v[1] = {0}, before[1], all[1];
  // (a page index may pass 31 bits by a block)
  const int64_t base = (int64_t)blockIdx.x * BLOCK;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int64_t i = base + j * 256 + threadIdx.x;
    v[0] += p.refs[min(i, (int64_t)p.pages - 1)] > 0 && i < p.pages;
  }
  scan<1>(v, before, all, lds);
  if (threadIdx.x == 0) p.counts[blockIdx.x] = all[0];
}

// Sums of the blocks' counts: of all, and of those in front of block `upto`.
__device__ __forceinline__ void block_sums(const CompactParams &p, int upto, int &all, int &front, int (*lds)[2]) {
  int v[2] = {0, 0}, before[2], sums[2];
  for (int i = threadIdx.x; i < p.blocks; i += 256) {
    const int n = p.counts[i];
    v[0] += n;
    if (i < upto) v[1] += n;
  }
  scan<2>(v, before, sums, lds);
  all = sums[0], front = sums[1];
}

__global__ __launch_bounds__(256) void compact_lists_kernel(CompactParams p) {
  __shared__ int lds[4][2];
  const int64_t base = (int64_t)blockIdx.x * BLOCK + (int)threadIdx.x * PER;
  int held[PER];
#pragma unroll
  for (int j = 0; j < PER; ++j) held[j] = p.refs[min(base + j, (int64_t)p.pages - 1)];
  int used, front, front_of_border, dummy;
  block_sums(p, blockIdx.x, used, front, lds);
  // pages in use in front of the border: those of the blocks before it, and of its own block
  const int border = used / BLOCK;
  block_sums(p, border, dummy, front_of_border, lds);
  int v[2] = {0, 0}, before[2], all[2];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int i = border * BLOCK + j * 256 + (int)threadIdx.x;
    v[1] += p.refs[min(i, p.pages - 1)] > 0 && i < used;
    held[j] = held[j] > 0 && base + j < p.pages, v[0] += held[j];
  }
  scan<2>(v, before, all, lds);
  front_of_border += all[1];
  const int moved = used - front_of_border;
  int rank = front + before[0];             // pages in use in front of this one
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int64_t i = base + j;
    if (i < p.pages) {
      if (held[j] && i >= used) {
        const int at = rank - front_of_border;
        p.moves[3 * (int64_t)at] = (int)i, p.rank[i] = at;
      } else if (!held[j] && i < used) {
        const int at = (int)i - rank;
        p.moves[3 * (int64_t)at + 1] = (int)i, p.moves[3 * (int64_t)at + 2] = p.page_size, p.rank[i] = at;
      }
    }
    rank += held[j];
  }
  // places of the list behind the last move
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.pages / 2; i += (int64_t)gridDim.x * 256)
    if (i >= moved) p.moves[3 * i] = -1, p.moves[3 * i + 1] = -1, p.moves[3 * i + 2] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) p.info[0] = moved, p.info[1] = used;
}

// The first page_wgs workgroups write the counts, the others the table.  Readings that wait for one another are what costs, so four of each
// are under way at a time, of places that need none too.
__global__ __launch_bounds__(256) void compact_apply_kernel(CompactParams p) {
  const int used = p.info[1];
  const int32_t *moves = p.pages > 1 ? p.moves : p.info;    // (a single page moves nowhere and its list may be null)
  const bool counts = (int)blockIdx.x < p.page_wgs;
  const int64_t wg = counts ? blockIdx.x : blockIdx.x - p.page_wgs, wgs = counts ? p.page_wgs : gridDim.x - p.page_wgs;
  const int64_t step = wgs * 1024, all = counts ? p.pages : p.entries;
  for (int64_t i0 = wg * 1024 + threadIdx.x; i0 < all; i0 += step) {
    int page[4], n[4], at[4];
    int64_t place[4];
    bool moves_it[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t i = min(i0 + j * 256, all - 1);
      if (counts) {
        page[j] = (int)i, place[j] = i;
      } else {
        const int64_t row = i <= 0x7fffffff ? (int64_t)p.by_cols.div((uint32_t)i) : i / p.cols;
        const int64_t col = i - row * p.cols;
        page[j] = p.table[row * p.table_ld + col], place[j] = row * p.out_ld + col;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int known = (uint32_t)page[j] < (uint32_t)p.pages ? page[j] : 0;
      n[j] = p.refs[known], at[j] = p.rank[known];
      moves_it[j] = counts ? page[j] < used && n[j] <= 0 : page[j] >= used && page[j] < p.pages && n[j] > 0;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) at[j] = moves[3 * (int64_t)(moves_it[j] ? at[j] : 0) + !counts];
    if (counts) {
#pragma unroll
      for (int j = 0; j < 4; ++j) at[j] = p.refs[moves_it[j] ? at[j] : 0];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i0 + j * 256 < all) p.refs_out[place[j]] = moves_it[j] ? at[j] : page[j] < used ? n[j] : 0;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i0 + j * 256 < all) p.table_out[place[j]] = moves_it[j] ? at[j] : page[j];
    }
  }
}

}  // namespace
}  // namespace f8

using namespace f8;

extern "C" {

size_t f8_kv_fork_workspace_bytes(int batch, int pages) {
  if (batch < 1 || pages < 1) return 0;
  return ((size_t)3 * pages + batch + 1) * sizeof(int32_t);
}

f8_status f8_kv_fork(const int32_t *parent, const int32_t *table, const int32_t *lens, const int32_t *refs, int32_t *table_out, int32_t *lens_out,
                     int32_t *refs_out, int64_t *slots, int32_t *moves, int32_t *info, const f8_kv_fork_desc *d, void *workspace,
                     size_t workspace_bytes, void *stream) {
  if (!d) return F8_ERR_NULL;
  if (d->batch < 0 || d->batch > 65535 || d->cols < 1 || d->pages < 1 || d->page_size < 1 || d->grow < 0 || d->table_ld < d->cols || d->out_ld < d->cols)
    return F8_ERR_SHAPE;
  // (loops over tokens and columns count in 32 bits, a workgroup's threads at a time)
  if ((int64_t)d->cols * d->page_size > 0x7fff0000 || d->grow > 0x7fff0000) return F8_ERR_SHAPE;
  if ((int64_t)d->batch * d->cols > 0x1fffffff || (int64_t)d->batch * (d->grow / d->page_size + 2) > 0x1fffffff || d->pages > 0x3fffffff)
    return F8_ERR_UNSUPPORTED;
  if (d->batch == 0) return F8_OK;
  if (!parent || !table || !lens || !refs || !table_out || !lens_out || !refs_out || (!slots && d->grow > 0) || !moves || !info || !workspace)
    return F8_ERR_NULL;
  for (const void *x : {(const void *)parent, (const void *)table, (const void *)lens, (const void *)refs, (const void *)table_out, (const void *)lens_out,
                        (const void *)refs_out, (const void *)moves, (const void *)info})
    if (!aligned_to(x, 4)) return F8_ERR_ALIGN;
  if (!aligned_to(slots, 8) || !aligned_to(workspace, 16)) return F8_ERR_ALIGN;
  if (workspace_bytes < f8_kv_fork_workspace_bytes(d->batch, d->pages)) return F8_ERR_SHAPE;
  if (table_out == table || lens_out == lens || lens_out == parent || refs_out == refs) return F8_ERR_SHAPE;      // (read while they are written)
  int32_t *ws = static_cast<int32_t *>(workspace);
  const size_t n = (size_t)d->pages;
  const ForkParams p{parent, table, lens, refs, table_out, lens_out, refs_out, slots, moves, info, Pool{refs_out, ws, ws + n, ws + 2 * n, ws + 3 * n},
                     ws + 3 * n + d->batch, d->table_ld, d->out_ld, d->batch, d->cols, d->pages, d->grow, FastDiv((uint32_t)d->page_size),
                     FastDiv((uint32_t)d->cols), FastDiv((uint32_t)(d->grow < 1 ? 1 : d->grow))};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d->batch <= THREADS && (int64_t)d->batch * d->cols <= SMALL_ENTRIES && d->pages <= SMALL_PAGES && (int64_t)d->batch * d->grow <= SMALL_GROW) {
    hipLaunchKernelGGL(fork_small_kernel, dim3(1), dim3(THREADS), 0, s, p);
    return launch_status();
  }
  const int rows = d->batch < 2048 ? d->batch : 2048, most = d->pages > 3 * d->batch ? d->pages : 3 * d->batch, counts = (most + 1023) / 1024;
  hipLaunchKernelGGL(fork_counts_kernel, dim3(counts < 2048 ? counts : 2048), dim3(256), 0, s, p);
  f8_status st = launch_status();
  if (st != F8_OK) return st;
  hipLaunchKernelGGL(fork_hold_kernel, dim3(rows), dim3(256), 0, s, p);
  if ((st = launch_status()) != F8_OK) return st;
  hipLaunchKernelGGL(fork_assign_kernel, dim3(1), dim3(THREADS), 0, s, p);
  if ((st = launch_status()) != F8_OK) return st;
  hipLaunchKernelGGL(fork_rows_kernel, dim3(rows), dim3(256), 0, s, p);
  return launch_status();
}

size_t f8_kv_compact_workspace_bytes(int pages) {
  if (pages < 1) return 0;
  return ((size_t)pages + ((size_t)pages + BLOCK - 1) / BLOCK) * sizeof(int32_t);
}

f8_status f8_kv_compact(const int32_t *table, const int32_t *refs, int32_t *table_out, int32_t *refs_out, int32_t *moves, int32_t *info,
                        const f8_kv_compact_desc *d, void *workspace, size_t workspace_bytes, void *stream) {
  if (!d) return F8_ERR_NULL;
  if (d->rows < 0 || d->cols < 0 || d->pages < 1 || d->page_size < 1 || d->table_ld < d->cols || d->out_ld < d->cols) return F8_ERR_SHAPE;
  if (d->pages > 0x3fffffff) return F8_ERR_UNSUPPORTED;
  const int64_t entries = (int64_t)d->rows * d->cols;
  if (!refs || !refs_out || (!moves && d->pages > 1) || !info || !workspace || (entries > 0 && (!table || !table_out))) return F8_ERR_NULL;
  for (const void *x : {(const void *)table, (const void *)refs, (const void *)table_out, (const void *)refs_out, (const void *)moves, (const void *)info})
    if (!aligned_to(x, 4)) return F8_ERR_ALIGN;
  if (!aligned_to(workspace, 16)) return F8_ERR_ALIGN;
  if (workspace_bytes < f8_kv_compact_workspace_bytes(d->pages) || refs_out == refs) return F8_ERR_SHAPE;
  if (entries > 0 && table_out == table && d->out_ld != d->table_ld) return F8_ERR_SHAPE;       // (its rows would lie over one another's)
  int32_t *ws = static_cast<int32_t *>(workspace);
  const int blocks = (d->pages + BLOCK - 1) / BLOCK;
  const auto wgs_of = [](int64_t n) { return (int)((n + 1023) / 1024 < 2048 ? (n + 1023) / 1024 : 2048); };
  const int page_wgs = wgs_of(d->pages);
  const CompactParams p{table, refs, table_out, refs_out, moves, info, ws + d->pages, ws, d->table_ld, d->out_ld, entries, d->cols, d->pages, d->page_size,
                        blocks, page_wgs, FastDiv((uint32_t)(d->cols < 1 ? 1 : d->cols))};
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (d->pages <= SMALL_PAGES && entries <= SMALL_ENTRIES) {
    hipLaunchKernelGGL(compact_small_kernel, dim3(1), dim3(THREADS), 0, s, p);
    return launch_status();
  }
  hipLaunchKernelGGL(compact_count_kernel, dim3(blocks), dim3(256), 0, s, p);
  f8_status st = launch_status();
  if (st != F8_OK) return st;
  hipLaunchKernelGGL(compact_lists_kernel, dim3(blocks), dim3(256), 0, s, p);
  if ((st = launch_status()) != F8_OK) return st;
  hipLaunchKernelGGL(compact_apply_kernel, dim3(page_wgs + wgs_of(entries)), dim3(256), 0, s, p);
  return launch_status();
}

}  // extern "C"
