// The pages of a cache as its block tables and a count of holders per page see them: forking requests and compacting the pool.  Integers
// only; what has to be copied in the cache comes out as a list for f8_kv_copy.
//
// A page is free where its count is not positive.  New pages are the free ones of the lowest index, handed out in the order of the
// requests, so a result depends on its inputs alone: the only atomics add to counts or take a minimum.
#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

constexpr int WAVES = 16, THREADS = 64 * WAVES;

// What other workgroups' or this one's atomics have written is read where they wrote it, behind the first-level cache.
__device__ __forceinline__ int seen(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void put(int32_t *p, int v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void add(int32_t *p, int v) { __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
// Between phases of one workgroup that hand on memory.
__device__ __forceinline__ void phase() {
  __threadfence();
  __syncthreads();
}

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

struct ForkParams {
  const int32_t *parent, *table, *lens, *refs;
  int32_t *table_out, *lens_out, *refs_out;
  int64_t *slots;
  int32_t *moves, *info;
  // workspace: of each page the lowest of those that write behind it, and how many they are; the new pages; of each request the place of
  // its first one among them (twice that, and 1 more where it is a copy); how many there are
  int32_t *lowest, *writers, *fresh, *at, *found;
  int64_t table_ld, out_ld;
  int batch, cols, pages, grow;
  FastDiv page_size;
};

__device__ __forceinline__ int pages_of(const ForkParams &p, int tokens) { return tokens > 0 ? (int)p.page_size.div((uint32_t)tokens - 1) + 1 : 0; }

struct Child {                               // what a request is to be: the parent's row, its tokens and pages
  int row, tokens, pages;
  __device__ __forceinline__ Child(const ForkParams &p, int b) {
    row = p.parent[b];
    const bool live = (uint32_t)row < (uint32_t)p.batch;
    const int most = p.cols * (int)p.page_size.d;
    tokens = live ? min(max(p.lens[row], 0), most) : 0;
    pages = pages_of(p, tokens);
    if (!live) row = -1;
  }
};

// A thread's place among `threads` that share a phase.
struct Share {
  int64_t first, step;
};

// Rows of the parents, counts as they were, lists without entries.
__device__ __forceinline__ void fork_rows(const ForkParams &p, int b, Share s) {
  const Child c(p, b);
  const int32_t *from = p.table + (int64_t)max(c.row, 0) * p.table_ld;
  int32_t *to = p.table_out + b * p.out_ld;
  for (int64_t i = s.first; i < p.cols; i += s.step) put(to + i, i < c.pages ? from[i] : -1);
}
__device__ __forceinline__ void fork_counts(const ForkParams &p, Share s) {
  for (int64_t i = s.first; i < p.pages; i += s.step) put(p.refs_out + i, p.refs[i]);
  for (int64_t i = s.first; i < 3 * (int64_t)p.batch; i += s.step) p.moves[i] = i % 3 == 2 ? 0 : -1;
}

// A page's holders: each child holds what its parent held.
__device__ __forceinline__ void fork_hold(const ForkParams &p, int b, int children, Share s) {
  if (children == 1) return;
  const int n = min(max(p.lens[b], 0), p.cols * (int)p.page_size.d);
  const int used = pages_of(p, n);
  for (int64_t i = s.first; i < used; i += s.step) {
    const int page = p.table[b * p.table_ld + i];
    if ((uint32_t)page < (uint32_t)p.pages) add(p.refs_out + page, children - 1);
  }
}

// Who copies, who gets which new page.  One workgroup.
__device__ __forceinline__ void fork_assign(const ForkParams &p) {
  __shared__ int lds[WAVES][2], moved;
  const int page_size = (int)p.page_size.d;
  // requests that will write into a page that is not full: the lowest of them keeps it, if all that hold it write
  auto tail_of = [&](int b) {
    const Child c(p, b);
    const int full = (int)p.page_size.div((uint32_t)c.tokens);
    if (p.grow == 0 || c.tokens == full * page_size) return -1;
    const int page = p.table[c.row * p.table_ld + full];
    return (uint32_t)page < (uint32_t)p.pages ? page : -1;
  };
  if (threadIdx.x == 0) moved = 0;
  for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
    const int page = tail_of(b);
    if (page >= 0) put(p.lowest + page, 0x7fffffff), put(p.writers + page, 0);
  }
  phase();
  for (int b = threadIdx.x; b < p.batch; b += blockDim.x) {
    const int page = tail_of(b);
    if (page >= 0) {
      __hip_atomic_fetch_min(p.lowest + page, b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      add(p.writers + page, 1);
    }
  }
  phase();
  // places among the new pages, and how many of those there are
  int wanted = 0, beyond = 0;
  for (int b0 = 0; b0 < p.batch; b0 += blockDim.x) {
    const int b = b0 + (int)threadIdx.x;
    int v[2] = {0, 0}, before[2], all[2];
    bool copies = false;
    if (b < p.batch) {
      const Child c(p, b);
      const int page = tail_of(b);
      copies = page >= 0 && !(seen(p.refs_out + page) == seen(p.writers + page) && seen(p.lowest + page) == b);
      if (c.row >= 0) {
        const int64_t need = ((int64_t)c.tokens + p.grow + page_size - 1) / page_size;
        v[0] = (int)min(need, (int64_t)p.cols) - c.pages + copies, v[1] = (int)(need - min(need, (int64_t)p.cols));
      }
    }
    scan<2>(v, before, all, lds);
    if (b < p.batch) put(p.at + b, 2 * (wanted + before[0]) + copies);
    wanted += all[0], beyond += all[1];
  }
  // the free pages of the lowest index, 4 to a thread at a time
  int found = 0;
  for (int64_t i0 = 0; i0 < p.pages && found < wanted; i0 += 4 * blockDim.x) {
    const int64_t i = i0 + 4 * (int)threadIdx.x;
    int free[4], v[1] = {0}, before[1], all[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      free[j] = i + j < p.pages && seen(p.refs_out + i + j) <= 0;
      v[0] += free[j];
    }
    scan<1>(v, before, all, reinterpret_cast<int(*)[1]>(lds));
    int place = found + before[0];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (free[j]) {
        if (place < wanted) put(p.fresh + place, (int)(i + j));
        ++place;
      }
    found += all[0];
  }
  found = min(found, wanted);
  phase();
  for (int i = threadIdx.x; i < found; i += blockDim.x) put(p.refs_out + seen(p.fresh + i), 1);
  if (threadIdx.x == 0) put(p.found, found);
  phase();
  // the copies, one behind the other (those that no page was left for are the last)
  int copied = 0;
  for (int b0 = 0; b0 < p.batch; b0 += blockDim.x) {
    const int b = b0 + (int)threadIdx.x, at = b < p.batch ? seen(p.at + b) : 0;
    int v[1] = {at & 1}, before[1], all[1];
    scan<1>(v, before, all, reinterpret_cast<int(*)[1]>(lds));
    if (v[0]) {
      const Child c(p, b);
      const int from = tail_of(b), to = (at >> 1) < found ? seen(p.fresh + (at >> 1)) : -1;
      add(p.refs_out + from, -1);
      if (to >= 0) {
        int32_t *m = p.moves + 3 * (int64_t)(copied + before[0]);
        m[0] = from, m[1] = to, m[2] = c.tokens - (int)p.page_size.div((uint32_t)c.tokens) * page_size;
        atomicMax(&moved, copied + before[0] + 1);
      }
    }
    copied += all[0];
  }
  __syncthreads();
  if (threadIdx.x == 0) p.info[0] = moved, p.info[1] = wanted - found + beyond;
}

// New entries of a request's row, where its new tokens go, its length.
__device__ __forceinline__ void fork_grow(const ForkParams &p, int b, Share s) {
  const Child c(p, b);
  const int page_size = (int)p.page_size.d, at = seen(p.at + b), copies = at & 1, full = (int)p.page_size.div((uint32_t)c.tokens);
  const int64_t most = (int64_t)p.cols * page_size, upto = min((int64_t)c.tokens + p.grow, most);
  const int need = c.row < 0 ? 0 : (int)((upto + page_size - 1) / page_size);
  int32_t *row = p.table_out + b * p.out_ld;
  const int found = seen(p.found);
  auto entry = [&](int col) {                  // of a new page, or of the last one that is there
    if (col < c.pages && !copies) return p.table[c.row * p.table_ld + col];
    const int i = (at >> 1) + (col < c.pages ? 0 : copies + col - c.pages);
    return i < found ? seen(p.fresh + i) : -1;
  };
  for (int64_t i = (copies ? full : c.pages) + s.first; i < need; i += s.step) put(row + i, entry((int)i));
  for (int64_t j = s.first; j < p.grow; j += s.step) {
    int64_t slot = -1;
    if (c.row >= 0 && c.tokens + j < most) {
      const int t = c.tokens + (int)j, col = (int)p.page_size.div((uint32_t)t), page = entry(col);
      if ((uint32_t)page < (uint32_t)p.pages) slot = (int64_t)page * page_size + (t - col * page_size);
    }
    p.slots[(int64_t)b * p.grow + j] = slot;
  }
  if (s.first == 0) p.lens_out[b] = c.row < 0 ? 0 : (int)upto;
}

// All of it in one workgroup.
__global__ __launch_bounds__(THREADS) void fork_small_kernel(ForkParams p) {
  __shared__ int children[THREADS];
  const Share all{threadIdx.x, THREADS}, wave{threadIdx.x & 63, 64};
  const int w = threadIdx.x >> 6;
  children[threadIdx.x] = 0;
  fork_counts(p, all);
  for (int b = w; b < p.batch; b += WAVES) fork_rows(p, b, wave);
  phase();
  for (int b = threadIdx.x; b < p.batch; b += THREADS)
    if ((uint32_t)p.parent[b] < (uint32_t)p.batch) atomicAdd(&children[p.parent[b]], 1);
  __syncthreads();
  for (int b = w; b < p.batch; b += WAVES) fork_hold(p, b, children[b], wave);
  phase();
  fork_assign(p);
  phase();
  for (int b = w; b < p.batch; b += WAVES) fork_grow(p, b, wave);
}

// The same phases as launches of many workgroups (256 threads each, but for the assignment).
__global__ __launch_bounds__(256) void fork_rows_kernel(ForkParams p) {
  const int64_t grid = (int64_t)gridDim.x * 256;
  fork_counts(p, Share{(int64_t)blockIdx.x * 256 + threadIdx.x, grid});
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) fork_rows(p, b, Share{threadIdx.x, 256});
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
    fork_hold(p, b, children, Share{threadIdx.x, 256});
    __syncthreads();
  }
}
__global__ __launch_bounds__(THREADS) void fork_assign_kernel(ForkParams p) { fork_assign(p); }
__global__ __launch_bounds__(256) void fork_grow_kernel(ForkParams p) {
  for (int b = blockIdx.x; b < p.batch; b += gridDim.x) fork_grow(p, b, Share{threadIdx.x, 256});
}

// ---- compaction ----

constexpr int PER = 16, BLOCK = 256 * PER;   // pages of a thread and of a workgroup

struct CompactParams {
  const int32_t *table, *refs;
  int32_t *table_out, *refs_out, *moves, *info;
  int32_t *counts, *rank;                   // workspace: pages in use of each block; of a page that goes, and of a hole, its place in the list
  int64_t table_ld, out_ld, entries;
  int cols, pages, page_size, blocks;
  FastDiv by_cols;
};

__global__ __launch_bounds__(256) void compact_count_kernel(CompactParams p) {
  __shared__ int lds[4][1];
  int v[1] = {0}, before[1], all[1];
  // (a page index may pass 31 bits by a block)
  const int64_t base = (int64_t)blockIdx.x * BLOCK;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const int64_t i = base + j * 256 + threadIdx.x;
    v[0] += i < p.pages && p.refs[i] > 0;
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
  int used, front, front_of_border, dummy;
  block_sums(p, blockIdx.x, used, front, lds);
  // pages in use in front of the border: those of the blocks before it, and of its own block
  const int border = used / BLOCK;
  block_sums(p, border, dummy, front_of_border, lds);
  {
    int v[2] = {0, 0}, before[2], all[2];
    for (int i = border * BLOCK + (int)threadIdx.x; i < used; i += 256) v[0] += p.refs[i] > 0;
    scan<2>(v, before, all, lds);
    front_of_border += all[0];
  }
  const int moved = used - front_of_border;
  const int64_t base = (int64_t)blockIdx.x * BLOCK + (int)threadIdx.x * PER;
  int held[PER], v[2] = {0, 0}, before[2], all[2];
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    held[j] = base + j < p.pages && p.refs[base + j] > 0;
    v[0] += held[j];
  }
  scan<2>(v, before, all, lds);
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

__global__ __launch_bounds__(256) void compact_apply_kernel(CompactParams p) {
  const int used = p.info[1];
  const int64_t step = (int64_t)gridDim.x * 256, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
  for (int64_t i = first; i < p.pages; i += step) {
    int n = 0;
    if (i < used) {
      n = p.refs[i];
      if (n <= 0) n = p.refs[p.moves[3 * (int64_t)p.rank[i]]];
    }
    p.refs_out[i] = n;
  }
  for (int64_t i = first; i < p.entries; i += step) {
    const int64_t row = i <= 0x7fffffff ? (int64_t)p.by_cols.div((uint32_t)i) : i / p.cols;
    const int col = (int)(i - row * p.cols);
    int e = p.table[row * p.table_ld + col];
    if (e >= used && e < p.pages && p.refs[e] > 0) e = p.moves[3 * (int64_t)p.rank[e] + 1];
    p.table_out[row * p.out_ld + col] = e;
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
  if ((int64_t)d->cols * d->page_size > 0x7fff0000) return F8_ERR_SHAPE;
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
  const ForkParams p{parent, table, lens, refs, table_out, lens_out, refs_out, slots, moves, info, ws, ws + n, ws + 2 * n, ws + 3 * n, ws + 3 * n + d->batch,
                     d->table_ld, d->out_ld, d->batch, d->cols, d->pages, d->grow, FastDiv((uint32_t)d->page_size)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t entries = (int64_t)d->batch * d->cols;
  if (d->batch <= THREADS && entries <= 16384 && d->pages <= 16384 && (int64_t)d->batch * d->grow <= 4096) {
    hipLaunchKernelGGL(fork_small_kernel, dim3(1), dim3(THREADS), 0, s, p);
    return launch_status();
  }
  const int rows = d->batch < 2048 ? d->batch : 2048, counts = (d->pages + 1023) / 1024 < 2048 ? (d->pages + 1023) / 1024 : 2048;
  hipLaunchKernelGGL(fork_rows_kernel, dim3(rows > counts ? rows : counts), dim3(256), 0, s, p);
  f8_status st = launch_status();
  if (st != F8_OK) return st;
  hipLaunchKernelGGL(fork_hold_kernel, dim3(rows), dim3(256), 0, s, p);
  if ((st = launch_status()) != F8_OK) return st;
  hipLaunchKernelGGL(fork_assign_kernel, dim3(1), dim3(THREADS), 0, s, p);
  if ((st = launch_status()) != F8_OK) return st;
  hipLaunchKernelGGL(fork_grow_kernel, dim3(rows), dim3(256), 0, s, p);
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
  int32_t *ws = static_cast<int32_t *>(workspace);
  const int blocks = (d->pages + BLOCK - 1) / BLOCK;
  const CompactParams p{table, refs, table_out, refs_out, moves, info, ws + d->pages, ws, d->table_ld, d->out_ld, entries, d->cols, d->pages, d->page_size,
                        blocks, FastDiv((uint32_t)(d->cols < 1 ? 1 : d->cols))};
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(compact_count_kernel, dim3(blocks), dim3(256), 0, s, p);
  f8_status st = launch_status();
  if (st != F8_OK) return st;
  hipLaunchKernelGGL(compact_lists_kernel, dim3(blocks), dim3(256), 0, s, p);
  if ((st = launch_status()) != F8_OK) return st;
  const int64_t work = (entries > d->pages ? entries : d->pages), wgs = (work + 1023) / 1024;
  hipLaunchKernelGGL(compact_apply_kernel, dim3((unsigned)(wgs < 2048 ? wgs : 2048)), dim3(256), 0, s, p);
  return launch_status();
}

}  // extern "C"
