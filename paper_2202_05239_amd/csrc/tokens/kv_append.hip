// New tokens' keys and values into a paged cache of 8 or 16 bits: the row of token t, head h goes to slot slots[t], that is page
// slot / page_size, place slot % page_size.  8-bit caches hold a row's codes and its scale (tokens_device.h).  Negative slots and
// slots past the last page are skipped.  16 lanes take a row; a step's few rows are a chain of two memory latencies (slot and row at
// once, then the store): 64 tokens of 8 heads 4.6 us.
#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

constexpr int LANES = 16;            // of a row: one 16-byte load each where a head has 128 dimensions of 16 bits

struct AppendParams {
  const void *x[2];
  const int64_t *slots;
  void *cache[2];
  float *scale[2];
  int64_t xt[2], xh[2];
  int64_t page, token, head, spage, stoken, shead, slot_count;
  int rows, dim;
  FastDiv heads, page_size;
};

template <typename T, typename C, int NV>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendParams p) {
  typedef RowMap<LANES, NV> Map;
  const int64_t row = row_block() * (256 / LANES) + (int)threadIdx.x / LANES;
  const int l = (int)threadIdx.x % LANES, kv = blockIdx.z;
  if (row >= p.rows) return;
  const int token = (int)p.heads.div((uint32_t)row), head = (int)row - token * (int)p.heads.d;
  const int64_t slot = p.slots[token];
  const bool there = slot >= 0 && slot < p.slot_count;
  float v[NV][8];
  const T *x = static_cast<const T *>(p.x[kv]) + token * p.xt[kv] + head * p.xh[kv];
#pragma unroll
  for (int i = 0; i < NV; ++i) load_piece<T, Map>(x, i, l, p.dim, v[i]);
  // (a division in 64 bits is half of this kernel: only for slots beyond 31)
  const int64_t page = !there ? 0 : slot <= 0x7fffffff ? (int64_t)p.page_size.div((uint32_t)slot) : slot / (int64_t)p.page_size.d;
  const int64_t place = there ? slot - page * (int64_t)p.page_size.d : 0;
  C *to = static_cast<C *>(p.cache[kv]) + page * p.page + place * p.token + head * p.head;
  if constexpr (sizeof(C) == 1) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, magnitude(v[i][j]));
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    const TokenScale s = token_scale(__uint_as_float(top));
    if (!there) return;
    lift(v, s);
    if (l == 0) p.scale[kv][page * p.spage + place * p.stoken + head * p.shead] = s.scale;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      int q[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) q[j] = code_of(v[i][j], s);
      store_codes<Map>(reinterpret_cast<int8_t *>(to), i, l, p.dim, q);
    }
  } else {
    if (!there) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) store_piece<C, Map>(to, i, l, p.dim, v[i]);
  }
}

template <typename T, typename C>
f8_status launch(const AppendParams &p, hipStream_t s) {
  dim3 grid = block_grid(((int64_t)p.rows + 256 / LANES - 1) / (256 / LANES));
  const dim3 block(256);
  grid.z = 2;
  static_assert(RowMap<LANES, 2>::most == 256, "the most dimensions of a head");
  if (p.dim <= RowMap<LANES, 1>::most) hipLaunchKernelGGL((kv_append_kernel<T, C, 1>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((kv_append_kernel<T, C, 2>), grid, block, 0, s, p);
  return launch_status();
}

template <typename T>
f8_status launch_cache(const AppendParams &p, int cache, hipStream_t s) {
  return cache == F8_S8 ? launch<T, int8_t>(p, s) : cache == F8_F16 ? launch<T, f16>(p, s) : launch<T, bf16>(p, s);
}

}  // namespace
}  // namespace f8

using namespace f8;

extern "C" f8_status f8_kv_append(const void *k, const void *v, const int64_t *slots, void *k_cache, void *v_cache, float *k_scale,
                                  float *v_scale, const f8_kv_layout *c, const f8_kv_append_desc *d, void *stream) {
  if (!c || !d) return F8_ERR_NULL;
  const f8_status st = check_kv_layout(*c);
  if (st != F8_OK) return st;
  if (!real_type(d->type)) return F8_ERR_DTYPE;
  if (d->tokens < 0 || (int64_t)d->tokens * c->heads > 0x7fffffffLL) return F8_ERR_SHAPE;
  if (d->tokens == 0) return F8_OK;
  const bool codes = c->type == F8_S8;
  if (!k || !v || !slots || !k_cache || !v_cache || (codes && (!k_scale || !v_scale))) return F8_ERR_NULL;
  const size_t e = bytes_of(d->type), o = bytes_of(c->type);
  if (!aligned_to(k, e) || !aligned_to(v, e) || !aligned_to(slots, 8) || !aligned_to(k_cache, o) || !aligned_to(v_cache, o) ||
      !aligned_to(k_scale, 4) || !aligned_to(v_scale, 4))
    return F8_ERR_ALIGN;
  const AppendParams p{{k, v}, slots, {k_cache, v_cache}, {k_scale, v_scale}, {d->k_token, d->v_token}, {d->k_head, d->v_head},
                       c->page_stride, c->token_stride, c->head_stride, c->scale_page, c->scale_token, c->scale_head,
                       (int64_t)c->pages * c->page_size, d->tokens * c->heads, c->dim, FastDiv((uint32_t)c->heads), FastDiv((uint32_t)c->page_size)};
  hipStream_t s = static_cast<hipStream_t>(stream);
  return d->type == F8_F32 ? launch_cache<float>(p, c->type, s)
                           : d->type == F8_F16 ? launch_cache<f16>(p, c->type, s) : launch_cache<bf16>(p, c->type, s);
}
