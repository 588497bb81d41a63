// Host-side helpers of the entry points on tokens: alignment tests, the check of a cache's layout, launch results.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../../include/f8.h"

namespace f8 {

inline bool aligned_to(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool real_type(int t) { return t == F8_F32 || t == F8_F16 || t == F8_BF16; }
inline size_t bytes_of(int t) { return t == F8_F32 ? 4 : t == F8_F16 || t == F8_BF16 ? 2 : 1; }
inline f8_status launch_status() { return hipGetLastError() == hipSuccess ? F8_OK : F8_ERR_DEVICE; }

// A grid of `blocks` workgroups whose extents stay below 2^32 threads: kernels number them by row_block() and turn away the surplus.
inline dim3 block_grid(int64_t blocks) {
  const int64_t x = blocks < (1 << 21) ? blocks : 1 << 21;
  return dim3((unsigned)x, (unsigned)((blocks + x - 1) / x));
}

inline f8_status check_kv_layout(const f8_kv_layout &c) {
  if (c.type != F8_S8 && c.type != F8_F16 && c.type != F8_BF16) return F8_ERR_DTYPE;
  if (c.pages < 1 || c.page_size < 1 || c.heads < 1 || c.dim < 16 || c.dim > 256 || c.dim % 16 != 0) return F8_ERR_SHAPE;
  if (c.page_stride < 0 || c.token_stride < 0 || c.head_stride < 0 || c.scale_page < 0 || c.scale_token < 0 || c.scale_head < 0) return F8_ERR_SHAPE;
  return F8_OK;
}

// The checks of the attention calls, before and behind the question whether there are requests at all.
inline f8_status check_attend(const f8_kv_layout &c, const f8_attend_desc &d) {
  const f8_status st = check_kv_layout(c);
  if (st != F8_OK) return st;
  if ((d.type != F8_F16 && d.type != F8_BF16) || (c.type != F8_S8 && c.type != d.type)) return F8_ERR_DTYPE;
  if (d.batch < 0 || d.batch > 65535 || d.q_heads < 1 || d.q_heads % c.heads != 0 || d.table_cols < 0 || d.max_len < 0) return F8_ERR_SHAPE;
  if ((int64_t)d.max_len > (int64_t)d.table_cols * c.page_size || d.max_len > 0x7fff0000) return F8_ERR_SHAPE;
  if (d.table_ld < d.table_cols || isnan(d.scale)) return F8_ERR_SHAPE;
  return F8_OK;
}
inline f8_status check_attend_pointers(const void *q, const void *k_cache, const void *v_cache, const float *k_scale, const float *v_scale,
                                       const int32_t *table, const int32_t *lens, const void *out, const f8_kv_layout &c, const f8_attend_desc &d) {
  const bool codes = c.type == F8_S8;
  if (!q || !k_cache || !v_cache || (!table && d.max_len > 0) || !lens || !out || (codes && (!k_scale || !v_scale))) return F8_ERR_NULL;
  const size_t e = bytes_of(c.type);
  if (!aligned_to(q, 2) || !aligned_to(out, 2) || !aligned_to(table, 4) || !aligned_to(lens, 4) || !aligned_to(k_scale, 4) || !aligned_to(v_scale, 4) ||
      !aligned_to(k_cache, 16) || !aligned_to(v_cache, 16) || c.page_stride * e % 16 || c.token_stride * e % 16 || c.head_stride * e % 16)
    return F8_ERR_ALIGN;
  return F8_OK;
}

// Tokens into codes [rows][ld] and scales, as f8_quant_tokens without a gate; columns cols .. pad - 1 of the codes become 0.
// The operands have passed the entry point's checks.
f8_status enqueue_quant_tokens(const void *x, int64_t ldx, int x_type, int8_t *codes, int64_t ld, int pad, float *scale, int rows, int cols,
                               hipStream_t s);

}  // namespace f8
