// Host-side helpers of the entry points on tokens: alignment tests, the check of a cache's layout, launch results.
#pragma once

#include <hip/hip_runtime.h>
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

// Tokens into codes [rows][ld] and scales, as f8_quant_tokens without a gate; columns cols .. pad - 1 of the codes become 0.
// The operands have passed the entry point's checks.
f8_status enqueue_quant_tokens(const void *x, int64_t ldx, int x_type, int8_t *codes, int64_t ld, int pad, float *scale, int rows, int cols,
                               hipStream_t s);

}  // namespace f8
