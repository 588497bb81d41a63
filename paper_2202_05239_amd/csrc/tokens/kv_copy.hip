// Copies of pages of a paged cache: the first n tokens of page src into page dst, for every (src, dst, n) of a list.
//
// A page is cut into runs that are contiguous in memory: all its tokens where a token's heads lie side by side and the tokens one behind the
// other, a head's tokens where heads lie outside the places of a page, otherwise a token, or a row of it.  A workgroup takes a piece
// of a page of one array (keys or values), 64 bytes a thread; the first piece takes the scales along.  Bound by HBM: every byte is
// read once and written once (2048 pages of 64 tokens, 8 heads of 128: 16 bits 215 us, 5.0 TB/s; 8 bits and scales 117 us, 4.7 TB/s).
#include "tokens_device.h"
#include "tokens_host.h"

namespace f8 {
namespace {

constexpr int THREADS = 256, DEPTH = 4, PIECE = THREADS * DEPTH;      // 16-byte units of a piece
constexpr int MOST_WGS = 8192;                                        // of an array; more pieces are taken in turn

// How a page's runs lie: one run, a run to a head, a run to a token, rows.
enum Form { ONE, HEADS, TOKENS, ROWS };

struct CopyParams {
  const int32_t *moves, *count;
  char *cache[2];
  float *scale[2];
  int64_t page, token, head;               // bytes
  int64_t spage, stoken, shead;            // elements
  int64_t items;                           // pieces of all moves
  int n, pages, page_size, heads;
  uint32_t row_units, token_units;         // of 16 bytes
  FastDiv pieces, run, by_heads, by_places;
};

template <int FORM>
__device__ __forceinline__ int64_t unit_at(const CopyParams &p, uint32_t u) {
  if constexpr (FORM == ONE) return (int64_t)u * 16;
  const uint32_t i = p.run.div(u);
  const int64_t in = (int64_t)(u - i * p.run.d) * 16;
  if constexpr (FORM == HEADS) return i * p.head + in;
  if constexpr (FORM == TOKENS) return i * p.token + in;
  const uint32_t t = p.by_heads.div(i);
  return t * p.token + (i - t * p.by_heads.d) * p.head + in;
}

template <int FORM>
__global__ __launch_bounds__(THREADS) void kv_copy_kernel(CopyParams p) {
  const int kv = blockIdx.y;
  const int n = p.count ? min(p.n, *p.count) : p.n;
  for (int64_t item = blockIdx.x; item < p.items; item += gridDim.x) {
    const int move = (int)p.pieces.div((uint32_t)item), piece = (int)item - move * (int)p.pieces.d;
    if (move >= n) break;
    const int32_t *m = p.moves + 3 * (int64_t)move;
    const int src = m[0], dst = m[1], tokens = min(m[2], p.page_size);
    if ((uint32_t)src >= (uint32_t)p.pages || (uint32_t)dst >= (uint32_t)p.pages || tokens <= 0 || src == dst) continue;
    const char *const from = p.cache[kv] + src * p.page;
    char *const to = p.cache[kv] + dst * p.page;
    // (a head's run is numbered by its whole page: units of it behind the last token are left out)
    const uint32_t units = (uint32_t)(FORM == HEADS ? p.page_size : tokens) * p.token_units;
    const uint32_t first = (uint32_t)piece * PIECE + threadIdx.x;
    int64_t at[DEPTH];
    v4i raw[DEPTH];
#pragma unroll
    for (int j = 0; j < DEPTH; ++j) {
      const uint32_t u = first + j * THREADS;
      bool real = u < units;
      if constexpr (FORM == HEADS) real = real && u - p.run.div(u) * p.run.d < (uint32_t)tokens * p.row_units;
      at[j] = real ? unit_at<FORM>(p, u) : -1;
      if (real) __builtin_memcpy(&raw[j], from + at[j], 16);
    }
#pragma unroll
    for (int j = 0; j < DEPTH; ++j)
      if (at[j] >= 0) *reinterpret_cast<v4i_any *>(to + at[j]) = raw[j];
    if (p.scale[kv] && piece == 0) {
      // neighbouring lanes take neighbouring scales: heads inside the places of a page or outside
      const float *const s = p.scale[kv] + src * p.spage;
      float *const d = p.scale[kv] + dst * p.spage;
      const bool inside = p.shead <= p.stoken;
      const uint32_t all = (uint32_t)(inside ? tokens : p.page_size) * p.heads;
      for (uint32_t i = threadIdx.x; i < all; i += THREADS) {
        uint32_t t, h;
        if (inside) t = p.by_heads.div(i), h = i - t * p.by_heads.d;
        else h = p.by_places.div(i), t = i - h * p.by_places.d;
        if (t < (uint32_t)tokens) d[t * p.stoken + h * p.shead] = s[t * p.stoken + h * p.shead];
      }
    }
  }
}

}  // namespace
}  // namespace f8

using namespace f8;

extern "C" f8_status f8_kv_copy(const int32_t *moves, const int32_t *count, void *k_cache, void *v_cache, float *k_scale, float *v_scale,
                                const f8_kv_layout *c, int n, void *stream) {
  if (!c) return F8_ERR_NULL;
  const f8_status st = check_kv_layout(*c);
  if (st != F8_OK) return st;
  if (n < 0) return F8_ERR_SHAPE;
  if (n == 0) return F8_OK;
  const bool codes = c->type == F8_S8;
  if (!moves || !k_cache || !v_cache || (codes && (!k_scale || !v_scale))) return F8_ERR_NULL;
  const int64_t e = (int64_t)bytes_of(c->type), row = c->dim * e;
  if (!aligned_to(moves, 4) || !aligned_to(count, 4) || !aligned_to(k_cache, e) || !aligned_to(v_cache, e) || !aligned_to(k_scale, 4) ||
      !aligned_to(v_scale, 4))
    return F8_ERR_ALIGN;
  const int64_t token = c->token_stride * e, head = c->head_stride * e, units = (int64_t)c->heads * row / 16, all = c->page_size * units;
  const int64_t pieces = (all + PIECE - 1) / PIECE, items = pieces * n;
  if (units > 0x7fffffff || all > 0x7fffffff - PIECE || (int64_t)c->page_size * c->heads > 0x7fffffff - THREADS || items > 0x7fffffff)
    return F8_ERR_UNSUPPORTED;
  const bool heads_side = head == row || c->heads == 1, tokens_side = token == row || c->page_size == 1;
  const Form form = heads_side && (token == c->heads * row || c->page_size == 1) ? ONE : tokens_side && c->page_size > 1 ? HEADS : heads_side ? TOKENS : ROWS;
  const int64_t run = form == HEADS ? c->page_size * row : form == TOKENS ? c->heads * row : row;
  const CopyParams p{moves, count, {static_cast<char *>(k_cache), static_cast<char *>(v_cache)}, {codes ? k_scale : nullptr, codes ? v_scale : nullptr},
                     c->page_stride * e, token, head, c->scale_page, c->scale_token, c->scale_head, items, n, c->pages, c->page_size, c->heads,
                     (uint32_t)(row / 16), (uint32_t)units, FastDiv((uint32_t)pieces), FastDiv((uint32_t)(run / 16)), FastDiv((uint32_t)c->heads), FastDiv((uint32_t)c->page_size)};
  const dim3 grid((unsigned)(items < MOST_WGS ? items : MOST_WGS), 2), block(THREADS);
  hipStream_t s = static_cast<hipStream_t>(stream);
  switch (form) {
    case ONE: hipLaunchKernelGGL(kv_copy_kernel<ONE>, grid, block, 0, s, p); break;
    case HEADS: hipLaunchKernelGGL(kv_copy_kernel<HEADS>, grid, block, 0, s, p); break;
    case TOKENS: hipLaunchKernelGGL(kv_copy_kernel<TOKENS>, grid, block, 0, s, p); break;
    default: hipLaunchKernelGGL(kv_copy_kernel<ROWS>, grid, block, 0, s, p);
  }
  return launch_status();
}
