// Checks of arguments that the C entry points over pages share: all of them run
// before any device work and throw.
#pragma once

#include <cstdint>

#include "common.h"
#include "kernels.h"
#include "paged.h"
#include "specrej_ops.h"

namespace sr {

inline void require(bool cond, const char* text) { SR_REQUIRE(cond, SR_ERR_INVALID_ARG, text); }
inline void supported(bool cond, const char* text) { SR_REQUIRE(cond, SR_ERR_UNSUPPORTED, text); }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

inline bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uint64_t)nb && y < x + (uint64_t)na;
}

// The sizes of a table and its pool; returns log2(page_tokens).
inline int check_table(int32_t rows, int32_t max_pages, int32_t page_tokens, int32_t n_pages) {
  require(rows >= 0 && max_pages >= 1 && n_pages >= 1, "bad rows / max_pages / n_pages");
  supported(rows <= kPageMaxRows && max_pages <= kPageMaxPerRow && n_pages <= kPageMaxPages,
            "at most 4096 rows, 65536 pages a row and 2^20 pages");
  const int shift = page_shift(page_tokens);
  supported(shift >= 0, "page_tokens must be 16, 32, 64, 128 or 256");
  return shift;
}

inline PagePool check_pool(void* pool, int64_t block_elems, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim,
                           int32_t elem_bytes, int shift, int32_t n_pages) {
  require(pool != nullptr && aligned16(pool), "pool is NULL or off a 16-byte boundary");
  require(n_layers >= 1 && n_layers <= 65536 && n_kv_heads >= 1 && n_kv_heads <= 65536 && head_dim >= 1 &&
              head_dim <= 65536,
          "bad shape");
  require(elem_bytes == 1 || elem_bytes == 2 || elem_bytes == 4, "elem_bytes must be 1, 2 or 4");
  if (elem_bytes == 1)
    supported(head_dim == 17 || head_dim == 34 || head_dim == 68, "pages of 4 bits hold 17, 34 or 68 bytes a token");
  else
    supported((int64_t)head_dim * elem_bytes % 16 == 0, "KV row must be a 16-byte multiple");
  supported(block_elems * elem_bytes % 16 == 0, "block must be a 16-byte multiple");
  const int64_t page = ((int64_t)n_kv_heads * head_dim) << shift;
  supported(page <= (int64_t)1 << 30, "pages above 2^30 elements");
  require(page * n_pages <= block_elems, "pool blocks too small for n_pages");
  supported(block_elems <= ((int64_t)1 << 50) / n_layers, "pool too large");
  return {pool, block_elems * elem_bytes, n_layers, n_kv_heads, head_dim * elem_bytes, shift, n_pages, elem_bytes == 1};
}

// In place or apart.
inline void check_in_out(const int32_t* in, const int32_t* out, int64_t n) {
  require(in == out || !overlap(in, 4 * n, out, 4 * n), "an output overlaps its input without being it");
}

struct Range {
  const void* p;
  int64_t bytes;
};
// Every pair of `a` and `b` apart.
template <int NA, int NB>
inline void check_apart(const Range (&a)[NA], const Range (&b)[NB]) {
  for (const Range& x : a)
    for (const Range& y : b) require(!x.p || !y.p || !overlap(x.p, x.bytes, y.p, y.bytes), "buffers overlap");
}
template <int N>
inline void check_distinct(const Range (&a)[N]) {
  for (int i = 0; i < N; ++i)
    for (int j = 0; j < i; ++j)
      require(!a[i].p || !a[j].p || !overlap(a[i].p, a[i].bytes, a[j].p, a[j].bytes), "outputs overlap");
}

inline void check_heads(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads) {
  require(dtype == SR_F32 || dtype == SR_BF16, "unknown dtype");
  supported(head_dim == 32 || head_dim == 64 || head_dim == 128, "head_dim must be 32, 64 or 128");
  require(n_heads >= 1 && n_kv_heads >= 1 && n_heads % n_kv_heads == 0, "bad head counts");
  supported(n_heads <= 4096, "at most 4096 query heads");
}

inline bool attention_args(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t rows,
                           int32_t lr, int32_t page_tokens, int32_t n_pages, int32_t max_pages, int32_t window,
                           int32_t sinks, int32_t shared, int32_t max_len, PagedAttnArgs* a) {
  check_heads(dtype, head_dim, n_heads, n_kv_heads);
  supported(n_heads / n_kv_heads <= 16, "at most 16 query heads per KV head");
  a->shift = check_table(rows, max_pages, page_tokens, n_pages);
  require(lr >= 0 && window >= 0 && sinks >= 0 && shared >= 0 && max_len >= 1, "bad lr / window / sinks / shared / max_len");
  supported((int64_t)rows * lr * n_heads <= (int64_t)1 << 28, "more than 2^28 queries");
  a->dtype = dtype; a->hd = head_dim; a->hq = n_heads; a->hkv = n_kv_heads; a->rows = rows; a->lr = lr;
  a->n_pages = n_pages; a->max_pages = max_pages; a->window = window; a->sinks = sinks; a->shared = shared;
  a->max_len = max_len;
  return rows > 0 && lr > 0;
}

// Byte ranges of a layer's blocks of keys or values (elements of dtype).
inline int64_t block_bytes(int32_t dtype, int32_t n_pages, int32_t n_kv_heads, int shift, int32_t head_dim) {
  return (((int64_t)n_pages * n_kv_heads * head_dim) << shift) * (dtype == SR_BF16 ? 2 : 4);
}

}  // namespace sr
