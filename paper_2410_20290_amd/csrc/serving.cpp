// C entry points of specrej_serving.h: arguments are checked here, before any
// device work; the kernels' launchers take them from there.
#include <cmath>
#include <cstdint>

#include "checks.h"
#include "specrej_serving.h"

using namespace sr;

namespace {

// Bytes of a layer's block of keys or values of any cache type.
int64_t cache_bytes(int32_t cache, int32_t n_pages, int32_t n_kv_heads, int shift, int32_t head_dim) {
  if (cache != SR_FP4) return block_bytes(cache, n_pages, n_kv_heads, shift, head_dim);
  return (((int64_t)n_pages * n_kv_heads) << shift) * (head_dim * 17 / 32);
}

void check_cache(int32_t cache) {
  require(cache == SR_F32 || cache == SR_BF16 || cache == SR_FP4, "unknown cache type");
}

// One number for all rows, or 4 bytes each.
template <typename T>
PerRow<T> per_row(const T* each, T all) {
  require((reinterpret_cast<uintptr_t>(each) & 3) == 0, "a row's settings off a 4-byte boundary");
  return {each, all};
}

}  // namespace

extern "C" {

sr_status sr_page_append_norm(int32_t cache, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t rows,
                              int32_t lr, const float* qkv, const double* freqs, int32_t rot_dim, int32_t interleaved,
                              const float* q_gain, const float* k_gain, double eps, void* kpool, void* vpool,
                              int32_t page_tokens, int32_t n_pages, const int32_t* table, int32_t max_pages,
                              const int32_t* lens, const int32_t* n_new, float* q, void* stream) {
  return (sr_status)guarded([&] {
    check_cache(cache);
    check_heads(SR_F32, head_dim, n_heads, n_kv_heads);
    PageAppendNormArgs na;
    PageAppendArgs& a = na.a;
    a.shift = check_table(rows, max_pages, page_tokens, n_pages);
    require(lr >= 0 && rot_dim >= 0 && rot_dim <= head_dim && rot_dim % 8 == 0,
            "lr >= 0 and rot_dim 0 or a multiple of 8 up to head_dim");
    require(std::isfinite(eps) && eps >= 0.0, "eps must be finite and >= 0");
    supported((int64_t)rows * lr <= kMaxGroups, "2^24 tokens or more");
    if (rows == 0 || lr == 0) return;
    require(qkv && kpool && vpool && table && lens && q && (rot_dim == 0 || freqs), "NULL buffer");
    require(aligned16(qkv) && aligned16(q) && aligned16(kpool) && aligned16(vpool),
            "qkv, q, kpool and vpool must be 16-byte aligned");
    const int64_t tokens = (int64_t)rows * lr, block = cache_bytes(cache, n_pages, n_kv_heads, a.shift, head_dim);
    const Range in[] = {{qkv, tokens * (n_heads + 2 * n_kv_heads) * head_dim * 4}, {freqs, 4 * (int64_t)rot_dim},
                        {table, 4 * (int64_t)rows * max_pages}, {lens, 4 * (int64_t)rows}, {n_new, 4 * (int64_t)rows},
                        {q_gain, 4 * (int64_t)head_dim}, {k_gain, 4 * (int64_t)head_dim}};
    const Range out[] = {{q, tokens * n_heads * head_dim * 4}, {kpool, block}, {vpool, block}};
    check_apart(in, out);
    check_distinct(out);
    a.dtype = cache; a.hd = head_dim; a.hq = n_heads; a.hkv = n_kv_heads; a.rows = rows; a.lr = lr; a.qkv = qkv;
    a.freqs = freqs; a.rot = rot_dim; a.interleaved = interleaved != 0; a.kpool = kpool; a.vpool = vpool;
    a.n_pages = n_pages; a.table = table; a.max_pages = max_pages; a.lens = lens; a.n_new = n_new; a.q = q;
    na.q_gain = q_gain; na.k_gain = k_gain; na.eps = eps;
    page_append_norm(na, (hipStream_t)stream);
  });
}

sr_status sr_page_read(int32_t cache, int32_t dtype, int32_t head_dim, int32_t n_kv_heads, int32_t rows, int32_t lr,
                       const void* kpool, const void* vpool, int32_t page_tokens, int32_t n_pages,
                       const int32_t* table, int32_t max_pages, const int32_t* lens, const int32_t* n_new, void* k_out,
                       void* v_out, void* stream) {
  return (sr_status)guarded([&] {
    check_cache(cache);
    check_heads(dtype, head_dim, n_kv_heads, n_kv_heads);
    PageReadArgs a;
    a.shift = check_table(rows, max_pages, page_tokens, n_pages);
    require(lr >= 0, "bad lr");
    supported((int64_t)rows * lr <= kMaxGroups, "2^24 tokens or more");
    if (rows == 0 || lr == 0 || (!k_out && !v_out)) return;
    require(table && lens && (!k_out || kpool) && (!v_out || vpool), "NULL buffer");
    require(aligned16(kpool) && aligned16(vpool) && aligned16(k_out) && aligned16(v_out),
            "pools and outputs must be 16-byte aligned");
    const int64_t block = cache_bytes(cache, n_pages, n_kv_heads, a.shift, head_dim);
    const int64_t held = (int64_t)rows * lr * n_kv_heads * head_dim * (dtype == SR_BF16 ? 2 : 4);
    const Range in[] = {{kpool, block}, {vpool, block}, {table, 4 * (int64_t)rows * max_pages},
                        {lens, 4 * (int64_t)rows}, {n_new, 4 * (int64_t)rows}};
    const Range out[] = {{k_out, held}, {v_out, held}};
    check_apart(in, out);
    check_distinct(out);
    a.cache = cache; a.dtype = dtype; a.hd = head_dim; a.hkv = n_kv_heads; a.rows = rows; a.lr = lr; a.kpool = kpool;
    a.vpool = vpool; a.n_pages = n_pages; a.table = table; a.max_pages = max_pages; a.lens = lens; a.n_new = n_new;
    a.k_out = k_out; a.v_out = v_out;
    page_read(a, (hipStream_t)stream);
  });
}

size_t sr_paged_attention_fp4_scratch(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                                      int32_t rows, int32_t lr, int32_t page_tokens, int32_t max_pages, int32_t window,
                                      int32_t sinks, int32_t shared, int32_t max_len) {
  size_t n = 0;
  guarded([&] {
    PagedAttnArgs a;
    if (attention_args(dtype, head_dim, n_heads, n_kv_heads, rows, lr, page_tokens, 1, max_pages, window, sinks,
                       shared, max_len, &a))
      n = paged_attn_fp4_scratch(a);
  });
  return n;
}

sr_status sr_paged_attention_fp4(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t rows,
                                 int32_t lr, const float* q, const void* kpool, const void* vpool,
                                 int32_t page_tokens, int32_t n_pages, const int32_t* table, int32_t max_pages,
                                 const int32_t* lens, const int32_t* n_new, int32_t window, int32_t sinks,
                                 int32_t shared, int32_t max_len, void* out, float* scratch, size_t scratch_elems,
                                 void* stream) {
  return (sr_status)guarded([&] {
    PagedAttnArgs a;
    if (!attention_args(dtype, head_dim, n_heads, n_kv_heads, rows, lr, page_tokens, n_pages, max_pages, window, sinks,
                        shared, max_len, &a))
      return;
    require(q && kpool && vpool && table && lens && out, "NULL buffer");
    require(aligned16(q) && aligned16(kpool) && aligned16(vpool) && aligned16(out),
            "q, kpool, vpool and out must be 16-byte aligned");
    const size_t need = paged_attn_fp4_scratch(a);
    SR_REQUIRE(scratch_elems >= need && (need == 0 || scratch), SR_ERR_WORKSPACE_TOO_SMALL,
               "attention scratch too small: need " + std::to_string(need) + " floats");
    require(aligned16(scratch), "scratch must be 16-byte aligned");
    const int64_t heads = (int64_t)rows * lr * n_heads * head_dim;
    const int64_t block = cache_bytes(SR_FP4, n_pages, n_kv_heads, a.shift, head_dim);
    supported(block >> 36 == 0, "a layer's keys of 64 GB or more");   // (the kernels hold places in 16 bytes, 32 bits)
    const Range in[] = {{q, 4 * heads}, {kpool, block}, {vpool, block}, {table, 4 * (int64_t)rows * max_pages},
                        {lens, 4 * (int64_t)rows}, {n_new, 4 * (int64_t)rows}};
    const Range dst[] = {{out, heads * (dtype == SR_BF16 ? 2 : 4)}, {need ? scratch : nullptr, 4 * (int64_t)need}};
    check_apart(in, dst);
    check_distinct(dst);
    a.q = q; a.kpool = kpool; a.vpool = vpool; a.table = table; a.lens = lens; a.n_new = n_new; a.out = out;
    a.part = scratch;
    paged_attn_fp4(a, (hipStream_t)stream);
  });
}

size_t sr_sample_filtered_scratch(int32_t rows, int32_t vocab) {
  if (rows < 1 || rows > 1 << 20 || vocab < 1 || vocab > 262144) return 0;
  return sample_filtered_scratch(rows, vocab);
}

sr_status sr_sample_filtered(int32_t dtype, const void* logits, int64_t row_stride, int32_t rows, int32_t vocab,
                             const float* temperature, float temperature_all, const int32_t* top_k, int32_t top_k_all,
                             const float* top_p, float top_p_all, const float* min_p, float min_p_all,
                             const uint32_t* random, int64_t random_stride, int32_t* token, float* logprob,
                             int32_t* kept, uint32_t* scratch, size_t scratch_elems, void* stream) {
  return (sr_status)guarded([&] {
    require(dtype == SR_F32 || dtype == SR_BF16, "unknown dtype");
    require(rows >= 0 && vocab >= 1 && row_stride >= vocab, "bad rows / vocab / row_stride");
    supported(vocab <= 262144, "vocab above 262144");
    supported(row_stride <= (int64_t)1 << 40, "row_stride above 2^40");
    supported(rows <= 1 << 20, "at most 2^20 rows");
    require(random_stride >= 0 && random_stride <= (int64_t)1 << 40, "bad random_stride");
    FilteredArgs a;
    a.temperature = per_row(temperature, temperature_all);
    a.top_k = per_row(top_k, top_k_all);
    a.top_p = per_row(top_p, top_p_all);
    a.min_p = per_row(min_p, min_p_all);
    if (rows == 0) return;
    require(logits && random, "NULL buffer");
    const int es = dtype == SR_BF16 ? 2 : 4;
    require((reinterpret_cast<uintptr_t>(logits) & (es - 1)) == 0, "logits off an element boundary");
    const size_t need = sample_filtered_scratch(rows, vocab);
    SR_REQUIRE(scratch_elems >= need && (need == 0 || scratch), SR_ERR_WORKSPACE_TOO_SMALL,
               "draw scratch too small: need " + std::to_string(need) + " elements");
    require(aligned16(scratch), "scratch must be 16-byte aligned");
    const int64_t nr = 4 * (int64_t)rows;
    const Range in[] = {{logits, ((rows - 1) * row_stride + vocab) * es}, {temperature, nr}, {top_k, nr}, {top_p, nr},
                        {min_p, nr}, {random, 4 * ((rows - 1) * random_stride + 1)}};
    const Range out[] = {{token, nr}, {logprob, nr}, {kept, nr}, {need ? scratch : nullptr, 4 * (int64_t)need}};
    check_apart(in, out);
    check_distinct(out);
    a.dtype = dtype; a.logits = logits; a.row_stride = row_stride; a.rows = rows; a.vocab = vocab; a.random = random;
    a.random_stride = random_stride; a.token = token; a.logprob = logprob; a.kept = kept; a.scratch = scratch;
    sample_filtered(a, (hipStream_t)stream);
  });
}

}  // extern "C"
