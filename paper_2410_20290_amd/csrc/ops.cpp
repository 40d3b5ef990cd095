// C entry points of specrej_ops.h: arguments are checked here, before any
// device work; the kernels' launchers take them from there.
#include <cmath>
#include <cstdint>

#include "checks.h"

using namespace sr;

extern "C" {

sr_status sr_page_fork(const int32_t* table, const int32_t* lens, int32_t rows, int32_t max_pages,
                       const int32_t* parent, int32_t new_rows, int32_t page_tokens, int32_t n_pages, int32_t window,
                       int32_t sinks, int32_t* table_out, int32_t* lens_out, int32_t* refs_out, void* stream) {
  return (sr_status)guarded([&] {
    PageForkArgs a;
    a.shift = check_table(rows, max_pages, page_tokens, n_pages);
    check_table(new_rows, max_pages, page_tokens, n_pages);
    require(window >= 0 && sinks >= 0, "bad window / sinks");
    require(rows == 0 || (table && lens), "NULL buffer");
    require(refs_out && (new_rows == 0 || (parent && table_out && lens_out)), "NULL buffer");
    const int64_t nt = 4 * (int64_t)rows * max_pages, no = 4 * (int64_t)new_rows * max_pages;
    const Range in[] = {{table, nt}, {lens, 4 * (int64_t)rows}, {parent, 4 * (int64_t)new_rows}};
    const Range out[] = {{table_out, no}, {lens_out, 4 * (int64_t)new_rows}, {refs_out, 4 * (int64_t)n_pages}};
    check_apart(in, out);
    check_distinct(out);
    a.table = table; a.lens = lens; a.rows = rows; a.max_pages = max_pages; a.parent = parent; a.new_rows = new_rows;
    a.n_pages = n_pages; a.window = window; a.sinks = sinks; a.table_out = table_out; a.lens_out = lens_out;
    a.refs_out = refs_out;
    page_fork(a, (hipStream_t)stream);
  });
}

size_t sr_page_reserve_scratch(int32_t rows, int32_t max_pages, int32_t n_pages) {
  if (rows < 0 || max_pages < 1 || n_pages < 1) return 0;
  return page_reserve_scratch(rows, max_pages, n_pages);
}

sr_status sr_page_reserve(void* pool, int64_t block_elems, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim,
                          int32_t elem_bytes, int32_t page_tokens, int32_t n_pages, const int32_t* table,
                          const int32_t* lens, const int32_t* refs, int32_t rows, int32_t max_pages,
                          const int32_t* n_add, int32_t n_add_all, int32_t* table_out, int32_t* lens_out,
                          int32_t* refs_out, int32_t* granted, int32_t* info, int32_t* scratch, size_t scratch_elems,
                          void* stream) {
  return (sr_status)guarded([&] {
    PageReserveArgs a;
    const int shift = check_table(rows, max_pages, page_tokens, n_pages);
    a.p = check_pool(pool, block_elems, n_layers, n_kv_heads, head_dim, elem_bytes, shift, n_pages);
    require(refs && refs_out && info, "NULL buffer");
    require(rows == 0 || (table && lens && table_out && lens_out && granted), "NULL buffer");
    const size_t need = page_reserve_scratch(rows, max_pages, n_pages);
    SR_REQUIRE(scratch && scratch_elems >= need, SR_ERR_WORKSPACE_TOO_SMALL,
               "reserve scratch too small: need " + std::to_string(need) + " elements");
    const int64_t nt = (int64_t)rows * max_pages, nr = rows;
    check_in_out(table, table_out, nt);
    check_in_out(lens, lens_out, nr);
    check_in_out(refs, refs_out, n_pages);
    const Range out[] = {{table_out, 4 * nt}, {lens_out, 4 * nr},  {refs_out, 4 * (int64_t)n_pages},
                         {granted, 4 * nr},   {info, 16},          {scratch, 4 * (int64_t)need},
                         {pool, 2 * n_layers * a.p.block_bytes}};
    check_distinct(out);
    const Range table_in[] = {{table, 4 * nt}}, lens_in[] = {{lens, 4 * nr}}, refs_in[] = {{refs, 4 * (int64_t)n_pages}};
    const Range add_in[] = {{n_add, 4 * nr}};
    const Range not_table[] = {out[1], out[2], out[3], out[4], out[5], out[6]};
    const Range not_lens[] = {out[0], out[2], out[3], out[4], out[5], out[6]};
    const Range not_refs[] = {out[0], out[1], out[3], out[4], out[5], out[6]};
    check_apart(table_in, not_table);
    check_apart(lens_in, not_lens);
    check_apart(refs_in, not_refs);
    check_apart(add_in, out);
    a.table = table; a.lens = lens; a.refs = refs; a.rows = rows; a.max_pages = max_pages; a.n_add = n_add;
    a.n_add_all = n_add_all; a.table_out = table_out; a.lens_out = lens_out; a.refs_out = refs_out;
    a.granted = granted; a.info = info; a.scratch = scratch;
    page_reserve(a, (hipStream_t)stream);
  });
}

size_t sr_page_compact_scratch(int32_t n_pages) { return n_pages < 1 ? 0 : page_compact_scratch(n_pages); }

sr_status sr_page_compact(void* pool, int64_t block_elems, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim,
                          int32_t elem_bytes, int32_t page_tokens, int32_t n_pages, const int32_t* table,
                          const int32_t* lens, const int32_t* refs, int32_t rows, int32_t max_pages,
                          int32_t* table_out, int32_t* refs_out, int32_t* info, int32_t* scratch,
                          size_t scratch_elems, void* stream) {
  return (sr_status)guarded([&] {
    PageCompactArgs a;
    const int shift = check_table(rows, max_pages, page_tokens, n_pages);
    a.p = check_pool(pool, block_elems, n_layers, n_kv_heads, head_dim, elem_bytes, shift, n_pages);
    require(refs && refs_out && info, "NULL buffer");
    require(rows == 0 || (table && lens && table_out), "NULL buffer");
    const size_t need = page_compact_scratch(n_pages);
    SR_REQUIRE(scratch && scratch_elems >= need, SR_ERR_WORKSPACE_TOO_SMALL,
               "compact scratch too small: need " + std::to_string(need) + " elements");
    const int64_t nt = (int64_t)rows * max_pages;
    check_in_out(table, table_out, nt);
    check_in_out(refs, refs_out, n_pages);
    const Range out[] = {{table_out, 4 * nt}, {refs_out, 4 * (int64_t)n_pages}, {info, 16},
                         {scratch, 4 * (int64_t)need}, {pool, 2 * n_layers * a.p.block_bytes}};
    check_distinct(out);
    const Range table_in[] = {{table, 4 * nt}}, refs_in[] = {{refs, 4 * (int64_t)n_pages}};
    const Range lens_in[] = {{lens, 4 * (int64_t)rows}};
    const Range not_table[] = {out[1], out[2], out[3], out[4]}, not_refs[] = {out[0], out[2], out[3], out[4]};
    check_apart(table_in, not_table);
    check_apart(refs_in, not_refs);
    check_apart(lens_in, out);
    a.table = table; a.lens = lens; a.refs = refs; a.rows = rows; a.max_pages = max_pages; a.table_out = table_out;
    a.refs_out = refs_out; a.info = info; a.scratch = scratch;
    page_compact(a, (hipStream_t)stream);
  });
}

sr_status sr_rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double low, double high,
                              double n, double* freqs) {
  return (sr_status)guarded([&] {
    require(freqs != nullptr, "NULL buffer");
    require(rot_dim >= 8 && rot_dim <= 256 && rot_dim % 8 == 0, "rot_dim must be a multiple of 8 in [8, 256]");
    require(std::isfinite(theta) && theta > 0.0, "theta must be finite and > 0");
    require(scaling == SR_ROPE_PLAIN || scaling == SR_ROPE_LINEAR || scaling == SR_ROPE_BANDS, "unknown scaling");
    require(scaling == SR_ROPE_PLAIN || (std::isfinite(factor) && factor >= 1.0), "factor must be finite and >= 1");
    require(scaling != SR_ROPE_BANDS ||
                (std::isfinite(high) && low > 0.0 && low < high && std::isfinite(n) && n >= 1.0),
            "bands need 0 < low < high and n >= 1");
    for (int i = 0; i < rot_dim / 2; ++i) {
      double f = std::pow(theta, -2.0 * i / rot_dim);
      if (scaling == SR_ROPE_LINEAR) f /= factor;
      if (scaling == SR_ROPE_BANDS) {
        const double turns = n * f / (2.0 * M_PI);   // n / wavelength
        const double s = std::fmin(1.0, std::fmax(0.0, (turns - low) / (high - low)));
        f *= (1.0 - s) / factor + s;
      }
      freqs[i] = f;
    }
  });
}

sr_status sr_page_append(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t rows,
                         int32_t lr, const float* qkv, const double* freqs, int32_t rot_dim, int32_t interleaved,
                         void* kpool, void* vpool, int32_t page_tokens, int32_t n_pages, const int32_t* table,
                         int32_t max_pages, const int32_t* lens, const int32_t* n_new, float* q, void* stream) {
  return (sr_status)guarded([&] {
    check_heads(dtype, head_dim, n_heads, n_kv_heads);
    PageAppendArgs a;
    a.shift = check_table(rows, max_pages, page_tokens, n_pages);
    require(lr >= 0 && rot_dim >= 0 && rot_dim <= head_dim && rot_dim % 8 == 0,
            "lr >= 0 and rot_dim 0 or a multiple of 8 up to head_dim");
    supported((int64_t)rows * lr <= kMaxGroups, "2^24 tokens or more");
    if (rows == 0 || lr == 0) return;
    require(qkv && kpool && vpool && table && lens && q && (rot_dim == 0 || freqs), "NULL buffer");
    require(aligned16(qkv) && aligned16(q) && aligned16(kpool) && aligned16(vpool),
            "qkv, q, kpool and vpool must be 16-byte aligned");
    const int64_t tokens = (int64_t)rows * lr, block = block_bytes(dtype, n_pages, n_kv_heads, a.shift, head_dim);
    const Range in[] = {{qkv, tokens * (n_heads + 2 * n_kv_heads) * head_dim * 4}, {freqs, 4 * (int64_t)rot_dim},
                        {table, 4 * (int64_t)rows * max_pages}, {lens, 4 * (int64_t)rows},
                        {n_new, 4 * (int64_t)rows}};
    const Range out[] = {{q, tokens * n_heads * head_dim * 4}, {kpool, block}, {vpool, block}};
    check_apart(in, out);
    check_distinct(out);
    a.dtype = dtype; a.hd = head_dim; a.hq = n_heads; a.hkv = n_kv_heads; a.rows = rows; a.lr = lr; a.qkv = qkv;
    a.freqs = freqs; a.rot = rot_dim; a.interleaved = interleaved != 0; a.kpool = kpool; a.vpool = vpool;
    a.n_pages = n_pages; a.table = table; a.max_pages = max_pages; a.lens = lens; a.n_new = n_new; a.q = q;
    page_append(a, (hipStream_t)stream);
  });
}

size_t sr_paged_attention_scratch(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t rows,
                                  int32_t lr, int32_t page_tokens, int32_t max_pages, int32_t window, int32_t sinks,
                                  int32_t shared, int32_t max_len) {
  size_t n = 0;
  guarded([&] {
    PagedAttnArgs a;
    if (attention_args(dtype, head_dim, n_heads, n_kv_heads, rows, lr, page_tokens, 1, max_pages, window, sinks,
                       shared, max_len, &a))
      n = paged_attn_scratch(a);
  });
  return n;
}

sr_status sr_paged_attention(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads, int32_t rows,
                             int32_t lr, const float* q, const void* kpool, const void* vpool, int32_t page_tokens,
                             int32_t n_pages, const int32_t* table, int32_t max_pages, const int32_t* lens,
                             const int32_t* n_new, int32_t window, int32_t sinks, int32_t shared, int32_t max_len,
                             void* out, float* scratch, size_t scratch_elems, void* stream) {
  return (sr_status)guarded([&] {
    PagedAttnArgs a;
    if (!attention_args(dtype, head_dim, n_heads, n_kv_heads, rows, lr, page_tokens, n_pages, max_pages, window, sinks,
                        shared, max_len, &a))
      return;
    require(q && kpool && vpool && table && lens && out, "NULL buffer");
    require(aligned16(q) && aligned16(kpool) && aligned16(vpool) && aligned16(out),
            "q, kpool, vpool and out must be 16-byte aligned");
    const size_t need = paged_attn_scratch(a);
    SR_REQUIRE(scratch_elems >= need && (need == 0 || scratch), SR_ERR_WORKSPACE_TOO_SMALL,
               "attention scratch too small: need " + std::to_string(need) + " floats");
    require(aligned16(scratch), "scratch must be 16-byte aligned");
    const int64_t heads = (int64_t)rows * lr * n_heads * head_dim;
    const int64_t block = block_bytes(dtype, n_pages, n_kv_heads, a.shift, head_dim);
    const Range in[] = {{q, 4 * heads}, {kpool, block}, {vpool, block}, {table, 4 * (int64_t)rows * max_pages},
                        {lens, 4 * (int64_t)rows}, {n_new, 4 * (int64_t)rows}};
    const Range dst[] = {{out, heads * (dtype == SR_BF16 ? 2 : 4)}, {need ? scratch : nullptr, 4 * (int64_t)need}};
    check_apart(in, dst);
    check_distinct(dst);
    a.q = q; a.kpool = kpool; a.vpool = vpool; a.table = table; a.lens = lens; a.n_new = n_new; a.out = out;
    a.part = scratch;
    paged_attn(a, (hipStream_t)stream);
  });
}

size_t sr_token_logprobs_scratch(int32_t rows, int32_t vocab, int32_t top) {
  if (rows < 1 || vocab < 1 || vocab > 262144 || top < 0 || top > 32 || top > vocab) return 0;
  return token_logprobs_scratch(rows, vocab, top);
}

sr_status sr_token_logprobs(int32_t dtype, const void* logits, int64_t row_stride, int32_t rows, int32_t vocab,
                            float temperature, const int32_t* tokens, int32_t top, float* logprob, float* entropy,
                            int32_t* top_ids, float* top_logprobs, float* scratch, size_t scratch_elems,
                            void* stream) {
  return (sr_status)guarded([&] {
    require(dtype == SR_F32 || dtype == SR_BF16, "unknown dtype");
    require(rows >= 0 && vocab >= 1 && row_stride >= vocab, "bad rows / vocab / row_stride");
    require(std::isfinite(temperature) && temperature > 0.f, "temperature must be finite and > 0");
    require(std::isfinite((float)(1.5 / (double)temperature)), "temperature too small");
    require(top >= 0 && top <= vocab, "top must be in [0, vocab]");
    supported(vocab <= 262144, "vocab above 262144");
    supported(top <= 32, "top above 32");
    supported(row_stride <= (int64_t)1 << 40, "row_stride above 2^40");
    supported(rows <= 1 << 20, "at most 2^20 rows");
    if (rows == 0) return;
    require(logits && (!logprob || tokens), "NULL buffer");
    const int es = dtype == SR_BF16 ? 2 : 4;
    require((reinterpret_cast<uintptr_t>(logits) & (es - 1)) == 0, "logits off an element boundary");
    const size_t need = token_logprobs_scratch(rows, vocab, top);
    SR_REQUIRE(scratch_elems >= need && (need == 0 || scratch), SR_ERR_WORKSPACE_TOO_SMALL,
               "log-probability scratch too small: need " + std::to_string(need) + " floats");
    const int64_t nk = 4 * (int64_t)rows * top;
    const Range in[] = {{logits, ((rows - 1) * row_stride + vocab) * es}, {tokens, 4 * (int64_t)rows}};
    const Range out[] = {{logprob, 4 * (int64_t)rows}, {entropy, 4 * (int64_t)rows}, {nk ? top_ids : nullptr, nk},
                         {nk ? top_logprobs : nullptr, nk}, {need ? scratch : nullptr, 4 * (int64_t)need}};
    check_apart(in, out);
    check_distinct(out);
    LogprobArgs a;
    a.dtype = dtype; a.logits = logits; a.row_stride = row_stride; a.rows = rows; a.vocab = vocab;
    a.temperature = temperature; a.tokens = tokens; a.top = top; a.logprob = logprob; a.entropy = entropy;
    a.top_ids = top_ids; a.top_logprobs = top_logprobs; a.scratch = scratch;
    token_logprobs(a, (hipStream_t)stream);
  });
}

}  // extern "C"
