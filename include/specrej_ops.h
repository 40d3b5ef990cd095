/*
 * specrej_ops.h -- kernel-level operators over a paged candidate cache, and
 * log-probabilities of given tokens (MI355X, gfx950).
 *
 * The cache of sr_generate holds every candidate in a contiguous row and
 * copies the survivors of a cut.  Here candidates are lists of pages: forking
 * a candidate, or dropping one, moves no keys and values, rows have lengths of
 * their own, and a sliding window lets go of the pages behind it.
 *
 * The conventions of specrej.h hold: statuses, sr_last_error, arguments
 * validated before any device work, caller-owned memory, no allocation, every
 * function asynchronous on `stream` (device work of the current device, which
 * must be the stream's).  Calls are re-entrant given distinct outputs and
 * scratch; two captured graphs may share a scratch buffer only if they never
 * run at the same time.  No function synchronises, so all may be captured.
 *
 * The pool.  2 * n_layers blocks as in sr_compact: block (l, kv), l the layer
 * and kv 0 for keys, 1 for values, starts at element (2 l + kv) * block_elems
 * and is laid out [n_pages][n_kv_heads][page_tokens][head_dim].  page_tokens
 * is 16, 32, 64, 128 or 256.  Pools are 16-byte aligned.
 *
 * The table.  DEVICE int32 [rows][max_pages]: token t of row r lies in slot
 * t % page_tokens of page table[r][t / page_tokens]; lens, DEVICE int32
 * [rows], counts the row's tokens.  Lengths are taken as if clamped to
 * [0, max_pages * page_tokens].  Entries at or past ceil(lens[r] /
 * page_tokens) are not read.  An entry outside [0, n_pages) names no page: its
 * tokens are as if masked, nothing is read or written there.  refs, DEVICE
 * int32 [n_pages], counts the entries that name each page; 0 is a free page.
 *
 * Limits: rows <= 4096, max_pages <= 65536, n_pages <= 2^20.
 */
#ifndef SPECREJ_OPS_H
#define SPECREJ_OPS_H

#include "specrej.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Forks, drops and reorders rows: new row j < new_rows is row parent[j] of
 * the old table (DEVICE int32 [new_rows]; outside [0, rows): an empty row).
 *   lens_out[j] = lens[parent[j]], table_out[j] = the parent's entries (-1
 *   past its length and for entries that name no page), refs_out[p] = number
 *   of entries of table_out that name p.
 * A candidate named twice is forked, one that no new row names is freed, and
 * no keys or values move.  window > 0: the entries of pages that no later
 * token can see under this window and these sinks (sr_paged_attention) become
 * -1, which frees the pages behind the window; window = 0 keeps all.
 * table_out, lens_out, refs_out: DEVICE int32 [new_rows][max_pages],
 * [new_rows], [n_pages]; they may not overlap the inputs. */
sr_status sr_page_fork(const int32_t *table, const int32_t *lens, int32_t rows, int32_t max_pages,
                       const int32_t *parent, int32_t new_rows, int32_t page_tokens, int32_t n_pages,
                       int32_t window, int32_t sinks, int32_t *table_out, int32_t *lens_out,
                       int32_t *refs_out, void *stream);

/* Room for n_add[r] more tokens (DEVICE int32 [rows]; NULL = n_add_all in
 * every row; negative counts as 0) of every row.
 *  - New pages are the free ones (refs 0), lowest first, dealt to the rows in
 *    ascending order and within a row in token order.
 *  - A row that adds tokens to a part-filled last page that other entries
 *    name too gets a page of its own, with the filled slots of all layers
 *    copied.  One row may keep the page: if every entry that names it is the
 *    part-filled last page of a row adding tokens, the lowest such row does.
 *    A part-filled last page whose entry names no page is replaced by a new
 *    page, without a copy: the row's len % page_tokens tokens in it, masked
 *    until then, would be whatever the page held before.  The caller writes
 *    them again, with the new ones (sr_page_append with n_new = len %
 *    page_tokens + the added tokens), before a call reads the row.
 *  - All or nothing: info (DEVICE int32 [4]) receives the missing pages, the
 *    rows whose new length passes max_pages * page_tokens, and, if both are
 *    0, the pages taken and the pages copied.  Otherwise nothing is reserved
 *    (those two are 0) and the outputs are the rows and counts as they were.
 * granted[r] = tokens reserved (0 in that case), lens_out = lens (clamped) +
 * granted, table_out, refs_out: the new table (-1 past lens_out and for entries
 * that name no page, in either case) and counts.  table_out, lens_out and
 * refs_out may each be the input itself; any other overlap is an error.  pool:
 * DEVICE, elements of elem_bytes 2 or 4.  scratch: DEVICE int32 of scratch_elems >=
 * sr_page_reserve_scratch(rows, max_pages, n_pages) elements. */
sr_status sr_page_reserve(void *pool, int64_t block_elems, int32_t n_layers, int32_t n_kv_heads,
                          int32_t head_dim, int32_t elem_bytes, int32_t page_tokens, int32_t n_pages,
                          const int32_t *table, const int32_t *lens, const int32_t *refs, int32_t rows,
                          int32_t max_pages, const int32_t *n_add, int32_t n_add_all, int32_t *table_out,
                          int32_t *lens_out, int32_t *refs_out, int32_t *granted, int32_t *info,
                          int32_t *scratch, size_t scratch_elems, void *stream);
size_t sr_page_reserve_scratch(int32_t rows, int32_t max_pages, int32_t n_pages);

/* Moves the live pages (refs > 0) to the front of the pool, in place: with n
 * live pages, the i-th live page at or past n moves to the i-th free page
 * below n (both ascending), in every layer.  table_out: the entries renamed
 * (-1 past the lengths and for entries that name no page); refs_out: counts of
 * the moved pages.  info (DEVICE int32 [4]) receives n, the pages moved, 0, 0.
 * Pages [n, n_pages) are free afterwards; their contents are left as they
 * were.  refs must count every page the table names; entries that name a page
 * with refs 0 keep their number.  table_out and refs_out may each be the input
 * itself; any other overlap is an error.  scratch: DEVICE int32 of at least
 * sr_page_compact_scratch(n_pages) elements. */
sr_status sr_page_compact(void *pool, int64_t block_elems, int32_t n_layers, int32_t n_kv_heads,
                          int32_t head_dim, int32_t elem_bytes, int32_t page_tokens, int32_t n_pages,
                          const int32_t *table, const int32_t *lens, const int32_t *refs, int32_t rows,
                          int32_t max_pages, int32_t *table_out, int32_t *refs_out, int32_t *info,
                          int32_t *scratch, size_t scratch_elems, void *stream);
size_t sr_page_compact_scratch(int32_t n_pages);

/* Rotary frequencies of pair i < rot_dim / 2, in radians a position:
 * theta^(-2 i / rot_dim), scaled for long contexts by
 *   SR_ROPE_PLAIN   nothing;
 *   SR_ROPE_LINEAR  1 / factor;
 *   SR_ROPE_BANDS   by wavelength w = 2 pi / f against the trained context n:
 *                   as it is where w < n / high, 1 / factor where w > n / low,
 *                   and between them (1 - s) / factor + s with
 *                   s = (n / w - low) / (high - low).
 * freqs: HOST double [rot_dim / 2].  rot_dim a multiple of 8 in [8, 256],
 * theta > 0, factor >= 1; low, high (0 < low < high) and n >= 1 are read for
 * SR_ROPE_BANDS only.  Host only. */
enum { SR_ROPE_PLAIN = 0, SR_ROPE_LINEAR = 1, SR_ROPE_BANDS = 2 };
sr_status sr_rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double low,
                              double high, double n, double *freqs);

/* Rotary positions and cache append: the step between a QKV projection
 * (sr_projection mode 0) and sr_paged_attention.  qkv (DEVICE float
 * [rows][lr][(n_heads + 2 n_kv_heads) head_dim]: q heads, k heads, v heads)
 * holds the projections of the last n_new[r] <= lr tokens of row r (DEVICE
 * int32 [rows]; NULL = lr everywhere; clamped to [0, min(lr, lens[r])]); token
 * t < n_new[r] sits at position lens[r] - n_new[r] + t.  The first rot_dim
 * dimensions of every q and k head are rotated by the angles position *
 * freqs[i] (DEVICE double [rot_dim / 2], formed in double): pair i is
 * dimensions (i, i + rot_dim / 2), or (2 i, 2 i + 1) where interleaved is not
 * 0; the others pass as they are.  q (DEVICE float [rows][lr][n_heads]
 * [head_dim]) receives the queries; keys and values go to their slots of kpool
 * and vpool (one layer's blocks, dtype elements, rounded to nearest).  Rows of
 * q past n_new[r], and tokens whose entry names no page, are not written.
 * Two rows that write one page write it in no fixed order: reserve the tokens
 * first (sr_page_reserve).  rot_dim: 0 or a multiple of 8 up to head_dim;
 * head_dim in {32, 64, 128}; rows * lr < 2^24; qkv, q 16-byte aligned. */
sr_status sr_page_append(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                         int32_t rows, int32_t lr, const float *qkv, const double *freqs, int32_t rot_dim,
                         int32_t interleaved, void *kpool, void *vpool, int32_t page_tokens,
                         int32_t n_pages, const int32_t *table, int32_t max_pages, const int32_t *lens,
                         const int32_t *n_new, float *q, void *stream);

/* Causal attention over the pages, for single tokens (lr = 1), a few (drafts)
 * or prompts: query t < n_new[r] of row r (q: DEVICE float [rows][lr][n_heads]
 * [head_dim]) sits at position p = lens[r] - n_new[r] + t, its own key and
 * value and all earlier ones in the cache, and sees key j of its row iff
 *   j <= p and (window == 0 or j > p - window or j < sinks);
 * out[r][t][i head_dim + d] (DEVICE dtype [rows][lr][n_heads head_dim]) =
 * sum_j softmax_j(q_i . key_j / sqrt(head_dim)) value_j[d], KV head
 * floor(i n_kv_heads / n_heads); 0 where nothing is visible, or every score is
 * -inf.  n_new as in sr_page_append; rows of out past n_new[r] are not written.
 * A NaN in a query, or in a key or value that it sees, gives NaN in the outputs
 * that depend on it and in no others.
 * An infinite value gives infinite outputs (NaN where signs meet, or where its
 * weight is 0 in fp32); an infinite query or key may give NaN.
 * Slots that no query of a row sees (past its length, behind its window, in
 * entries that name no page) may hold anything, NaN included; a key or value
 * that one query sees and another query of the call does not must be finite.
 * shared: a number of leading tokens whose pages most rows have in common with
 * row 0 (a forked prompt).  bf16 calls of at most 16 query columns a row (lr
 * n_heads / n_kv_heads) compute their part once for all rows whose entries
 * equal row 0's, which is checked on the device, where that saves 300 MB of
 * reads or more; rows that name other pages, or whose window has left key 0,
 * read their own.  The result does not depend on it beyond rounding.
 * max_len: the longest row the caller expects (plans the split of the work over
 * the keys; rows may be longer), >= 1.
 * head_dim in {32, 64, 128}; n_heads / n_kv_heads <= 16; rows * lr * n_heads <=
 * 2^28; calls of 2^24 work-groups are refused, counted for one KV head where
 * they hold up to 8 query columns (fp32, head_dim 32) and for all of them where
 * they hold 128 (prompts in bf16).  bf16 with head_dim 64 or 128 runs on the
 * matrix cores: probabilities rounded to bf16, sums in fp32, queries in 16 bits
 * where a row has at most 16 query columns, rounded to bf16 where it has more.
 * q, kpool, vpool, out 16-byte aligned.  scratch: DEVICE float of scratch_elems
 * >= sr_paged_attention_scratch(...) elements. */
sr_status sr_paged_attention(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                             int32_t rows, int32_t lr, const float *q, const void *kpool,
                             const void *vpool, int32_t page_tokens, int32_t n_pages,
                             const int32_t *table, int32_t max_pages, const int32_t *lens,
                             const int32_t *n_new, int32_t window, int32_t sinks, int32_t shared,
                             int32_t max_len, void *out, float *scratch, size_t scratch_elems,
                             void *stream);
size_t sr_paged_attention_scratch(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                                  int32_t rows, int32_t lr, int32_t page_tokens, int32_t max_pages,
                                  int32_t window, int32_t sinks, int32_t shared, int32_t max_len);

/* Log-probabilities under softmax(logits[r] / temperature) (temperature > 0; for
 * finite logits the distribution that sr_sample draws from), for every row r < rows of logits
 * (DEVICE dtype [rows][row_stride], vocab <= row_stride entries used, vocab <=
 * 262144, rows <= 2^20).  Any output may be NULL:
 *   logprob[r] = ln p(tokens[r]) (tokens: DEVICE int32 [rows]; -1, padding: 0;
 *                any other value outside [0, vocab): NaN),
 *   entropy[r] = - sum_i p_i ln p_i (nats),
 *   top_ids, top_logprobs [rows][top]: the top <= 32 most likely tokens, by
 *                logit descending, then token ascending; top <= vocab.
 * A NaN logit counts as -inf (as in sr_sample).  -inf has probability 0 (ln p
 * = -inf); logits of +inf share the probability evenly; a row without a logit
 * above -inf has no distribution: logprob and top_logprobs -inf, entropy 0.
 * Sums in fp32, in an order fixed by the call's sizes.  scratch: DEVICE float
 * of scratch_elems >= sr_token_logprobs_scratch(rows, vocab, top) elements. */
sr_status sr_token_logprobs(int32_t dtype, const void *logits, int64_t row_stride, int32_t rows,
                            int32_t vocab, float temperature, const int32_t *tokens, int32_t top,
                            float *logprob, float *entropy, int32_t *top_ids, float *top_logprobs,
                            float *scratch, size_t scratch_elems, void *stream);
size_t sr_token_logprobs_scratch(int32_t rows, int32_t vocab, int32_t top);

#ifdef __cplusplus
}
#endif

#endif /* SPECREJ_OPS_H */
