/*
 * specrej_serving.h -- operators for a decoding loop over a candidate cache
 * held in 4 bits (MI355X, gfx950): head norms, rotation and append in one pass,
 * attention over the pages, reading them back, and the filtered draw of the next
 * tokens.
 *
 * The conventions of specrej.h and specrej_ops.h hold (statuses, sr_last_error,
 * arguments validated before any device work, caller-owned memory, asynchronous
 * on `stream`, tables, lengths and limits).  sr_page_fork, sr_page_reserve and
 * sr_page_compact serve these pools too (elem_bytes 1).
 *
 * SR_FP4, a cache of 4 bits.  32 neighbouring dimensions (32 g .. 32 g + 31) of
 * a key or value share a scale 2^(b - 127), b a byte in [2, 252], and each is one
 * of +-(0, 0.5, 1, 1.5, 2, 3, 4, 6), codes 0 .. 7 (sign in bit 3), times the
 * scale.  b = 255: every value of the group is NaN.  The operators write the
 * least b with which the group's largest magnitude is below 7 scales (2 where it
 * is 0, 252 where it is 2^127 or more), the nearest values, ties to the even
 * code, magnitudes above 5 scales as 6; a group that holds a NaN or an infinity
 * gets b = 255 and codes 0.  On normal draws the values are 11 % off in the
 * 2-norm.
 * A layer's block of keys (or values) is laid out [n_pages][n_kv_heads], each of
 * these page_tokens * head_dim / 2 bytes of codes [page_tokens][head_dim / 2],
 * dimension 2 i in the low half of byte i, then page_tokens * head_dim / 32 bytes
 * b [page_tokens][head_dim / 32]: 17 head_dim / 32 bytes a token.  Blocks are 16-byte
 * aligned.
 */
#ifndef SPECREJ_SERVING_H
#define SPECREJ_SERVING_H

#include "specrej_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Cache types beside SR_F32 and SR_BF16. */
enum { SR_FP4 = 2 };

/* sr_page_append with the norms that some models put on every query and key
 * head, and for caches of 4 bits.  q_gain, k_gain: DEVICE float [head_dim] or
 * NULL (no norm there); a head x becomes x / sqrt(mean(x^2) + eps) * gain, all
 * head_dim dimensions, before the first rot_dim of them are rotated.  cache:
 * SR_F32, SR_BF16 or SR_FP4, the type of kpool and vpool.  Everything is computed
 * in 64 bits and rounded once, so that what a cache holds does not turn on the order
 * of a sum.  Everything else (qkv, freqs, tables, n_new, tokens without a page, limits) is as
 * sr_page_append has it.  eps >= 0 and finite; with eps = 0 a head of zeros gives
 * NaN. */
sr_status sr_page_append_norm(int32_t cache, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                              int32_t rows, int32_t lr, const float *qkv, const double *freqs,
                              int32_t rot_dim, int32_t interleaved, const float *q_gain,
                              const float *k_gain, double eps, void *kpool, void *vpool,
                              int32_t page_tokens, int32_t n_pages, const int32_t *table,
                              int32_t max_pages, const int32_t *lens, const int32_t *n_new, float *q,
                              void *stream);

/* Keys and values of the rows' last tokens, as the pages hold them: token t <
 * n_new[r] (NULL = lr everywhere; clamped to [0, min(lr, lens[r])]) of row r sits
 * at position lens[r] - n_new[r] + t and goes to k_out, v_out [r][t] (DEVICE dtype
 * [rows][lr][n_kv_heads][head_dim], dtype SR_F32 or SR_BF16, rounded to nearest
 * where the cache has more bits; values of 4 bits are exact in both).  Tokens whose
 * entry names no page read as 0; rows of the outputs past n_new[r] are not written.
 * k_out or v_out may be NULL, and then so may its pool.  head_dim in {32, 64, 128};
 * rows * lr < 2^24; outputs 16-byte aligned and apart from everything else. */
sr_status sr_page_read(int32_t cache, int32_t dtype, int32_t head_dim, int32_t n_kv_heads, int32_t rows,
                       int32_t lr, const void *kpool, const void *vpool, int32_t page_tokens,
                       int32_t n_pages, const int32_t *table, int32_t max_pages, const int32_t *lens,
                       const int32_t *n_new, void *k_out, void *v_out, void *stream);

/* sr_paged_attention over pools of SR_FP4: the same formula, visibility, rows,
 * n_new, window, sinks, shared, max_len, NaN rules and limits, on the values that the
 * pages stand for.  out: dtype SR_BF16 or SR_F32.  On the matrix cores, which keys
 * and values enter exactly.  SR_BF16: queries keep 16 bits where a row has at most 16
 * query columns (lr n_heads / n_kv_heads), and where it has more are off by up to 2^-13
 * of the largest of every 32 dimensions (products of such a query with keys are exact); probabilities keep 16 bits where a row has at
 * most 8 columns, 8 where it has more and for shared keys that are read once for all
 * rows; sums are in fp32.  SR_F32: queries and probabilities enter as three parts, all
 * 24 bits.  A layer's keys take less than
 * 2^36 bytes.  scratch: DEVICE float of scratch_elems >=
 * sr_paged_attention_fp4_scratch(...) elements. */
sr_status sr_paged_attention_fp4(int32_t dtype, int32_t head_dim, int32_t n_heads, int32_t n_kv_heads,
                                 int32_t rows, int32_t lr, const float *q, const void *kpool,
                                 const void *vpool, int32_t page_tokens, int32_t n_pages,
                                 const int32_t *table, int32_t max_pages, const int32_t *lens,
                                 const int32_t *n_new, int32_t window, int32_t sinks, int32_t shared,
                                 int32_t max_len, void *out, float *scratch, size_t scratch_elems,
                                 void *stream);
size_t sr_paged_attention_fp4_scratch(int32_t dtype, int32_t head_dim, int32_t n_heads,
                                      int32_t n_kv_heads, int32_t rows, int32_t lr, int32_t page_tokens,
                                      int32_t max_pages, int32_t window, int32_t sinks, int32_t shared,
                                      int32_t max_len);

/* Next tokens by temperature, top-k, top-p and min-p, from given random words: for
 * every row r < rows of logits (DEVICE dtype [rows][row_stride], vocab <= row_stride
 * entries used, vocab <= 262144, rows <= 2^20).  Every setting is one number for all
 * rows (the _all argument) or, where its pointer is not NULL, DEVICE [rows].
 *   weights  w_i = trunc(e^((l_i - max) / T) 2^32), the integers that sr_sample draws
 *            by (1 / T rounded to fp32, the exponential by its rounded steps).  T that
 *            is not above 0, or whose 1 / T is not finite in fp32: the first largest
 *            logit, for certain.  A NaN logit counts as -inf; logits of +inf
 *            share the probability evenly.
 *   order    by logit descending (-0 = +0), then index ascending.
 *   top_k    1 <= top_k < vocab keeps the first top_k in that order.
 *   top_p    keeps, of those, the shortest prefix that holds at least top_p of their
 *            weight (top_p taken down to a multiple of 2^-32), one at least; not below
 *            1, or NaN: all; negative counts as 0.
 *   min_p    keeps those of weight >= trunc(min_p 2^32), that is of probability
 *            min_p times the largest; not above 0, or NaN: all; above 1 counts as 1.
 *   draw     x = random[r * random_stride] (DEVICE uint32), W the kept weight: token[r]
 *            = the least index i with the kept weights of indices <= i above
 *            floor(x W / 2^32).
 * Integers throughout, so a result depends on no order of summation; with nothing
 * filtered the token is sr_sample's for the same word (finite maxima).  Outputs
 * (token or any other may be NULL): token DEVICE int32 [rows]; logprob DEVICE float
 * [rows], ln(w_token / W); kept DEVICE int32 [rows], the kept entries of weight above 0.
 * A row without a logit above -inf: token 0, logprob -inf, kept 0.
 * scratch: DEVICE uint32 of scratch_elems >= sr_sample_filtered_scratch(rows, vocab)
 * elements, 16-byte aligned. */
sr_status sr_sample_filtered(int32_t dtype, const void *logits, int64_t row_stride, int32_t rows,
                             int32_t vocab, const float *temperature, float temperature_all,
                             const int32_t *top_k, int32_t top_k_all, const float *top_p,
                             float top_p_all, const float *min_p, float min_p_all,
                             const uint32_t *random, int64_t random_stride, int32_t *token,
                             float *logprob, int32_t *kept, uint32_t *scratch, size_t scratch_elems,
                             void *stream);
size_t sr_sample_filtered_scratch(int32_t rows, int32_t vocab);

#ifdef __cplusplus
}
#endif

#endif /* SPECREJ_SERVING_H */
