/*
 * The key holder's steps in the clear, on the device: what a transformer block computes on decrypted activations
 * between two encrypted projections (ckks.h).  Layer norm with its gradient, the key / value cache with the attention
 * over it, in the activations' type or in 8 bits, the rules on logits and the draw of the next token.
 *
 * Conventions are those of ckks.h: 0 or a negative CKKS_E_* code with ckks_last_error(), device pointers carry "d_",
 * `stream` is a hipStream_t, calls enqueue and return, nothing is allocated and nothing is kept between calls, so they
 * may be captured into a graph.  No parameter set is involved.  An argument struct is read before the call returns.
 *
 *  - Types: CKKS_CLEAR_F32 / F16 / BF16.  Sums, statistics and softmax are held in 32 bits whatever the type; each
 *    output is rounded to its type once (attention also rounds its weights, see there).
 *  - Strides count elements; the last dimension is contiguous.  Every pointer is aligned to its type; wider alignment is
 *    not needed.
 *  - Lengths, page tables, token ids and positions are device data and are not read by the host.  A value that is out of
 *    range never makes a kernel touch memory outside the arrays described; what it does instead is said below.
 *  - Outputs may not overlap inputs unless said: CKKS_E_INVAL, nothing enqueued.  The test goes by the whole extent
 *    of an array, first to last element, unless said.  Neither may the rows of one output overlap one another.
 */
#ifndef CKKS_CLEAR_H
#define CKKS_CLEAR_H

#include "ckks.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CKKS_CLEAR_F32 0u
#define CKKS_CLEAR_F16 1u
#define CKKS_CLEAR_BF16 2u

/* ---- layer norm ----------------------------------------------------------
 * y = (x - mean) * rstd * weight + bias over the `cols` entries of each row, mean and rstd = 1/sqrt(var + eps) of that row,
 * var = sum (x - mean)^2 / cols.  d_weight, d_bias: [cols] of weight_dtype (F32 or dtype), either NULL (1 and 0).
 * d_mean, d_rstd: f32 [rows], both or neither NULL; the gradient needs them.  d_y may be d_x with the same stride. */
typedef struct {
    const void *d_x, *d_weight, *d_bias;
    void *d_y;
    float *d_mean, *d_rstd;
    int64_t x_stride, y_stride; /* between rows */
    uint32_t rows, cols, dtype, weight_dtype;
    float eps; /* >= 0 */
    uint32_t reserved;
} ckks_clear_norm_t;
int ckks_clear_layer_norm(const ckks_clear_norm_t *a, void *stream);

/* Gradient: with xh = (x - mean) rstd and g = dy * weight,
 *   dx = rstd (g - mean(g) - xh mean(g xh)),  dweight = sum over rows of dy xh,  dbias = sum over rows of dy.
 * d_dx [rows] by dx_stride, may be d_dy with the same stride; or NULL.  d_dweight, d_dbias [cols] of weight_dtype, either NULL;
 * zeros for rows = 0.  Row sums are joined in a fixed order: the same inputs give the same bits; cols below 2^28 for either.
 * d_work: at least ckks_clear_layer_norm_grad_work_bytes(rows, cols, dtype) bytes, 4-byte aligned, contents free;
 * may be NULL when both d_dweight and d_dbias are. */
typedef struct {
    const void *d_dy, *d_x, *d_weight;
    const float *d_mean, *d_rstd;
    void *d_dx, *d_dweight, *d_dbias;
    void *d_work;
    uint64_t work_bytes;
    int64_t dy_stride, x_stride, dx_stride;
    uint32_t rows, cols, dtype, weight_dtype;
} ckks_clear_norm_grad_t;
uint64_t ckks_clear_layer_norm_grad_work_bytes(uint32_t rows, uint32_t cols, uint32_t dtype);
int ckks_clear_layer_norm_grad(const ckks_clear_norm_grad_t *a, void *stream);

/* ---- key / value cache ---------------------------------------------------
 * Pages: d_k and d_v [n_pages][kv_heads][page_size][head_dim] by their strides {page, head, token}; head_dim a multiple
 * of 8, at most 256; any page_size >= 1.  A page stride is below 2^32 entries, the tokens of a page within 2^31.
 * Batch: n_seq sequences whose new tokens lie one after the other in n_tokens rows, sequence b in rows
 * q_start[b] .. q_start[b+1]-1 (int32 [n_seq+1], rising from 0 to n_tokens; values outside are clamped).  kv_len[b] counts the
 * tokens of sequence b with its new ones: new token i of n sits at position kv_len[b] - n + i.  Position p is row p % page_size
 * of page page_table[b * table_stride + p / page_size]; kv_len is taken as at most table_width * page_size. */
typedef struct {
    void *d_k, *d_v;
    int64_t k_stride[3], v_stride[3];
    uint32_t n_pages, page_size, kv_heads, head_dim, dtype, reserved;
} ckks_clear_pages_t;
typedef struct {
    const int32_t *d_q_start, *d_kv_len, *d_page_table;
    int64_t table_stride;
    uint32_t n_seq, n_tokens, table_width, reserved;
} ckks_clear_batch_t;

/* Writes the new tokens' keys and values into their pages, the keys rotated by their position, and the queries rotated
 * alike.  The first `rot` entries of a head (even, <= head_dim; 0: none) are pairs (x1, x2) -> (x1 cos - x2 sin,
 * x2 cos + x1 sin): entries j and j + rot/2, or with CKKS_CLEAR_INTERLEAVED 2j and 2j + 1, by the angle of
 * d_cos / d_sin [n_pos][rot/2] (f32) at the token's position, or at d_positions[row] (int32 [n_tokens]) if that is given.
 * The rotation is computed in 32 bits and rounded once.  A position outside [0, n_pos) has no angle: the rotated
 * entries come out as NaN.  Tokens at a position below 0 and pages outside [0, n_pages) are not stored.
 * Keys and values may lie in one array as long as they share no entry of it.
 * d_k, d_v: rows by strides {token, head}.  d_q may be NULL; d_q_out may be d_q with the same strides, and then lie between the
 * rows of the new keys and values (columns of one array) as long as it shares no entry with them.  A row in no sequence has no
 * position.  heads and kv_heads: at most 65536. */
#define CKKS_CLEAR_INTERLEAVED 1u
typedef struct {
    ckks_clear_pages_t pages;
    ckks_clear_batch_t batch;
    const void *d_new_k, *d_new_v, *d_q;
    void *d_q_out;
    const float *d_cos, *d_sin;
    const int32_t *d_positions;
    int64_t new_k_stride[2], new_v_stride[2], q_stride[2], q_out_stride[2];
    uint32_t heads, rot, n_pos, flags;
} ckks_clear_append_t;
int ckks_clear_cache_append(const ckks_clear_append_t *a, void *stream);

/* Attention of the new tokens over the cache (which holds them already).  Query head h reads kv head h / (heads / kv_heads).
 * A query at position t sees the keys j < kv_len, with CKKS_CLEAR_CAUSAL only j <= t, with window > 0 (causal only) only
 * j > t - window:
 *   out = sum_j softmax_j(scale q.k_j) v_j,  lse = log sum_j exp(scale q.k_j)   (natural logarithm)
 * A query that sees no key (or only keys with scores of -infinity) gets out = 0 and lse = -infinity.  Keys and values that a query
 * does not see do not reach its result, whatever they hold.  A page outside [0, n_pages) reads as zeros.  scale > 0 and finite,
 * scores scale q.k and their multiples by log2(e) within the range of 32 bits.  Rows of q in no sequence are not written.
 * heads: a multiple of kv_heads, at most 65536, n_tokens * heads / kv_heads below 2^31.  One launch has to have a block of 256 threads or
 * 512 for each tile of queries and kv head, so some 2^23 single tokens times kv heads are the most.
 * All sums are 32-bit.  With 16-bit types a weight of the softmax meets the values as a high and a low number of that type for
 * single tokens and short chunks: only the result is rounded to the type.  For chunks whose products fill the device, by the
 * measured costs of either way, it is rounded to the type: F16 with its 11 bits down to 2^-25 of the row's largest so far, to steps
 * of 2^-35 of that below.
 * d_q, d_out: [n_tokens][heads][head_dim] by strides {token, head}; d_lse f32 [n_tokens][heads] or NULL.
 * d_work: at least ckks_clear_attend_work_bytes bytes, 16-byte aligned, contents free (NULL if that is 0). */
#define CKKS_CLEAR_CAUSAL 1u
typedef struct {
    ckks_clear_pages_t pages;
    ckks_clear_batch_t batch;
    const void *d_q;
    void *d_out;
    float *d_lse;
    void *d_work;
    uint64_t work_bytes;
    int64_t q_stride[2], out_stride[2];
    uint32_t heads, window, flags;
    float scale;
} ckks_clear_attend_t;
/* Only the counts (n_seq, n_tokens, table_width, page_size, heads, kv_heads, head_dim, dtype, flags, window) are read; 0 for
 * arguments that ckks_clear_attend refuses. */
uint64_t ckks_clear_attend_work_bytes(const ckks_clear_attend_t *a);
int ckks_clear_attend(const ckks_clear_attend_t *a, void *stream);

/* ---- logits --------------------------------------------------------------
 * The rules on the logits of the next token, row by row, in this order:
 *   history (d_tokens[token_start[r] .. token_start[r+1]), the first n_prompt[r] of them prompt, the others generated):
 *     a token of the history:  l = l > 0 ? l / repetition[r] : l * repetition[r]
 *     l -= frequency[r] * (times generated);  l -= presence[r] if generated at all
 *   biases (bias_ids / bias [bias_start[r] .. bias_start[r+1])): l += bias; of several for one token the last counts
 *   mask: bit v % 32 of word d_mask[r * mask_stride + v / 32] clear:  l = -infinity, whatever l was
 * d_repetition, d_frequency, d_presence: f32 [rows], any may be NULL (1, 0, 0).  d_n_prompt NULL: all generated.
 * Ids outside [0, vocab) are ignored; token_start / bias_start outside [0, n_tokens / n_biases] are clamped.  n_tokens and n_biases
 * are below 2^30.
 * Computed in 32 bits, rounded once to out_dtype (dtype or F32).  d_out may be d_logits with the same stride and type. */
typedef struct {
    const void *d_logits;
    void *d_out;
    const int32_t *d_tokens, *d_token_start, *d_n_prompt;
    const float *d_repetition, *d_frequency, *d_presence;
    const int32_t *d_bias_ids, *d_bias_start;
    const float *d_bias;
    const int32_t *d_mask;
    int64_t logits_stride, out_stride, mask_stride;
    uint32_t rows, vocab, n_tokens, n_biases, dtype, out_dtype;
} ckks_clear_logits_t;
int ckks_clear_logits(const ckks_clear_logits_t *a, void *stream);

/* ---- key / value cache of 8 bits ------------------------------------------
 * Pages whose entries are a byte each, a code, and whose rows have one byte more for each 32 entries of a head (the
 * last block of a head may be shorter): the block's power of two.  An entry stands for code * 2^(power - 127), and the whole block for
 * not-a-number where the power is 255.  Formats: CKKS_CLEAR_E4M3 (sign, 4 bits of exponent, 3 of mantissa, largest 448, no infinity,
 * 0x7f and 0xff not-a-number), CKKS_CLEAR_I8 (two's complement).
 * d_k, d_v [n_pages][kv_heads][page_size][head_dim] bytes and d_k_power, d_v_power [n_pages][kv_heads][page_size][ceil(head_dim / 32)]
 * bytes, each by its strides {page, head, token}; limits, addressing of the batch and what values out of range do are those of
 * ckks_clear_pages_t.  dtype: the type of queries, new rows and results. */
#define CKKS_CLEAR_E4M3 16u
#define CKKS_CLEAR_I8 17u
typedef struct {
    uint8_t *d_k, *d_v, *d_k_power, *d_v_power;
    int64_t k_stride[3], v_stride[3], k_power_stride[3], v_power_stride[3];
    uint32_t n_pages, page_size, kv_heads, head_dim, format, dtype;
} ckks_clear_packed_t;

/* Writes the new tokens' keys and values into their pages; keys and queries are normed and rotated first:
 *   with d_k_norm (d_q_norm), [head_dim] of norm_dtype (F32 or dtype):  x = x / sqrt(mean(x^2) + eps) * weight over each head's entries
 *   rotation as in ckks_clear_cache_append
 *   each block of 32 entries: e = the smallest number >= -100 with max |x| <= M 2^e, M = 448 (E4M3) or 127 (I8),
 *   power = e + 127, codes = x / 2^e rounded to the nearest, ties to even; of a block that dtype holds, to the nearest whose value it
 *   holds too (finite entries up to the type's largest stay finite).
 * A block that holds an infinity, a NaN or an entry of 2^128 or more is stored as power 255 and codes 0.  Norm and rotation are
 * computed in 64 bits; keys meet no other rounding than that to their code, queries are rounded to 32 bits and to dtype.
 * Rotated entries without an angle are NaN, and so is, in the cache, their block.  What is not stored, what may lie in what, rows in
 * no sequence: as in ckks_clear_cache_append. */
typedef struct {
    ckks_clear_packed_t pages;
    ckks_clear_batch_t batch;
    const void *d_new_k, *d_new_v, *d_q;
    void *d_q_out;
    const void *d_k_norm, *d_q_norm;
    const float *d_cos, *d_sin;
    const int32_t *d_positions;
    int64_t new_k_stride[2], new_v_stride[2], q_stride[2], q_out_stride[2];
    uint32_t heads, rot, n_pos, flags, norm_dtype;
    float eps; /* >= 0 */
} ckks_clear_packed_append_t;
int ckks_clear_packed_append(const ckks_clear_packed_append_t *a, void *stream);

/* Attention of the new tokens over the packed pages, in every respect as ckks_clear_attend over pages that hold, in dtype, what the
 * codes stand for (beyond its range F16 is infinite, as a conversion is; numbers below 2^-126 may count as 0). */
typedef struct {
    ckks_clear_packed_t pages;
    ckks_clear_batch_t batch;
    const void *d_q;
    void *d_out;
    float *d_lse;
    void *d_work;
    uint64_t work_bytes;
    int64_t q_stride[2], out_stride[2];
    uint32_t heads, window, flags;
    float scale;
} ckks_clear_packed_attend_t;
uint64_t ckks_clear_packed_attend_work_bytes(const ckks_clear_packed_attend_t *a);
int ckks_clear_packed_attend(const ckks_clear_packed_attend_t *a, void *stream);

/* Reads the new tokens' keys and values (all of a sequence's, if as many rows as kv_len are asked for) back: the values that the codes
 * stand for, in dtype.  A token at a position below 0 or in a page outside [0, n_pages) reads as zeros; rows in no sequence
 * are not written.  Rows that ckks_clear_packed_append wrote give the same values when they are read and appended again, in F16 where it
 * holds them: its largest number is 65504, which normed keys may pass, and it rounds small ones to multiples of 2^-24.
 * d_k_out, d_v_out [n_tokens][kv_heads][head_dim] by strides {token, head}, either NULL; they share no entry. */
typedef struct {
    ckks_clear_packed_t pages;
    ckks_clear_batch_t batch;
    void *d_k_out, *d_v_out;
    int64_t k_out_stride[2], v_out_stride[2];
} ckks_clear_packed_read_t;
int ckks_clear_packed_read(const ckks_clear_packed_read_t *a, void *stream);

/* ---- the next token --------------------------------------------------------
 * Draws a token of each row of logits l by a number u of [0, 1) that the caller gives:
 *   w = exp((l - max l) / temperature)
 *   top_k > 0:    the top_k tokens with the largest logits are kept (of equal ones the lowest ids)
 *   top_p < 1:    of these, largest first, a token is kept while those before it sum to less than top_p times the sum of all of
 *                 them (the first always is)
 *   min_p > 0:    of these, a token is kept if w >= min_p  (1 or more: the largest ones)
 *   token = the lowest id for which the sum of w over the kept tokens up to it exceeds u times the sum over all;
 *   prob = its w over that sum
 * d_temperature, d_top_p, d_min_p, d_u: f32 [rows], d_top_k: int32 [rows]; all but d_u may be NULL (1; no limit).  A
 * temperature of 0 or below takes the largest logit (the lowest id; prob 1), top_p of 0 or below the first token only.  u below 0
 * counts as 0, u of 1 or more takes the last token kept; NaN counts as no limit, temperature 1, u = 0.
 * A logit of -infinity or NaN is never drawn, and one whose w is below 2^-64 counts as -infinity; logits of +infinity are drawn alike.
 * A row without any other gets token -1, prob 0.  Sums are held in 64 bits, off by less than 2^-40 of themselves, and joined in a fixed
 * order: the same inputs give the same token.  d_prob: f32 [rows] or NULL.  vocab: 1 to 2^20, rows below 2^31. */
typedef struct {
    const void *d_logits;
    int32_t *d_token;
    float *d_prob;
    const float *d_u, *d_temperature, *d_top_p, *d_min_p;
    const int32_t *d_top_k;
    int64_t logits_stride;
    uint32_t rows, vocab, dtype, reserved;
} ckks_clear_sample_t;
int ckks_clear_sample(const ckks_clear_sample_t *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* CKKS_CLEAR_H */
