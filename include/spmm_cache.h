/*
 * spmm_cache.h - C ABI of the paged key/value cache between the sparse projections of a decoder.
 *
 * A decoder layer runs   spmm_run (stacked Q/K/V weights)  ->  spmm_cache_append  ->  spmm_cache_attend
 * ->  spmm_run (output projection):  append takes the projection's output as spmm_run writes it (rows =
 * features, tokens contiguous), attend writes its result the same way, as U8 where it is to be the next
 * spmm_run's activations.  spmm_cache_fork and spmm_cache_compact change which pages belong to which
 * sequence; they run on the device as well, and no call waits for the host.
 *
 * The cache is memory of the caller, in pages of `page_tokens` tokens:
 *   k        [n_layers][n_pages][n_heads][page_tokens][head_dim]    BF16 or S8
 *   v        [n_layers][n_pages][n_heads][head_dim][page_tokens]    (tokens contiguous, like activations)
 *   k_scale, v_scale  [n_layers][n_pages][n_heads][page_tokens]     binary32, S8 only:  value = code * scale
 *   bounds   [n_layers][n_pages][n_heads][2][head_dim]              BF16: largest and smallest value of each dim of a page's keys
 *   weight   [n_layers][n_pages][n_heads][page_tokens]              binary32: attention that a token has had so far
 * The last two are there where long contexts are read in part (spmm_cache_score) or cut down (spmm_cache_evict); fork, compact
 * and copy move all parts of a page.
 * One page table serves all layers: row b names the pages of sequence b in order, token p lies in page
 * table[b][p / page_tokens]; entries that are not in use are -1.
 *
 * Conventions are those of spmm.h: C linkage, statuses, outputs untouched on error, every pointer is said
 * to be host or device, device pointers stay the caller's until the launch that uses them has finished, and
 * launches are asynchronous on the stream that is handed over.  Structures may gain fields at their ends (as spmm_cache_t
 * has: bounds, weight), and nothing says which a caller knows: callers are compiled against the header of the library
 * that they load, and set what they do not use to 0.  What lies in device memory (tables, lengths)
 * cannot be checked by the host: the kernels bring it into range, so that a bad entry gives wrong values and
 * never an access outside the operands.
 */
#ifndef SPMM_CACHE_H_
#define SPMM_CACHE_H_

#include "spmm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SPMM_CACHE_BF16 = 0, SPMM_CACHE_S8 = 1 } spmm_cache_type_t;

/* Bfloat16 outputs: attend only (spmm_run has none). */
#define SPMM_OUT_BF16 4

typedef struct {
    void *k, *v;                /* device, 16-byte aligned                                       */
    float *k_scale, *v_scale;   /* device, S8 only (16-byte aligned), otherwise NULL             */
    spmm_cache_type_t type;
    int32_t n_layers;
    int32_t n_heads;            /* key/value heads                                               */
    int32_t head_dim;           /* multiple of 16, at most 128 (else SPMM_E_UNSUPPORTED)         */
    int32_t page_tokens;        /* 16, 32, 64, 128 or 256 (else SPMM_E_UNSUPPORTED)              */
    int64_t n_pages;            /* 1 .. 2^31 - 1                                                 */
    void *bounds;               /* device, 16-byte aligned, or NULL: no call needs them but
                                   spmm_cache_bounds and spmm_cache_score                        */
    float *weight;              /* device, 16-byte aligned, or NULL: no call needs them but
                                   spmm_cache_weigh and spmm_cache_evict                         */
} spmm_cache_t;

/* A batch of sequences and their new tokens.  The new tokens of sequence b are the columns q_start[b] ..
 * q_start[b + 1] - 1 of the operands, and the last ones of its kv_len[b] tokens: column t is at position
 * kv_len[b] - (q_start[b + 1] - t).  Columns of no sequence, and columns at a negative position, are
 * padding: append gives zeros for them in q and stores nothing else; attend gives zeros for the latter and leaves
 * columns of no sequence as they were. */
typedef struct {
    int64_t n_seqs;
    const int32_t *q_start;     /* device [n_seqs + 1], not decreasing                           */
    const int32_t *kv_len;      /* device [n_seqs], the new tokens included; what lies beyond the
                                   table's width is not there                                    */
    const int32_t *table;       /* device [n_seqs][ld_table], page numbers                       */
    int64_t ld_table;           /* pages of a row; ld_table * page_tokens < 2^30                 */
} spmm_batch_t;

/* How new queries, keys and values are made of the projection's output x [(q_heads + 2 n_heads) head_dim][ldx]
 * (first the query heads, then the key heads, then the value heads).  For queries and keys:
 *   value  = x                           F32      value = (x - x_zero_point) * x_scale      S8 / U8
 *   y      = value * rsqrt(mean over the head's dims of value^2 + eps) * weight      with a weight, else y = value
 *   rotated, with a table, by its position's angles: pairs (a, b) -> (a cos - b sin, b cos + a sin), in the
 *   first rope_dim dims; pair i is (y[i], y[i + rope_dim / 2]), or (y[2 i], y[2 i + 1]) where interleaved.
 * Positions outside the rotation table give NaN.  Values are not normalised or rotated.  All of it is
 * computed in binary32 and rounded once: queries to bfloat16, keys and values to the cache's type.
 * S8: scale = amax / 127 over the head's dims of a token, code = rint(value * (127 / amax)).  Where these are not all
 * finite, the scale is not either and all codes are 0, so that the token's head is NaN as a whole. */
typedef struct {
    int32_t q_heads;            /* multiple of the cache's n_heads                               */
    spmm_out_t x_type;          /* F32, S8 or U8                                                 */
    float x_scale;              /* S8 / U8                                                       */
    int32_t x_zero_point;       /* S8 / U8                                                       */
    const float *q_weight;      /* device [head_dim] or NULL                                     */
    const float *k_weight;      /* device [head_dim] or NULL                                     */
    float eps;                  /* >= 0                                                          */
    const float *rope;          /* device [rope_len][rope_dim / 2][2] (cos, sin) or NULL         */
    int64_t rope_len;
    int32_t rope_dim;           /* even, at most head_dim                                        */
    int32_t interleaved;
    const int32_t *positions;   /* device [T]: where a column is rotated to; NULL: its position
                                   in the cache                                                  */
} spmm_append_t;

/* Writes the T new tokens' queries to q (device, bfloat16 [T][q_heads][head_dim], 16-byte aligned) and their
 * keys and values to the pages of layer `layer`.  x: device, ldx >= T in elements. */
spmm_status_t spmm_cache_append(const spmm_cache_t *cache, int32_t layer, const spmm_batch_t *batch, const void *x,
                                int64_t T, int64_t ldx, const spmm_append_t *how, void *q, void *hip_stream);

/* Attention of the new tokens over their sequences' tokens in the cache:
 *   out[h][d][t] = sum_j p_j v_j[d],   p = softmax over the visible j of scale * (q_t . k_j),
 * query head h reading key/value head h / (q_heads / n_heads).  Token j is visible to the token at position
 * i if j < kv_len, with `causal` j <= i, and with a window j > i - window.  Where nothing is visible the
 * result is 0.  What is not visible has no influence, whatever it holds (NaN and infinities too).
 * Scores, softmax statistics and sums are held in binary32.  Operands of the products are rounded, whatever out_type is:
 *   BF16 caches: weights to bfloat16; the sum of weights is that of the rounded ones.
 *   S8 caches: queries, and weights, to binary16, over powers of two.  Up to 32 columns a key/value head (the query heads that
 *   share it times max_new) codes are exact, weights are rounded with the values' scales in them, and the sum is of
 *   the unrounded ones; with more columns keys and values, code * scale, are rounded too, and the sum is of the rounded weights.
 *   What is below 2^-24 of the largest query, weight or scale it is multiplied beside is lost.
 * Values that are not finite reach the columns that see them, as infinities or NaN (an infinity whose weight is rounded to 0 gives NaN);
 * a score of NaN or +inf makes its column NaN, and so do scores of -inf alone.  A scale of keys that is not finite makes the
 * token's scores NaN.
 * One kernel is chosen for all sequences, by max_new: a batch that mixes prompts with single tokens of long contexts is
 * faster in two calls (q_start, kv_len and table can be entered at any sequence, q and out are the same), and a max_new far above
 * what there is costs as much as such a prompt would. */
typedef struct {
    int32_t q_heads;            /* multiple of the cache's n_heads                               */
    int64_t max_new;            /* most new tokens of any sequence, or an upper bound (>= 1); of a sequence
                                   with more, the first max_new columns are computed             */
    float scale;                /* > 0, finite                                                   */
    int32_t causal;
    int32_t window;             /* 0: none                                                       */
    int32_t out_type;           /* SPMM_OUT_F32, SPMM_OUT_BF16, SPMM_OUT_S8, SPMM_OUT_U8         */
    float out_scale;            /* S8 / U8: q = sat(rint(o * (1 / out_scale)) + out_zero_point)  */
    int32_t out_zero_point;
} spmm_attend_t;

/* Bytes of scratch that spmm_cache_attend takes for such a call; *bytes is HOST memory. */
spmm_status_t spmm_attend_work_bytes(const spmm_cache_t *cache, int64_t n_seqs, int64_t T, const spmm_attend_t *how,
                                     int64_t *bytes);

/* q: device, bfloat16 [T][q_heads][head_dim], 16-byte aligned, as append writes it.  out: device,
 * [q_heads * head_dim][ldo], ldo >= T.  work: device, spmm_attend_work_bytes bytes, 16-byte aligned;
 * needs no initialisation, holds nothing between calls, and calls on different streams need their own. */
spmm_status_t spmm_cache_attend(const spmm_cache_t *cache, int32_t layer, const spmm_batch_t *batch, const void *q,
                                int64_t T, const spmm_attend_t *how, void *out, int64_t ldo, void *work,
                                void *hip_stream);

/* The next generation of a batch's sequences: row j of the new table goes on from row parent[j] of the old one
 * (-1: from none) with its first kept = min(keep[j], kv_len[parent[j]]) tokens, and gets pages for want[j] tokens.
 * Old rows that are nobody's parent, and what was cut off, are freed; this one call forks, trims, frees and grows.
 *   - Pages that the kept tokens fill are shared by everyone who keeps them.
 *   - A page that kept tokens end inside will be written to, so it is one row's alone: it stays the lowest such
 *     row's if nobody keeps it as a whole page; every other row gets a copy (all layers).
 *   - New pages are the lowest numbers that the old table does not hold, given out by rows, in order.
 * table, table_out: device [n_rows_in][ld_table], [n_rows][ld_table], two different buffers (as kv_len and
 * kv_len_out are): the old generation stays readable, and the call can be repeated.  A page is in use if the old
 * table names it anywhere, so rows that no sequence runs on can hold prefixes.  kv_len_out[j] = kept.
 * info: device [4]: pages that were missing, pages copied, pages in use by the new table, 0.  If pages are missing
 * (or a want exceeds the width), nothing but info is written.  work: as for attend, spmm_cache_work_bytes bytes. */
spmm_status_t spmm_cache_fork(const spmm_cache_t *cache, const int32_t *table, int64_t ld_table, const int32_t *kv_len,
                              int64_t n_rows_in, const int32_t *parent, const int32_t *keep, const int32_t *want,
                              int64_t n_rows, int32_t *table_out, int32_t *kv_len_out, int32_t *info, void *work,
                              void *hip_stream);

/* Moves the pages in use to the front of the pool: with n of them, those numbered n and higher go to the free
 * numbers below n, the lowest to the lowest, in all layers, and table_out is the table with the new numbers (it
 * may be `table` itself).  Pages that stay are not touched.  info: device [4]: 0, pages moved, pages in use, 0. */
spmm_status_t spmm_cache_compact(const spmm_cache_t *cache, const int32_t *table, int64_t ld_table, int64_t n_rows,
                                 int32_t *table_out, int32_t *info, void *work, void *hip_stream);

/* Copies page src[i] to page dst[i] in all layers, i < n (device arrays).  Pairs with a number outside the pool
 * are left out; no page may be written twice, or be read and written, in one call. */
spmm_status_t spmm_cache_copy(const spmm_cache_t *cache, const int32_t *src, const int32_t *dst, int64_t n,
                              void *hip_stream);

/* Bytes of scratch of spmm_cache_fork (n_rows: of the new table) and spmm_cache_compact; *bytes is HOST memory. */
spmm_status_t spmm_cache_work_bytes(const spmm_cache_t *cache, int64_t n_rows, int64_t *bytes);

/* ---- Long contexts: reading the pages that matter, dropping the tokens that do not ----------------------------
 *
 * A step of new tokens   spmm_cache_append -> spmm_cache_bounds -> spmm_cache_score -> spmm_cache_select ->
 * spmm_cache_attend_selected   reads the pages of a list for each new token and key/value head instead of all of them.
 * spmm_cache_weigh adds up what attention each token gets, and spmm_cache_evict keeps the tokens that got most of it.
 * Limits (else SPMM_E_UNSUPPORTED): 65535 sequences or rows in spmm_cache_bounds, _weigh and _evict, T * n_heads <= 2^22 and lists of up to 2^20
 * pages in spmm_cache_score, _select and _attend_selected (2^40 numbers of lists in all; in _attend_selected, with G = q_heads / n_heads, also
 * T * n_heads * ceil(G / 16) * ceil(pages / 1024) < 2^24), lds <= 2^30, n_layers * n_heads <= 2^20 in spmm_cache_evict.
 * "Visible" is what it is in spmm_cache_attend (kv_len, causal, window), token by token; columns at a negative position see nothing. */

/* Bounds of the pages that the batch's new tokens lie in (of layer `layer`): of each head and dim the largest and the
 * smallest of the keys' values (code * scale in S8 caches, in binary32, rounded to bfloat16) of all tokens of the page below kv_len;
 * where one of them is not finite, both are NaN.  The call follows spmm_cache_append of the same batch.  A batch that says that all
 * tokens of its sequences are new (q_start[b + 1] - q_start[b] = kv_len[b]) has all of their pages' bounds made again, as after an
 * eviction.  (Pages that fork copies and cuts keep the bounds of all their tokens, which hold for those that are left, until new ones come to them.)
 * T: columns of the batch; a number that is too small or too large costs time and nothing else. */
spmm_status_t spmm_cache_bounds(const spmm_cache_t *cache, int32_t layer, const spmm_batch_t *batch, int64_t T, void *hip_stream);

/* Which pages a new token reads. */
typedef struct {
    int32_t q_heads;            /* multiple of the cache's n_heads                               */
    int32_t pages;              /* most pages of a list (>= 1)                                   */
    int32_t first, last;        /* >= 0, together at most `pages`: so many of the first and of the last
                                   pages with a visible token are taken whatever their scores are */
    int32_t causal;
    int32_t window;             /* 0: none                                                       */
} spmm_select_t;

/* scores[t][h][i] (device, binary32 [T][n_heads][lds], lds >= ld_table, 4-byte aligned): of every column t, key/value head h and
 * page i of its sequence's row with a visible token, an upper bound (in S8 caches but for the bounds' rounding) of the products q . k of the page's keys:
 *   max over the query heads of h of   sum_d q_d > 0 ? q_d hi_d : q_d lo_d,
 * binary32 sums of products of the bounds hi, lo; NaN where a bound is.  Pages without a visible token, up to ld_table: -inf.  Columns of no
 * sequence are left as they were.  q: as for spmm_cache_attend.  (pages, first and last are not read, but checked.)
 * One kernel is chosen, by the mean number of columns of a sequence: a batch that mixes chunks with single tokens is faster in two calls (63 single tokens
 * and a chunk of 500, 8 thousand tokens each: 38 us, 73 in one), which give the same scores. */
spmm_status_t spmm_cache_score(const spmm_cache_t *cache, int32_t layer, const spmm_batch_t *batch, const void *q, int64_t T,
                               const spmm_select_t *how, float *scores, int64_t lds, void *hip_stream);

/* lists[t][h] (device, int32 [T][n_heads][pages]): of the pages of a column's row with a visible token the first `first`, the last
 * `last`, and those of highest score, `pages` in all or as many as there are: in ascending order, then -1.  Of equal
 * scores the lower page is taken; NaN counts as the highest.  Columns of no sequence are left as they were.  The scores may come from
 * anywhere; those of spmm_cache_score are for the same causal and window. */
spmm_status_t spmm_cache_select(const spmm_cache_t *cache, const spmm_batch_t *batch, const float *scores, int64_t T, int64_t lds,
                                const spmm_select_t *how, int32_t *lists, void *hip_stream);

/* Bytes of scratch that spmm_cache_attend_selected takes for such a call; *bytes is HOST memory. */
spmm_status_t spmm_selected_work_bytes(const spmm_cache_t *cache, int64_t T, const spmm_attend_t *how, int64_t pages, int64_t *bytes);

/* spmm_cache_attend over the pages of lists [T][n_heads][pages] (device, int32): column t's softmax for the query heads of h is over the visible
 * tokens of the pages lists[t][h] of its row.  Numbers below 0 or not below ld_table name no page; pages may come in any order, and one that is
 * named twice counts twice.  All columns of a sequence are computed (how->max_new is not read, but checked).  Results, out, ldo and work as for
 * spmm_cache_attend, but weights are not rounded to 16 bits: BF16 caches: values are multiplied by three bfloat16 numbers, whose sum is the weight.  S8
 * caches: codes are multiplied by two binary16 numbers, whose sum is 22 bits of a weight times its value's scale; queries to binary16, over a power of two.  What is below
 * 2^-24 of the largest query, or of the largest scale it is multiplied beside, is lost.  The sum of weights is that of the unrounded ones. */
spmm_status_t spmm_cache_attend_selected(const spmm_cache_t *cache, int32_t layer, const spmm_batch_t *batch, const void *q, int64_t T,
                                         const spmm_attend_t *how, const int32_t *lists, int64_t pages, void *out, int64_t ldo, void *work,
                                         void *hip_stream);

/* How attention is added up. */
typedef struct {
    int32_t q_heads;            /* multiple of the cache's n_heads                               */
    int64_t max_new;            /* the last max_new new tokens of a sequence count (>= 1)        */
    float scale;                /* > 0, finite: of the scores, as for spmm_cache_attend          */
    int32_t causal;
    int32_t window;             /* 0: none                                                       */
    float decay;                /* 0 .. 1: what stays of the weights of earlier calls            */
} spmm_weigh_t;

/* Bytes of scratch that spmm_cache_weigh takes for such a call (of the batch its n_seqs and ld_table count); *bytes is HOST memory. */
spmm_status_t spmm_weigh_work_bytes(const spmm_cache_t *cache, const spmm_batch_t *batch, int64_t T, const spmm_weigh_t *how, int64_t *bytes);

/* The cache's weights of layer `layer`, for every token j < kv_len of every sequence with new tokens, and every key/value head h:
 *   weight[j] = (j is one of the new tokens ? 0 : decay * weight[j]) + sum over the last max_new new tokens t and the query heads of h of
 *               softmax over the visible tokens of scale * (q_t . k)   at j  (0 where j is not visible).
 * So weights need no initialisation.  Sequences without a new token are left as they were.  Scores, statistics and sums are binary32, and nothing
 * is rounded to less (codes of S8 caches are exact in the products, and scales are on the scores).  A score of NaN or +inf makes its column's weights NaN,
 * and so do scores of -inf alone.  The order of the sums does not change from call to call.
 * A page that several rows with new tokens name, at the same place of each, as spmm_cache_fork makes them: its tokens' weights fade once and get the shares of
 * all of these rows (a token is new if it is one of the new tokens of one of them).  Weights of a page that rows name at different places, or a row twice, are not defined.
 * q: as for spmm_cache_attend.  work: spmm_weigh_work_bytes bytes, as for attend. */
spmm_status_t spmm_cache_weigh(const spmm_cache_t *cache, int32_t layer, const spmm_batch_t *batch, const void *q, int64_t T,
                               const spmm_weigh_t *how, void *work, void *hip_stream);

/* What stays. */
typedef struct {
    int32_t first, recent;      /* >= 0: so many of the first and of the last tokens stay, whatever their weights are */
    int64_t most;               /* most tokens of a row that stay, or an upper bound (>= 1)      */
} spmm_evict_t;

/* Keeps n = min(keep[b], kv_len[b], most) tokens of every row b, in every layer and key/value head of their own: the first min(first, n), then
 * the last ones, recent of them if n has room, and of the others those of the largest weight (of equal ones the earlier token; NaN counts as the largest).
 * They go, in their order, to the first n tokens of row b of table_to: keys, values, scales and weights, as they are.
 *   table, table_to  device [n_rows][ld_table].  table_to names the pages that take what stays: the same table (rows are then cut down in place, and
 *                    pages behind them can be freed by spmm_cache_fork), or pages that fork has given out, which neither `table` nor another row
 *                    names; no page may be in two rows that both write to it.  What table_to has no page for is lost.
 *   kept             device, int32 [n_layers][n_rows][n_heads][most]: the tokens that stay, ascending, then -1
 *   kv_len_out       device [n_rows], another buffer than kv_len: n
 * What stays is rotated to where it was, so later tokens are appended with `positions` (spmm_append_t) that go on counting from where the
 * sequence was before; a window of spmm_attend_t is one of places in the cache.  Bounds of the pages are not moved: see spmm_cache_bounds. */
spmm_status_t spmm_cache_evict(const spmm_cache_t *cache, const int32_t *table, int64_t ld_table, const int32_t *kv_len, int64_t n_rows,
                               const int32_t *keep, const spmm_evict_t *how, const int32_t *table_to, int32_t *kv_len_out, int32_t *kept,
                               void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SPMM_CACHE_H_ */
