/*
 * torpor_serve.h - operators of libtorpor for serving tokens to many tenants, called by themselves beside those of
 * torpor_ops.h: a paged key/value cache (append, read, attention over it) and low-rank adapters of many requests beside a
 * shared projection.
 *
 * Conventions, scratch and streams as in torpor_ops.h: TP_OK or a negative TP_E_* code with a message in tp_last_error(); invalid
 * arguments launch nothing; calls are asynchronous on `stream`, allocate nothing, keep nothing from one call for the next,
 * may be captured into a graph and may come from several host threads; `work` (256-byte aligned, may be NULL) needs no preparation,
 * is undefined afterwards, and calls that may overlap need scratch of their own. A call uses what fits; TPO_WORK_BYTES is what the calls are
 * made for. (More lets attention split many rows' long caches further, and adapters take more than 64,000 rows at once.)
 */
#ifndef TORPOR_SERVE_H
#define TORPOR_SERVE_H

#include "torpor_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- a paged key/value cache ----
 *
 * A pool of `pages` pages of page_size tokens (a power of two, 16 to 4096), shared by any number of sequences. table[b][c]
 * (device, rows table_stride apart, max_pages entries each) is the page that holds tokens c page_size .. of sequence b. An entry
 * outside [0, pages) is no page: a token there is not written, reads as zeros and is seen by no query. So a page that a
 * window has left may be taken from its sequence, with -1 in its place.
 *
 * Values of page p, token t of it, key/value head h start at element p stride[0] + t stride[1] + h stride[2] and are contiguous
 * (head_dim 64 or 128), at 16-byte boundaries: strides in whole 16 bytes, that between tokens at least head_dim and at most
 * 2^23, (page_size - 1) times it below 2^30. TP_BF16: the values. TPS_E4M3: 8-bit floats (4 exponent, 3 mantissa bits, largest 448, no infinities) of which
 * each token's head has a scale 2^(x - 127), NaN if x is 255, x = exps[p][0 for k, 1 for v][h][t] (contiguous, 4-byte aligned, pages 2 kv_heads
 * page_size below 2^31). tps_cache_append takes the smallest power of two, 2^-126 or more, for which no value's magnitude divided by it is
 * over 448; values divided by it are rounded to the nearest, ties to even (off by at most 2^-4 of themselves, or 2^-10 of the
 * scale). An infinity or NaN becomes NaN, and the scale is that of the others.
 *
 * Sequence b holds kv_lens[b] tokens, the new ones included; q_lens[b] of them are new, the last ones (NULL: q_len). Row i of the new ones
 * is token kv_lens[b] - q_lens[b] + i; one in front of token 0, or behind the table's last, is in no page. Both lengths are
 * device values, q_lens clamped to [0, q_len], and a negative kv_lens counts as 0. */

#define TPS_E4M3 16

typedef struct {
  void *k, *v;
  uint8_t* exps;             /* TPS_E4M3, else NULL */
  int64_t k_stride[3], v_stride[3];
  int32_t dtype;             /* TP_BF16 or TPS_E4M3 */
  int32_t pages, page_size, kv_heads, head_dim;
  int32_t reserved;          /* 0 */
} tps_cache;

/* Rows of keys and values, bf16, in and out of the cache: strides in elements between sequences, rows and heads, the values of a head
 * contiguous, at 16-byte boundaries (strides multiples of 8; those of a dimension of one entry are not used).
 * tps_cache_append writes rows i < q_lens[b] of k and v into the pages. Two rows of one call that stand for the same place (sequences
 * that share the page they append to) leave a mixture of the two there. Pages that it does not write are not touched.
 * tps_cache_read writes rows i < q_lens[b] from the pages (q_lens = kv_lens: whole sequences); other rows are left
 * as they are. 8-bit values that a scale takes beyond bf16's range are infinities, those below it are rounded. Rows do
 * not overlap each other (when written) nor the cache. batch * q_len * kv_heads is below 2^26, batch *
 * kv_heads below 2^22. */
typedef struct {
  tps_cache cache;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* q_lens;     /* device, [batch], or NULL */
  const int32_t* kv_lens;    /* device, [batch] */
  void *k, *v;
  int64_t k_stride[3], v_stride[3];
  int32_t batch, q_len, max_pages;
  int32_t reserved;          /* 0 */
} tps_cache_rows_args;
TP_API tp_status tps_cache_append(const tps_cache_rows_args* a, void* stream);
TP_API tp_status tps_cache_read(const tps_cache_rows_args* a, void* stream);

/* Attention of the new tokens over the cache, which holds them already. The query of token p sees token j of its sequence if j <= p
 * and (j < sinks or window < 0 or j >= p - window), and j is in a page. out = sum over the seen j of softmax_j(scale q k_j) v_j; a
 * query that sees no key, or whose scores are all -infinity, gives zeros. Keys that a query does not see do not touch it, whatever
 * their places hold. Rows i >= q_lens[b] of out are left as they are. kv_len is at least every sequence's length
 * (longer ones are cut to it; below 2^30; max_pages page_size, or 2^30 - 1, is always enough, and a closer bound plans the call better).
 * Scores, exponentials and sums are fp32. Each exponential (times the scale of its 8-bit v_j) multiplies v_j as two bf16 parts, which leave
 * 2^-15 of it; the result is rounded once: off by 2^-15 of sum softmax_j |v_j| and 2^-8 of itself at
 * most. Values of which 2^8 times a query's sum reaches 2^128 may overflow, and so may the results of a query that sees an
 * 8-bit v_j of scale 2^120 or more; scales below 2^-100 leave fewer bits, nothing of what is below 2^-126. An infinity or NaN in a seen v_j makes its
 * column infinite or NaN.
 * q and out: bf16, `heads` heads (each key/value head serves heads / kv_heads consecutive ones), strides in elements between
 * sequences, tokens and heads, as in tpo_attention (out's not 0; it overlaps no input). Made for single tokens and a few drafted ones: keys are
 * read once for every 64 rows of q_len heads / kv_heads. batch * q_len * heads is below 2^27, batch * kv_heads below 2^22.
 * q_len or batch 0 does nothing. */
typedef struct {
  tps_cache cache;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* q_lens;     /* device, [batch], or NULL */
  const int32_t* kv_lens;    /* device, [batch] */
  const void* q;
  void* out;
  int64_t q_stride[3], out_stride[3];
  int32_t batch, heads, q_len, kv_len, max_pages;
  int32_t window, sinks;
  float scale;               /* > 0, at most 2^127; 0: 1 / sqrt(head_dim) */
  void* work;
  uint64_t work_bytes;
} tps_cache_attention_args;
TP_API tp_status tps_cache_attention(const tps_cache_attention_args* a, void* stream);

/* ---- low-rank adapters of many requests ----
 *
 * y[m][n] = act(base[m][n] + scale_a sum_{r < rank_a} (sum_k x[m][k] A_a[r][k]) B_a[n][r]), a = adapter[m], m < M, n < N.
 * A row whose adapter is not in [0, adapters) has none: y = act(base). Rows may name adapters in any order; adapters that no
 * row names are not read. Rows of many adapters in turn are put in order for pools of fewer than 4096 adapters and up to 2^17 rows at once; beyond, the
 * adapters of 64 rows are taken one after the other, and slowly.
 * x bf16, rows ldx apart (a multiple of 8); y and base bf16 or fp32 (dtype), rows ldy and ldbase apart, base NULL: zeros. y may be base (same row
 * stride), else it overlaps no input. A [adapters][R][K] and B [adapters][N][R] bf16, adapters a_stride and b_stride elements apart, rows
 * contiguous; R a multiple of 8 up to 128, K of 8 up to 2^20. x, A and B start at 16-byte boundaries, a_stride
 * and b_stride are multiples of 8. ranks (device, NULL: R for all) are clamped to [0, R]: what lies behind an adapter's rank is not
 * used, whatever it holds. scales (device, fp32, NULL: 1).
 * Products are exact, sums fp32; the inner sums times the scale are rounded to two bf16 parts (2^-16 of themselves; three, 2^-24, for fp32 results)
 * for the second product; one rounding of the result. A row's result depends on its own values and adapter alone, whatever others
 * hold and wherever in the call it stands (M, N and work_bytes choose the order of addition, so that between calls that differ in these its
 * last bits may differ); an infinity or NaN among these makes results infinite or NaN. Inner sums beyond bf16's range overflow. M = 0 does nothing. M in whole 16s times N in whole 256s is below 2^36.
 * work holds the inner sums; with less of it than 4 M (R + 2) bytes rows are taken part after part, and with less than 1024 of them need (4096 where
 * N is 256 or less), or none, the inner sums are computed anew for every 256 outputs. */
typedef struct {
  const void* x;
  int64_t ldx;
  const void *a, *b;
  int64_t a_stride, b_stride;
  const int32_t* adapter;    /* device, [M] */
  const int32_t* ranks;      /* device, [adapters], or NULL */
  const float* scales;       /* device, [adapters], or NULL */
  const void* base;
  int64_t ldbase;
  void* y;
  int64_t ldy;
  int32_t dtype;             /* of base and y: TP_BF16 or TP_F32 */
  int32_t M, N, K, R, adapters;
  int32_t act;               /* TP_ACT_* */
  int32_t reserved;          /* 0 */
  void* work;
  uint64_t work_bytes;
} tps_lora_args;
TP_API tp_status tps_lora(const tps_lora_args* a, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TORPOR_SERVE_H */
