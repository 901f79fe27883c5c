/*
 * torpor_ops.h - operators of libtorpor that can be called by themselves, beside the models of torpor.h
 * that use them: linear layers with 4-bit weights (models of dtype TP_W4G32, TP_W4G64 and TP_W4G128), and
 * attention with lengths, a window and sinks (BERT models with TP_BERT_ATTENTION).
 *
 * Conventions, as in torpor.h: TP_OK or a negative TP_E_* code with a message in tp_last_error(); invalid
 * arguments launch nothing; device pointers are plain addresses, streams hipStream_t as void* (NULL: the
 * null stream). Calls are asynchronous on `stream`, allocate nothing, keep nothing from one call for the next, may be
 * captured into a graph and may come from several host threads. A call runs on the device of
 * `stream` (NULL: the current device), which must be able to reach every buffer.
 *
 * Scratch: `work` (256-byte aligned, may be NULL) lets a call split a long sum over more workgroups and add
 * the parts afterwards. A call uses what fits; with less, or none, it computes the same, slower and in another order
 * of addition. Its contents need no preparation and are undefined afterwards. Calls that may overlap (on
 * different streams, or replays of different graphs) need scratch of their own. TPO_WORK_BYTES is as much as any call uses.
 * (tpo_attention splits its keys; tpo_linear_w4 splits its columns inside a workgroup and leaves the scratch alone.)
 */
#ifndef TORPOR_OPS_H
#define TORPOR_OPS_H

#include "torpor.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TPO_WORK_BYTES (32u << 20)

/* ---- 4-bit weights ----
 *
 * A matrix W[N][K] as codes 0..15, each the value plus 8, and a bf16 scale for every `group` consecutive columns of a row
 * (group 32, 64 or 128, K a multiple of it): W[n][k] = scale[n][k / group] (code[n][k] - 8).
 *
 * Plain order, as checkpoints hold it: codes [N][K / 2] bytes, the even column in the low half; scales [N][K / group].
 * Blocked order, as the kernels read it: N padded to N' = a multiple of 16, K to K' = a multiple of 128. The block of
 * rows 16 i.. and columns 128 j.. is the 1024 bytes at (i K' / 128 + j) 1024; in it the little-endian 32-bit word
 * 4 (16 q + r) + t (q, t < 4, r < 16) holds row r, columns 32 t + 8 q + c for c = 0..7, column c in the 4 bits at
 * 4 (c / 2) + 16 (c % 2). Scales: [N' / 16][K' / group][16], the row last. Padding: code 8, scale 0. */

/* Bytes of the blocked order. Host only. TP_E_INVAL for a shape that is not supported (N or K < 1, N > 2^24,
 * K > 2^20, a group that is not 32, 64 or 128 or does not divide K). */
TP_API tp_status tpo_w4_bytes(int32_t N, int32_t K, int32_t group, uint64_t* code_bytes, uint64_t* scale_bytes);

/* Plain order to blocked order, both in host memory. codes_out and scales_out: tpo_w4_bytes, no overlap with the input. */
TP_API tp_status tpo_w4_pack(const uint8_t* codes, const uint16_t* scales, int32_t N, int32_t K, int32_t group,
                             uint8_t* codes_out, uint16_t* scales_out);

/* Rounds fp32 weights [N][K] to the plain order, in host memory: a group's scale is its largest magnitude / 7
 * rounded to bf16, codes the nearest of the 15 values -7..7 (ties to even) to weight / scale; a group of zeros has
 * scale 0. TP_E_INVAL if a weight is infinite or NaN, or so large that the scale is not finite. */
TP_API tp_status tpo_w4_quantize(const float* w, int32_t N, int32_t K, int32_t group, uint8_t* codes, uint16_t* scales);

/* y[m][n] = act(sum_k x[m][k] W[n][k] + bias[n] + res[m][n]), m < M, n < N.
 * x, res bf16, y bf16 or fp32 (y_dtype), rows ldx, ldr and ldy elements apart; bias bf16 or NULL, res or NULL. Products
 * and sums are exact bf16 products in fp32 sums, scales applied to each group's sum, one rounding at the end.
 * x starts at a 16-byte boundary and ldx is a multiple of 8 below 2^23; wq and scales start at 16-byte boundaries. y may
 * be res (same ldr and ldy, both bf16); apart from that outputs do not overlap inputs. M = 0 does nothing. M in whole 128s
 * times N in whole 256s is below 2^38. An infinite or NaN x[m][k] makes row m NaN, whatever the activation; finite inputs of
 * which 31 times a group's sum of |x| reaches 2^128 may overflow. */
typedef struct {
  const void* x;
  int64_t ldx;
  const void* wq;            /* blocked order */
  const void* scales;
  const void* bias;
  const void* res;
  int64_t ldr;
  void* y;
  int64_t ldy;
  int32_t y_dtype;           /* TP_BF16 or TP_F32 */
  int32_t M, N, K, group;
  int32_t act;               /* TP_ACT_* */
  void* work;
  uint64_t work_bytes;
} tpo_linear_w4_args;
TP_API tp_status tpo_linear_w4(const tpo_linear_w4_args* a, void* stream);

/* ---- attention ----
 *
 * Sequence b has q_lens[b] new tokens (queries), the last of its kv_lens[b] tokens in all (NULL: q_len, kv_len for every
 * sequence; values are clamped to [0, q_len] and [0, kv_len]). Query i stands at p = kv_lens[b] - q_lens[b] + i, and sees
 * key j < kv_lens[b] if
 *   (causal: j <= p) and (j < sinks, or p - window_left <= j <= p + window_right; a negative bound is none).
 * out = sum over the seen j of softmax_j(scale q k_j) v_j; a query that sees no key (or whose
 * scores are all -infinity) gives zeros. Keys that a query does not see do not touch it, whatever they hold. Rows
 * i >= q_lens[b] of out are left as they are. Scores, exponentials and sums are fp32; each exponential is rounded to bf16
 * before it multiplies v_j (not in the sum that divides), the result once more: off by 2^-8 of sum softmax_j |v_j| and 2^-8 of
 * itself at most. Values of which 2^8 times a query's sum reaches 2^128 may overflow. An infinity or NaN in a seen v_j shows in its
 * column, however little it weighs.
 * q and out: heads of head_dim (64 or 128) bf16 values; k and v: kv_heads, of which each serves heads / kv_heads
 * consecutive query heads. Strides in elements between sequences, tokens and heads ([0], [1], [2]); the values of a
 * head are contiguous. Every head's values start at a 16-byte boundary (strides are multiples of 8; k's and v's between tokens at most 2^23). A stride of 0
 * (a broadcast input) is allowed except in out; the stride of a dimension of one entry is not used. out's heads overlap
 * neither each other nor an input. batch * q_len * heads is below 2^30, batch * kv_heads below 2^22. q_len or batch 0 does nothing. */
typedef struct {
  const void *q, *k, *v;
  void* out;
  int64_t q_stride[3], k_stride[3], v_stride[3], out_stride[3];
  const int32_t* q_lens;     /* device, [batch], or NULL */
  const int32_t* kv_lens;
  int32_t batch, heads, kv_heads, head_dim, q_len, kv_len;
  int32_t causal;
  int32_t window_left, window_right, sinks;
  float scale;               /* > 0, at most 2^127; 0: 1 / sqrt(head_dim) */
  void* work;
  uint64_t work_bytes;
} tpo_attention_args;
TP_API tp_status tpo_attention(const tpo_attention_args* a, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TORPOR_OPS_H */
