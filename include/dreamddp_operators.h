/*
 * dreamddp_operators.h - C ABI of the operators of a transformer's forward and backward pass that are no plain matrix products:
 * norms, rotary positions, attention and the cross entropy of a language model's head.  They produce the gradients that
 * ddp_local_update and ddp_fused_sync_update[_layers] (dreamddp.h) consume, and like those
 *   - return a ddp_status, never throw, abort or print; ddp_last_error(NULL) has the message of this thread's last failure;
 *   - check their arguments on the host before any kernel is launched;
 *   - only enqueue kernels on the caller's stream (a hipStream_t as void*, NULL = the default stream) of the current device: they
 *     never allocate, free, copy to the host or synchronise, and may be captured into a HIP graph;
 *   - give the same bits for the same arguments: no result depends on the order of atomics.
 * They need no context.  Memory is the caller's: device pointers with the alignment of their element type, no output overlapping
 * an input unless stated.  dtype is DDP_F32 or DDP_BF16; sums, softmax statistics and norms are held in fp32 for both.
 * Strides count elements; the last dimension of every tensor is contiguous.  A `workspace` is device memory of at least
 * the bytes that the call's *_workspace function gives (< 0: -ddp_status), 256-byte aligned; nothing in it is kept between calls.
 */
#ifndef DREAMDDP_OPERATORS_H
#define DREAMDDP_OPERATORS_H

#include <stdint.h>

#include "dreamddp.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- layer norm and root-mean-square norm -------------------------------------------------------------------------
 * Per row x of [rows, cols]:  LAYER  mean = sum(x) / cols, rstd = 1 / sqrt(sum((x - mean)^2) / cols + eps), h = (x - mean) * rstd
 *                             RMS    mean = 0, otherwise the same;       y = h * weight (+ bias)
 * Backward, with g = dy * weight:  dx = rstd * (g - sum(g) / cols [LAYER] - h * sum(g * h) / cols)
 *                                  dweight = sum over rows of dy * h,  dbias = sum over rows of dy
 *   x, y, dy, dx       [rows, cols] of dtype; x_stride between the rows of x, y_stride between those of y and dy, dx_stride between those of
 *                      dx (0: x_stride)
 *   weight, bias, dweight, dbias  [cols] of dtype; bias nullable
 *   mean, rstd         fp32 [rows], written by the forward call and read by the backward call; mean nullable for RMS
 *   dx nullable; dweight and dbias nullable (no workspace is needed without both).  dx may be dy if their strides agree. */
enum { DDP_NORM_LAYER = 0, DDP_NORM_RMS = 1 };
typedef struct {
    int32_t kind, dtype;
    int64_t rows, cols;
    int64_t x_stride, y_stride;
    float eps;
    int64_t dx_stride;
} ddp_norm;
int ddp_norm_forward(const ddp_norm *norm, const void *x, const void *weight, const void *bias, void *y, float *mean, float *rstd, void *stream);
int64_t ddp_norm_backward_workspace(const ddp_norm *norm);
int ddp_norm_backward(const ddp_norm *norm, const void *dy, const void *x, const void *weight, const float *mean, const float *rstd, void *dx,
                      void *dweight, void *dbias, void *workspace, int64_t workspace_bytes, void *stream);

/* ---- rotary positions ---------------------------------------------------------------------------------------------
 * The first `rotated` channels of every head are pairs (a, b): channels i and i + rotated / 2 (HALF), or 2i and 2i + 1
 * (INTERLEAVED).  A pair at position p becomes (a c - b s, a s + b c), c and s the table's cosine and sine of row p, pair i; with
 * `inverse` (a c + b s, b c - a s), the transposed map, which takes the gradient of the output to that of the input.  The other channels
 * are copied.
 *   q, k        [tokens, heads, head_dim] with strides between tokens and heads; k nullable with k_heads = 0
 *   q_out, k_out  likewise, with strides of their own; may be q and k if the strides are the same
 *   table       fp32 [table_rows, rotated / 2, 2]: cosine, sine
 *   positions   nullable, [tokens] of int32 or int64 (position_bytes 4 or 8).  NULL: token t has position t mod sequence, which
 *               must be at most table_rows.  The rotated channels of a token whose position is outside the table become NaN.
 * ddp_rotary_frequencies (host): freq[i] = base^(-2 i / rotated), changed for long contexts by `scaling`:
 *   PLAIN  as it is;  LINEAR  freq / factor;  STRETCHED  base * factor^(rotated / (rotated - 2)) in place of base (rotated > 2);
 *   BY_WAVELENGTH  with turns = context * freq / (2 pi): freq above high turns, freq / factor below low turns, and in between
 *                  (1 - s) * freq / factor + s * freq with s = (turns - low) / (high - low).
 * ddp_rotary_table: row p of the table holds amplitude * cos and sin of p * freq[i] (freq: host, rotated / 2 values), p from 0,
 *   angles, cosines and sines computed in fp64 and rounded once. */
enum { DDP_ROTARY_HALF = 0, DDP_ROTARY_INTERLEAVED = 1 };
enum { DDP_ROTARY_PLAIN = 0, DDP_ROTARY_LINEAR = 1, DDP_ROTARY_STRETCHED = 2, DDP_ROTARY_BY_WAVELENGTH = 3 };
enum { DDP_ROTARY_MAX_ROTATED = 256 };
typedef struct {
    int32_t layout, dtype;
    int64_t tokens;
    int32_t q_heads, k_heads, head_dim, rotated;
    int64_t q_token, q_head, k_token, k_head;                 /* strides of q and k */
    int64_t q_out_token, q_out_head, k_out_token, k_out_head; /* of q_out and k_out */
    int64_t table_rows, sequence;
    int32_t position_bytes, inverse;
} ddp_rotary_shape;
int ddp_rotary_frequencies(int scaling, int rotated, double base, double factor, double low, double high, double context, double *freq);
int ddp_rotary_table(int rotated, const double *freq, double amplitude, int64_t rows, float *table, void *stream);
int ddp_rotary(const ddp_rotary_shape *shape, const void *q, const void *k, const float *table, const void *positions, void *q_out, void *k_out,
               void *stream);

/* ---- attention ----------------------------------------------------------------------------------------------------
 * Per sequence and query head, queries i of q_len and keys j of k_len, key head = query head / (q_heads / k_heads):
 *   s_ij = scale * q_i . k_j, where causal only for j <= i + k_len - q_len (the last query sees every key)
 *   lse_i = log sum_j exp(s_ij), o_i = sum_j exp(s_ij - lse_i) v_j;  a query that sees no key has o = 0, lse = -inf and no gradient
 * Backward, with p_ij = exp(s_ij - lse_i), formed again from q, k and lse:
 *   dv_j = sum_i p_ij do_i;  ds_ij = p_ij (do_i . v_j - do_i . o_i);  dq_i = scale sum_j ds_ij k_j;  dk_j = scale sum_i ds_ij q_i,
 *   dk and dv summed over the query heads that share the key head.
 * Sequences either have the same lengths (packed 0, cu_q and cu_k NULL: `batch` sequences of q_tokens queries and k_tokens keys), or lie
 * behind each other (packed 1, batch stride unused): sequence b has queries [cu_q[b], cu_q[b+1]) of q_tokens in all and keys
 * [cu_k[b], cu_k[b+1]) of k_tokens; cu_q and cu_k are device int32 [batch + 1], non-decreasing; the first sequence starts at 0
 * whatever entry 0 says, and queries (keys) behind the last one see no key (no query).  Entries outside [0, tokens] are taken as the
 * nearest bound, and rows outside a sequence are never read on its account.
 *   q, o, do, dq  [.., q_heads, head_dim]; k, v, dk, dv  [.., k_heads, head_dim]; of dtype, 1 <= head_dim <= 128
 *   lse           fp32 [batch, q_heads, q_tokens] ([q_heads, q_tokens] when packed)
 * Operands are read in 16-byte groups of bf16.  bf16 tensors whose start, strides and head_dim allow it are read as they are (q, k and v
 * may be parts of one projection's output); others, and fp32 ones as three bf16 planes whose products are as exact as fp32's, are
 * copied into the workspace.  The workspace calls look at the tensors' addresses and strides only; NULL: as if copied.
 * Where heads and blocks of queries (keys) are few, parts of a sum over the keys (queries) lie in the workspace as well, in fp32.
 * A pair of a query and a key that it does not see has p = ds = 0, which multiply the pair's rows in the second products: values that are not finite, and
 * in the backward call such keys, queries and d_o, may make rows of the sequence NaN that they are masked from, as a masked product would.
 * In bf16 the probabilities and ds are rounded to bf16 as operands of the second products, whose sums are fp32. */
typedef struct {
    void *data;
    int64_t batch, token, head; /* strides */
} ddp_heads;
typedef struct {
    int32_t dtype, causal;
    int32_t q_heads, k_heads, head_dim, batch;
    int64_t q_tokens, k_tokens;
    float scale;
    int32_t packed;
} ddp_attention;
int64_t ddp_attention_forward_workspace(const ddp_attention *attention, const ddp_heads *q, const ddp_heads *k, const ddp_heads *v);
int ddp_attention_forward(const ddp_attention *attention, const ddp_heads *q, const ddp_heads *k, const ddp_heads *v, const int32_t *cu_q,
                          const int32_t *cu_k, const ddp_heads *o, float *lse, void *workspace, int64_t workspace_bytes, void *stream);
int64_t ddp_attention_backward_workspace(const ddp_attention *attention, const ddp_heads *d_o, const ddp_heads *q, const ddp_heads *k, const ddp_heads *v);
int ddp_attention_backward(const ddp_attention *attention, const ddp_heads *d_o, const ddp_heads *q, const ddp_heads *k, const ddp_heads *v,
                           const ddp_heads *o, const float *lse, const int32_t *cu_q, const int32_t *cu_k, const ddp_heads *dq,
                           const ddp_heads *dk, const ddp_heads *dv, void *workspace, int64_t workspace_bytes, void *stream);

/* ---- cross entropy of a language model's head ---------------------------------------------------------------------
 * z = x weight^T, which for more than a few tokens is never there as a whole;  lse_t = log sum_v exp(z_tv);  loss_t = lse_t - z_t,target(t)
 * Backward, with the loss' gradient g per token:  dz_tv = g_t (exp(z_tv - lse_t) - [v = target(t)]);  dx = dz weight;  dweight = dz^T x
 * A target outside [0, vocab) (such as -100) has loss 0 and no gradient.
 *   x, dx            [tokens, hidden] of dtype, x_stride and dx_stride between rows
 *   weight, dweight  [vocab, hidden] of dtype, w_stride and dw_stride between rows
 *   targets          int64 [tokens];  loss, lse, dloss  fp32 [tokens]
 *   dx or dweight may be NULL.  Any two of tokens, vocab and hidden are less than 2^23 tiles of 256 x 256: tokens * vocab up to 2^39.
 *   The workspace calls look at x and weight's addresses only, not at what is there: rows whose start, stride or
 *   hidden are no multiples of 16 and 128 bytes, and fp32 ones of more than 64 tokens, are copied into padded ones in the workspace.
 * z is formed piece by piece of the vocabulary, in the backward call again; dz is rounded to dtype as an operand of the second
 * products, whose sums are fp32. */
typedef struct {
    int32_t dtype;
    int64_t tokens, vocab, hidden;
    int64_t x_stride, w_stride, dx_stride, dw_stride;
} ddp_head;
int64_t ddp_cross_entropy_forward_workspace(const ddp_head *head, const void *x, const void *weight);
int ddp_cross_entropy_forward(const ddp_head *head, const void *x, const void *weight, const int64_t *targets, float *loss, float *lse, void *workspace,
                              int64_t workspace_bytes, void *stream);
int64_t ddp_cross_entropy_backward_workspace(const ddp_head *head, const void *x, const void *weight);
int ddp_cross_entropy_backward(const ddp_head *head, const float *dloss, const void *x, const void *weight, const int64_t *targets, const float *lse,
                               void *dx, void *dweight, void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* DREAMDDP_OPERATORS_H */
