/*
 * freescale_encoder.h - C ABI of what stands between a lookup (fs_gather_jagged) and the gradients it gets back
 * (fs_prioritized_step, fs_segment_reduce_grads) in a model that reads user-interaction histories: attention over a
 * jagged batch with a learned relative position bias, the norms before and after a block with its gate and residual
 * scale, and rows held in 8 bits from Forward to Backward.
 *
 * The conventions of freescale.h hold, and on top of them:
 *   - The context is used for its GPU, its device error flags and its error text only.  None of its workspace is touched:
 *     scratch memory is the caller's (`work`, sized by the *_work_bytes functions), so that calls on several streams of
 *     one context, and graphs captured from them, may overlap as long as each has scratch of its own.
 *   - The context's GPU need not be the current one; the current device is the same before and after a call.
 *   - Pointers to rows are 16-byte aligned, row strides are counted in elements and multiples of 16 bytes.  A stride may
 *     be larger than the row: q, k, v (and dq, dk, dv) may be the parts of one tensor.
 *   - Results do not vary from run to run: every sum is taken in a fixed order.
 *   - Entries of the records that a call does not read may hold anything.
 *   - What a call writes lies over nothing that it reads or writes besides, but where it says that it may.
 */
#ifndef FREESCALE_ENCODER_H
#define FREESCALE_ENCODER_H

#include "freescale.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- rows in 8 bits -------------------------------------------------------------------------- */

/* Columns that share a power of two. */
#define FS_ROWS8_GROUP 32
#define FS_MAX_BLOCK_DIM 1024

/* rows [n, dim] (fp32 or bf16, rows `stride` elements apart) in 8 bits: codes [n, dim] int8 and one exponent byte for
 * every FS_ROWS8_GROUP columns, exps [n, dim / FS_ROWS8_GROUP]:
 *     value = code * 2^(exp - 127)
 * The power of two is the smallest for which the largest magnitude of the group rounds to at most 127 steps and is at
 * least 2^-126 (at most 2^121, where magnitudes from 127.5 * 2^121 on become 127 steps: 128 are beyond fp32); codes are
 * rounded to nearest even.  An element is off by at most 1/127 of the group's largest magnitude, or by 2^-127 where that is
 * more (magnitudes below 127 * 2^-127).  A group with an infinity or a NaN has exponent 255 and reads back as NaN throughout.
 * dim a multiple of FS_ROWS8_GROUP, at most FS_MAX_BLOCK_DIM. */
int fs_rows_pack8(fs_ctx *ctx, const void *rows, int64_t stride, fs_dtype dt, int64_t n, int32_t dim, int8_t *codes,
                  uint8_t *exps, fs_stream stream);

/* The values that codes and exps stand for, in fp32 or rounded to bf16 (exact: a code has 7 bits). */
int fs_rows_unpack8(fs_ctx *ctx, const int8_t *codes, const uint8_t *exps, int64_t n, int32_t dim, void *rows,
                    int64_t stride, fs_dtype dt, fs_stream stream);

/* ---- the norms around a block --------------------------------------------------------------- */

/* What joins a block's output to the residual rows and makes the next block's input of them, in one pass over n rows:
 *     y = x + scale * w_post * rms(a) * silu(g)        rms(t) = t / sqrt(mean of t^2 over the columns + eps)
 *     h = w_pre * rms(y)                               silu(t) = t / (1 + exp(-t))
 * with a the block's output, g its gate, w_post / scale / w_pre [dim] fp32 learned.  Arithmetic in fp32, one rounding at
 * the end (h is made of the unrounded y).
 *   a == NULL: y = x and is not written (the norm in front of the first block; a, g, w_post, scale are not read)
 *   h == NULL: no norm of y (behind the last block; w_pre is not read)
 *   a_codes / g_codes / y_codes (OPTIONAL, each with its exps): a, g and the rounded y in 8 bits as fs_rows_pack8 makes
 *         them, for the backward pass; dim a multiple of FS_ROWS8_GROUP then
 * x, y [n, dim] of rows_dt; a, g (strides a_stride, g_stride) and h [n, dim] of dt.  y may be x.  dim a multiple of 4
 * (both fp32) / 8, at most FS_MAX_BLOCK_DIM. */
typedef struct fs_block_args {
    int64_t n;
    int32_t dim;
    int32_t rows_dt, dt;             /* fs_dtype */
    float eps;
    const void *x, *a, *g;
    int64_t a_stride, g_stride;
    const float *w_post, *scale, *w_pre;
    void *y, *h;
    int8_t *a_codes, *g_codes, *y_codes;
    uint8_t *a_exps, *g_exps, *y_exps;
    /* backward only */
    const void *dy, *dh;
    void *dx, *da, *dg;
    int64_t da_stride, dg_stride;
    float *dw_post, *dscale, *dw_pre;
    void *work;
    size_t work_bytes;
} fs_block_args;

int fs_block_norm(fs_ctx *ctx, const fs_block_args *args, fs_stream stream);

/* Its gradients.  With dy [n, dim] of rows_dt (NULL: zero) and dh [n, dim] of dt (NULL: h was not made) those of y and h:
 *     dx = dy + gradient of h with respect to y       the whole gradient of y, and so of x
 *     da, dg (strides da_stride, dg_stride)           those of a and g (not written where a was NULL)
 *     dw_post, dscale, dw_pre [dim] fp32              sums over the rows, overwritten
 * Reads y as the forward pass left it (x where a was NULL), a, g, w_post, scale, w_pre; x, h are not read.  Each of y, a, g
 * may be NULL with its codes and exps given instead: the gradient is then taken at the values those stand for.  To leave
 * the join out, a and a_codes are both NULL.  The norms are computed anew from the rows.  dx may be dy.
 * n == 0: those of dw_post, dscale (together) and dw_pre that are not NULL are written, as zeros, and no other entry tells what
 * is wanted.
 * work: fs_block_norm_work_bytes(n, dim) bytes, contents irrelevant before and after. */
int fs_block_norm_backward(fs_ctx *ctx, const fs_block_args *args, fs_stream stream);
size_t fs_block_norm_work_bytes(int64_t n, int32_t dim);

/* ---- attention over a jagged batch -------------------------------------------------------------------- */

#define FS_MAX_HEAD_DIM 128
#define FS_MAX_BIAS_BUCKETS 1024
#define FS_MAX_BIAS_DISTANCES 4096
#define FS_MAX_ROW_STRIDE (1 << 22)       /* elements */
#define FS_HIDDEN_BIAS (-40000.f)         /* a bias so low hides its pairs */

/* Attention of each user's query rows over the user's keys and values, with a learned bias for the bucket that the distance
 * between the two lies in:
 *     s_ij = scale q_i . k_j + bias[bucket(pos_i - pos_j), head]      o_i = sum over j of softmax(s_i)_j v_j
 * User b has the query rows q_offsets[b] .. q_offsets[b+1] and the keys kv_offsets[b] .. kv_offsets[b+1], of which the first
 * kv_lengths[b] are in use (kv_lengths == NULL: all; a cache that grows has rows to spare).  The query rows are the last ones
 * of the history: with nk keys in use and nq query rows, row i stands at position nk - nq + i, key j at j.  For a batch
 * that attends to itself q_offsets and kv_offsets are the same.
 *   causal == 1: row i sees the keys up to its own position; == 0: all keys in use.  A row that sees no key (there are more
 *         query rows than keys, or every bias it meets hides) gives zeros, and no gradient.  What a row does not see does not
 *         reach it, infinities and NaN included.  A bias of FS_HIDDEN_BIAS or less, -infinity and every type's lowest value
 *         among them, hides its pairs.
 *   q [n_q, heads, head_dim], k and v [n_kv, kv_heads, head_dim] of dt, heads of a row next to each other, rows q_stride,
 *         k_stride, v_stride elements apart; query heads h .. h + heads/kv_heads - 1 share a key head
 *   bias  [num_buckets, heads] fp32 (NULL: none), bucket_of int32: the bucket of each distance, tabulated by the caller -
 *         causal: [num_distances] for the distances 0, 1, ...; else [2 num_distances - 1] for -(num_distances - 1) ...
 *         num_distances - 1.  Distances beyond the table are its last entry on that side.  A bucket out of range counts as
 *         no bias and is reported as FS_ERANGE by fs_check_async.
 *   out   [n_q, heads, head_dim] of dt, packed
 *   lse   [heads, n_q] fp32 (OPTIONAL; the backward pass reads it): log of the sum of exp(s_i), -infinity for a row that sees
 *         nothing
 *   out_f32 [n_q, heads, head_dim] fp32 (OPTIONAL, bf16 only): out before its rounding.  The backward pass reads it where it
 *         is given: without it, dbias carries the roundings of out.
 *   max_q no user has more query rows than this (0: unknown).  With max_q * heads / kv_heads <= 16 the keys are cut up over
 *         the chip, which is the form for single tokens; a user with more rows is then reported as FS_ERANGE and its rows of
 *         out are left as they were.
 *   work  fs_jagged_attention_work_bytes(args) bytes, 16-byte aligned, contents irrelevant (0 bytes and NULL but for the form
 *         above)
 * scale is positive.  Scores, softmax and sums are in fp32; P and dS are rounded to dt where they go into a product, but for P of
 * out_f32 and of the form for single tokens, which keeps its 24 bits.  head_dim a multiple of 4 (fp32) / 8 (bf16), at most
 * FS_MAX_HEAD_DIM; strides of q, k and v at most FS_MAX_ROW_STRIDE.  (rows / 64 + batch) * heads < 2^24, and a user has fewer
 * than 2^30 rows.  Boundaries that do not ascend from 0 to n_q (n_kv) and lengths that do not fit their room are reported as
 * FS_ERANGE by fs_check_async; out of the user concerned is not written or is that of the keys there are. */
typedef struct fs_attention_args {
    const void *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;
    int64_t n_q, n_kv, batch;
    const int64_t *q_offsets, *kv_offsets, *kv_lengths;
    int32_t heads, kv_heads, head_dim;
    int32_t dt;                      /* fs_dtype */
    int32_t causal, max_q;
    float scale;
    int32_t num_buckets, num_distances;
    const float *bias;
    const int32_t *bucket_of;
    void *out;
    float *out_f32, *lse;
    /* backward only */
    const void *dout;
    void *dq, *dk, *dv;
    int64_t dq_stride, dk_stride, dv_stride;
    float *dbias;
    void *work;
    size_t work_bytes;
} fs_attention_args;

int fs_jagged_attention(fs_ctx *ctx, const fs_attention_args *args, fs_stream stream);
size_t fs_jagged_attention_work_bytes(const fs_attention_args *args);

/* Its gradients, from dout [n_q, heads, head_dim] of dt (packed) and out, lse and out_f32 as the forward pass left them:
 *     dq, dk, dv of dt, rows dq_stride, dk_stride, dv_stride elements apart; rows of k and v that are not in use get zeros
 *     dbias [num_buckets, heads] fp32 (NULL: not wanted), overwritten; what fs_rowwise_adagrad_update takes as `reduced` with
 *     the bias as a table of num_buckets rows of `heads` columns
 * Where a pair that is seen has an infinity or a NaN in it, the gradients that it goes into may be NaN where the formula has a
 * number.
 * work: fs_jagged_attention_backward_work_bytes(args) bytes, 16-byte aligned, contents irrelevant. */
int fs_jagged_attention_backward(fs_ctx *ctx, const fs_attention_args *args, fs_stream stream);
size_t fs_jagged_attention_backward_work_bytes(const fs_attention_args *args);

#ifdef __cplusplus
}
#endif
#endif /* FREESCALE_ENCODER_H */
