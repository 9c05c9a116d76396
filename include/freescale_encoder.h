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
 * rounded to nearest even.  An element is off by at most 1/127 of the group's largest magnitude.  A group with an
 * infinity or a NaN has exponent 255 and reads back as NaN throughout.
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
 * n == 0: the sums over the rows are written, as zeros.
 * work: fs_block_norm_work_bytes(n, dim) bytes, contents irrelevant before and after. */
int fs_block_norm_backward(fs_ctx *ctx, const fs_block_args *args, fs_stream stream);
size_t fs_block_norm_work_bytes(int64_t n, int32_t dim);

#ifdef __cplusplus
}
#endif
#endif /* FREESCALE_ENCODER_H */
