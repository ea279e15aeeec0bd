/*
 * elsaa_heads.h - from the rows of the Q/K/V projections to the heads that
 * the attention calls read, part of the C ABI of libelsaa (elsaa.h).
 *
 * elsaa_forward, elsaa_exact_forward and elsaa_cache_append take heads
 * [B, heads, N, d_h]; a projection writes rows [B, N, heads, d_h]. The calls
 * here stand between the two, in one pass over the data: the norm of every
 * query and key head, the rotation by the token's position, and the change of
 * layout; and the backward pass of the three.
 *
 * The conventions of elsaa.h hold: device pointers owned by the caller, no
 * allocation, asynchronous on the caller's stream, arguments validated on the
 * host before any launch, ELSAA_* return codes, elsaa_last_error(). Every call
 * can be captured into a CUDA graph: positions and lengths are read on the
 * device. The calls work on the current device, which must be that of the
 * tensors.
 *
 * For the row x of token n and head h of sequence b, in fp32:
 *     y = x w / sqrt(mean(x^2) + eps)        (norm = 1; else y = x)
 *     out_lo = y_lo cos a - y_hi sin a,  out_hi = y_hi cos a + y_lo sin a
 * for every pair (lo, hi) of the first rotary.dim channels, the others as they
 * are, rounded once to the element type. Values (v) are neither normed nor
 * rotated. The angle of pair p is
 *     a = 2 pi frac(position * turns[p] / 2^64),
 * position that of the pair's axis: the product is taken modulo 2^64, so that
 * a far position's angle is as exact as a near one's. Sines and cosines are
 * those of fp32 (dtype fp32) or off by 2^-20 at most (bf16, whose heads and rows
 * are rounded to 2^-8; the fp32 dw_q and dw_k of bf16 rows are off by 2^-20 of
 * their terms' sizes for it). mean(x^2) is taken in fp32: rows of numbers near 2^64
 * overflow to 0.
 */
#ifndef ELSAA_HEADS_H
#define ELSAA_HEADS_H

#include "elsaa.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ELSAA_MAX_PAIRS 64
#define ELSAA_MAX_AXES 4

typedef struct elsaa_rotary {
    int dim;         /* rotated channels, the first ones of a head: 0 .. d_h;
                        a multiple of 16, or of 2 when interleaved           */
    int interleaved; /* pair p is channels (p, p + dim/2), or (2p, 2p + 1)   */
    int axes;        /* position axes, 1 .. ELSAA_MAX_AXES                   */
    int reserved;    /* 0                                                    */
    uint64_t turns[ELSAA_MAX_PAIRS]; /* pair p's turns per position, as a
                        fraction of 2^64 (whole turns left out; a negative
                        frequency as its two's complement)                   */
    uint8_t axis[ELSAA_MAX_PAIRS];   /* pair p's axis                        */
} elsaa_rotary;

typedef struct elsaa_heads {
    int B;           /* sequences                                            */
    int H;           /* query heads, at most 65535                           */
    int H_kv;        /* key and value heads; H a multiple of it              */
    int N;           /* rows of every sequence; B * N at most 2^30           */
    int d_h;         /* 32, 64 or 128                                        */
    int dtype;       /* ELSAA_BF16 or ELSAA_FP32: type of rows and heads     */
    int norm;        /* 1: queries and keys are normed                       */
    int expand;      /* 0: k, v heads [B, H_kv, N, d_h]; 1: [B, H, N, d_h],
                        head h a copy of K/V head h / (H / H_kv), for
                        elsaa_forward, which knows no groups                 */
    int grad_fp32;   /* type of the heads' gradients: 0 dtype, 1 fp32 (as
                        elsaa_backward writes them)                          */
    float eps;       /* of the norm, > 0                                     */
    elsaa_rotary rotary;
} elsaa_heads;

/* Rows of B sequences, N tokens and a number of heads: row (b, n, h) begins
 * at data + (b batch + n row + h head) elements and is d_h long. data is
 * 16-byte aligned and the strides of axes longer than one are multiples of 16
 * bytes. */
typedef struct elsaa_rows {
    void *data;
    int64_t batch, row, head;
} elsaa_rows;

/* Bytes of scratch that elsaa_heads_backward needs. One workspace serves calls
 * that are ordered on one stream; calls that may overlap need one each. No
 * initialisation, 256-byte aligned. No CUDA call is made. */
int elsaa_heads_workspace_size(const elsaa_heads *heads, size_t *bytes);

/*
 * Rows to heads.
 *
 * q, k, v    rows of H, H_kv and H_kv heads (read); NULL: not wanted. Strides
 *            may be 0 or negative.
 * w_q, w_k   [d_h] fp32 weights of the norm, or NULL for ones.
 * positions  [axes, B, N] int32, any value, or NULL for positions 0, 1, ...,
 *            the same in every axis; with lengths, row n of sequence b is then
 *            at lengths[b] - n_b + n (new tokens of a cache, lengths advanced
 *            first, as elsaa_cache_append has them).
 * lengths    [B] int32, or NULL; not together with positions.
 * new_len    [B] int32 in [0, N]: sequence b's rows n_b, or NULL for N each.
 *            Rows behind them are not read, and their heads are left as they
 *            were.
 * q_out      [B, H, N, d_h], k_out and v_out as expand says, contiguous,
 *            16-byte aligned; of those asked for. They must not overlap the
 *            rows.
 */
int elsaa_heads_forward(const elsaa_heads *heads, const elsaa_rows *q,
                        const elsaa_rows *k, const elsaa_rows *v,
                        const float *w_q, const float *w_k,
                        const int32_t *positions, const int32_t *lengths,
                        const int32_t *new_len, void *q_out, void *k_out,
                        void *v_out, void *stream);

/*
 * The heads' gradients to those of the rows and of the norm's weights.
 *
 * dq, dk, dv   gradients of q_out, k_out, v_out, of dtype or fp32 (grad_fp32),
 *              contiguous, 16-byte aligned; NULL: not wanted. Those of copied
 *              heads (expand) are added up.
 * q, k         the rows given to elsaa_heads_forward, read with norm = 1.
 * w_q .. new_len  as given to elsaa_heads_forward.
 * dq_rows, dk_rows, dv_rows  rows of dtype (written, those of new_len only),
 *              of those asked for; no two of their rows may share an element.
 * dw_q, dw_k   [d_h] fp32 (written: the sum over all rows and heads, the same
 *              bits on every call), or NULL.
 *
 * With u the gradient rotated back, xh = x / sqrt(mean(x^2) + eps), t = u w:
 *     dx = (t - xh mean(t xh)) / sqrt(mean(x^2) + eps),  dw = sum u xh.
 */
int elsaa_heads_backward(const elsaa_heads *heads, const void *dq,
                         const void *dk, const void *dv, const elsaa_rows *q,
                         const elsaa_rows *k, const float *w_q,
                         const float *w_k, const int32_t *positions,
                         const int32_t *lengths, const int32_t *new_len,
                         const elsaa_rows *dq_rows, const elsaa_rows *dk_rows,
                         const elsaa_rows *dv_rows, float *dw_q, float *dw_k,
                         void *workspace, size_t workspace_bytes,
                         void *stream);

#ifdef __cplusplus
}
#endif

#endif /* ELSAA_HEADS_H */
