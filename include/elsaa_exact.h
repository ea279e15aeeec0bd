/*
 * elsaa_exact.h - exact softmax attention and its backward pass, part of the C
 * ABI of libelsaa (elsaa.h).
 *
 * The operator that elsaa_forward approximates, on the same heads: for the
 * layers that a model keeps exact, for prompts too short to gain from an
 * approximation, and to compare with. The N x N scores are never stored.
 *
 * The conventions of elsaa.h hold: device pointers owned by the caller, no
 * allocation, asynchronous on the caller's stream, arguments validated on the
 * host before any launch, ELSAA_* return codes, elsaa_last_error(). Every call
 * can be captured into a CUDA graph: lengths are read on the device. The calls
 * work on the current device, which must be that of the tensors.
 *
 * Query row i of sequence b (of its q_len, all N_q by default) sees key row j
 * of its k_len (all N_k) when causal = 0 or j <= i + k_len - q_len: the last
 * query sees every key. With s_ij = scale <q_i, k_j> over those j,
 *     lse_i = log sum_j exp(s_ij),   O_i = sum_j exp(s_ij - lse_i) v_j;
 * a query that sees nothing has O_i = 0 and lse_i = -inf, and so has one whose
 * scores are all -inf. Lengths outside [0, N_q] and [0, N_k] are clipped.
 *
 * Rows behind the lengths may hold anything, NaN too. A NaN or an infinity in a
 * row that a sequence has may, with causal = 1, also reach rows that do not see
 * it or that it does not see, as a weight of 0 times it is NaN:
 *     v in the forward pass and k of dq: query rows in one tile of 128 with a
 *     row that sees it or one of its 128 keys. Tiles hold the rows of a K/V
 *     head's query heads one behind the other, so that a head's first rows may
 *     share one with the last of the head before;
 *     q and d_o of dk and dv: the keys of the same 128 as one that they see.
 */
#ifndef ELSAA_EXACT_H
#define ELSAA_EXACT_H

#include "elsaa.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct elsaa_exact {
    int B;           /* sequences                                            */
    int H;           /* query heads, at most 65535                           */
    int H_kv;        /* K/V heads; H a multiple of it: query head h reads
                        K/V head h / (H / H_kv)                              */
    int N_q, N_k;    /* rows of q and of k, v; B * H * N_q and
                        B * H_kv * N_k at most 2^30                          */
    int d_h;         /* 32, 64 or 128                                        */
    int dtype;       /* ELSAA_BF16 or ELSAA_FP32, of every tensor but lse    */
    int causal;
    float scale;     /* score scale, at most 1e38; 0 -> 1/sqrt(d_h)         */
    int impl;        /* ELSAA_IMPL_AUTO (bf16 on the tensor cores) or
                        ELSAA_IMPL_SIMT                                      */
} elsaa_exact;

/*
 * Bytes of scratch that elsaa_exact_forward (backward = 0) or both calls
 * (backward = 1) need. One workspace serves calls that are ordered on one
 * stream; calls that may overlap need one each. Its contents need no
 * initialisation; its first bytes are the status that elsaa_check_status
 * reads. 256-byte aligned. No CUDA call is made.
 */
int elsaa_exact_workspace_size(const elsaa_exact *exact, int backward,
                               size_t *bytes);

/*
 * q        [B, H, N_q, d_h], k, v [B, H_kv, N_k, d_h], contiguous, 16-byte
 *          aligned, as all tensors here. Outputs must not overlap inputs.
 * q_len, k_len  [B] int32, or NULL. Rows of o and lse behind q_len are left as
 *          they were.
 * o        [B, H, N_q, d_h] (written).
 * lse      [B, H, N_q] fp32 (written), or NULL.
 *
 * bf16 on the tensor cores: scores and sums in fp32, weights (relative to a
 * reference within 2^9 of the row's largest) rounded to bf16 for their product
 * with V, their sum taken before that; o rounded once. A score below -6.9e37
 * counts as -inf; with either dtype one above 2.3e38 is infinite. The results
 * do not depend on timing, but the division of rows over CTAs, and with it the
 * last bits, depends on the sizes, the lengths and the number of SMs.
 */
int elsaa_exact_forward(const elsaa_exact *exact, const void *q,
                        const void *k, const void *v, const int32_t *q_len,
                        const int32_t *k_len, void *o, float *lse,
                        void *workspace, size_t workspace_bytes,
                        void *stream);

/*
 * The gradients of q, k and v from d_o, that of o. o and lse are those of
 * elsaa_exact_forward on the same q, k, v and lengths; the weights are
 * computed again from lse. With P_ij = exp(s_ij - lse_i) and
 * D_i = <d_o_i, o_i>:
 *     dV = P^T d_o,  dS = P (d_o V^T - D),  dQ = scale dS K,
 *     dK = scale dS^T Q,
 * summed over the query heads of a K/V head in a fixed order: a call gives the
 * same bits every time. Rows behind the lengths are left as they were; those
 * of queries that see nothing and of keys that no query sees are zeros; a query
 * with lse = -inf has weights of 0. bf16 on the tensor cores: P and dS in fp32,
 * each rounded to bf16 for its products, sums in fp32, results rounded once.
 *
 * lse is fp32, and so a weight is off by a factor of up to e^(|lse| 2^-22).
 * Where |lse| is above 2^16 ln 2, one within that factor squared of 1 counts as
 * 1: the gradients of a row that one key has to itself are right at any size of
 * its scores; how several share a row is lost from |lse| = 2^22 on.
 */
int elsaa_exact_backward(const elsaa_exact *exact, const void *q,
                         const void *k, const void *v, const void *o,
                         const float *lse, const void *d_o,
                         const int32_t *q_len, const int32_t *k_len, void *dq,
                         void *dk, void *dv, void *workspace,
                         size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* ELSAA_EXACT_H */
