/*
 * elsaa_cache.h - decoding from a paged cache whose keys and values are held
 * in 8 bits, part of the C ABI of libelsaa (elsaa.h).
 *
 * elsaa.h computes attention over whole prompts. The calls here keep the
 * prompt's K and V and answer for the tokens that follow it, a few at a time:
 *
 *   elsaa_cache_append     rows of K and V enter the cache
 *   elsaa_cache_select     a cheap score per page, the best pages
 *   elsaa_cache_attention  attention over all pages, or over those selected
 *   elsaa_cache_evict      the tokens of least accumulated attention weight
 *                          leave
 *
 * This is exact softmax attention over the cached tokens, or over selected
 * pages of them: elsaa.h's low-rank branch, fusion weight and gates have no
 * part in it.
 *
 * The conventions of elsaa.h hold: device pointers owned by the caller, no
 * allocation, asynchronous on the caller's stream, arguments validated on the
 * host before any launch, ELSAA_* return codes, elsaa_last_error(). Every call
 * can be captured into a CUDA graph: lengths and tables are read on the
 * device. The calls work on the current device, which must be that of the
 * tensors.
 *
 * The cache. A page holds the same page_size consecutive tokens for every K/V
 * head. Sequence b's token j is row j mod page_size of page
 * page_table[b][j / page_size]. An element is
 *     value = e4m3(code) * scale,    one scale per page and head,
 * and every scale is a power of two 2^e, -64 <= e <= 120. A floating-point
 * code gains no precision from a finer scale, and with powers of two a page's
 * codes move to another scale without rounding (but for codes that become
 * subnormal), so that a page can grow a token at a time.
 */
#ifndef ELSAA_CACHE_H
#define ELSAA_CACHE_H

#include "elsaa.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct elsaa_cache {
    int B;           /* sequences                                            */
    int H;           /* query heads                                          */
    int H_kv;        /* K/V heads; H a multiple of it: query head h reads
                        K/V head h / (H / H_kv)                              */
    int d_h;         /* 32, 64 or 128                                        */
    int dtype;       /* ELSAA_BF16 or ELSAA_FP32: type of the rows given to
                        elsaa_cache_append, of the queries and of O          */
    int page_size;   /* tokens per page: 16, 32, 64 or 128                   */
    int num_pages;   /* pages of the pool                                    */
    int max_pages;   /* entries of a page-table row; max_pages * page_size at
                        most 2^31 - 2^16                                     */
    float scale;     /* score scale; 0 -> 1/sqrt(d_h)                        */
    int impl;        /* ELSAA_IMPL_AUTO or ELSAA_IMPL_SIMT                   */
    void *k, *v;     /* [num_pages, H_kv, page_size, d_h] e4m3 codes,
                        16-byte aligned                                      */
    float *k_scale, *v_scale;  /* [num_pages, H_kv]                          */
    int8_t *bounds;  /* [num_pages, H_kv, 2, d_h], 16-byte aligned: per
                        channel the largest key code of the page over 4,
                        rounded up, then the smallest, rounded down          */
    const int32_t *page_table; /* [B, max_pages]: pages in [0, num_pages);
                        entries behind a sequence's last page are not read   */
    const int32_t *lengths;    /* [B]: tokens held, those of the call at hand
                        included, in [0, max_pages * page_size]              */
    int32_t *status; /* 4 ints, 16-byte aligned, zeroed by the caller when
                        the cache is made, or NULL: the first fault that a
                        call meets (a page outside the pool, a length outside
                        the table, a wait that ran out). Such entries and
                        lengths are skipped or clipped, never followed.
                        elsaa_check_status(status, stream) reads it          */
} elsaa_cache;

/*
 * Bytes of scratch that the calls below need: elsaa_cache_select and
 * elsaa_cache_attention for up to T tokens a sequence (weights = 1: with
 * weight_out), elsaa_cache_evict down to `keep` tokens (0: not called). One
 * workspace serves calls that are ordered on one stream; calls that may
 * overlap need one each. Its contents need no initialisation. 256-byte
 * aligned. No CUDA call is made.
 */
int elsaa_cache_workspace_size(const elsaa_cache *cache, int T, int weights,
                               int keep, size_t *bytes);

/*
 * Writes the newest tokens' rows into their pages.
 *
 * k, v      [B, H_kv, T, d_h] of cache->dtype, 16-byte aligned;
 *           T + max_pages * page_size <= 2^31 - 2^16.
 * new_len   [B] int32 in [0, T]: sequence b's new tokens n_b, or NULL for T
 *           each. Row t < n_b is token lengths[b] - n_b + t: advance lengths
 *           first. Rows t >= n_b, and those of a token before the first,
 *           are not read, and rows of a page behind lengths[b] keep what they
 *           held.
 *
 * With e_new the least e in [-64, 120] with |x| <= 448 2^e for every new x of
 * a page and head, the page's exponent becomes e_new if it held no older
 * token, else max(e_old, e_new), and its older codes move to it, rounded to
 * nearest even. bounds follows: hi = max(ceil(hi_old 2^(e_old - e)),
 * ceil(max code / 4)), lo likewise with min and floor. NaN stays NaN and is
 * left out of e and of bounds (a channel without a number in the page has the
 * widest, hi = 112 and lo = -112); an infinity counts as the type's largest
 * value and is stored as the page's largest, 448 2^e.
 *
 * A page that is written may be in one sequence's table only.
 */
int elsaa_cache_append(const elsaa_cache *cache, int T, const void *k,
                       const void *v, const int32_t *new_len, void *stream);

/*
 * The pages that the newest tokens' queries should read, for every sequence
 * and K/V head.
 *
 * q         [B, H, T, d_h] of cache->dtype, 16-byte aligned; new_len as above.
 * pages     [B, H_kv, n_sel] int32 (written): page indices p (entries of the
 *           sequence's table row), increasing, then -1.
 *
 * The score of page p is an upper bound of <q, k> over the box that bounds
 * describes, with the query in 8 bits: qhat = rint(q / 2^e), e the least in
 * [-60, 120] with |q| <= 127 2^e (NaN counts as 0, an infinity as +-127),
 *     u_p = max over the head's queries of
 *           (sum_i max(qhat_i hi_i, qhat_i lo_i)) 2^e 4 k_scale_p.
 * The sum is a whole number below 2^24 and its factors powers of two, so u is
 * exact in fp32 and the selection does not depend on the order of summation.
 * (From 2^128 on it counts as infinite, and such pages are equal.)
 * Taken are the first `first` pages, the last `last` and then those of
 * largest u (equal: lower p), n_sel in all or as many as the sequence has; a
 * sequence with n_b = 0 gets none. first, last >= 0 and first + last <= n_sel.
 * n_sel * page_size <= 2^31 - 2^16.
 */
int elsaa_cache_select(const elsaa_cache *cache, int T, const void *q,
                       const int32_t *new_len, int n_sel, int first, int last,
                       int32_t *pages, void *workspace,
                       size_t workspace_bytes, void *stream);

/*
 * Attention of the newest tokens over the cache:
 *     s_j = scale <q, k_j>,  lse = log sum_j exp(s_j),
 *     O = sum_j exp(s_j - lse) v_j
 * for query t < n_b of sequence b over the tokens j <= lengths[b] - n_b + t
 * (of the pages listed, if any). The rows just appended are in the cache, as
 * every other in 8 bits. A query without a key gets O = 0, lse = -inf. A NaN
 * code reaches the queries that see its token (a value's: that channel of
 * theirs) and no other.
 *
 * q, o      [B, H, T, d_h] of cache->dtype, 16-byte aligned. Rows t >= n_b of
 *           o and lse keep what they held.
 * pages     [B, H_kv, n_sel] as elsaa_cache_select writes them, or NULL for
 *           all (n_sel is then ignored). Lists of the caller's own: distinct
 *           pages of the sequence first, in any order; entries outside its
 *           pages count as none and come behind them. Of a sequence of m
 *           pages the first min(m, n_sel) entries are read, so that pages
 *           behind others' entries may be missed.
 * weight_in, weight_out  [B, H_kv, max_pages * page_size] fp32, 16-byte
 *           aligned, or both NULL:
 *           weight_out_j = weight_in_j + sum of exp(s_j - lse) over the K/V
 *           head's queries, for j < lengths[b]; entries behind keep what they
 *           held. weight_in may be weight_out, or NULL for zeros.
 * lse       [B, H, T] fp32, or NULL.
 *
 * T at most 64 and T * H / H_kv at most 128 (longer runs of queries are
 * prompts). bf16 with d_h 64 or 128 runs on the tensor cores, which take the
 * codes as they are: a query is split into two e4m3 numbers that hold its 8
 * bits, a weight, rounded to fp16, into three. fp32 and d_h = 32 run on CUDA
 * cores, and with impl = ELSAA_IMPL_SIMT everything does: weights and values
 * are multiplied in fp32 there. Exponentials are the hardware's, 2^-22 off
 * beside the rounding of their arguments. The tensor cores multiply keys by
 * queries that are scaled to at most 448: keys from 2^112 on may overflow,
 * queries whose largest element lies below 2^-92 lose bits below 2^-113. The
 * row of a query that holds a NaN or an infinity is not defined; it reaches no
 * other row.
 */
int elsaa_cache_attention(const elsaa_cache *cache, int T, const void *q,
                          const int32_t *new_len, const int32_t *pages,
                          int n_sel, const float *weight_in,
                          float *weight_out, void *o, float *lse,
                          void *workspace, size_t workspace_bytes,
                          void *stream);

/*
 * Cuts every sequence to at most `keep` tokens (keep <= 2^31 - 2^16), for each
 * K/V head its own: the last `recent` ones (recent <= keep), and of the others
 * those of largest weight (equal: lower position; NaN below every number).
 * They keep their order.
 *
 * weight     [B, H_kv, max_pages * page_size] fp32, as accumulated by
 *            elsaa_cache_attention.
 * dst_table  [B, dst_pages] int32 pages of the same pool that receive the
 *            kept tokens, dst_pages * page_size >= keep. No page of it may be
 *            in use, by this call or by another. The old pages are free
 *            afterwards. A page's exponent and bounds are those that
 *            elsaa_cache_append gives to the values held.
 *            A page of it outside the pool is not written. Of a page of
 *            page_table outside the pool, whose tokens attention skips, the
 *            kept tokens become rows of zeros, which later calls do see.
 * weight_out [B, H_kv, dst_pages * page_size] fp32: the kept tokens' weights;
 *            entries behind them keep what they held. Not weight itself.
 * lengths_out [B] int32: min(lengths, keep); may be cache->lengths.
 * kept       [B, H_kv, keep] int32: the kept positions, increasing, then -1;
 *            or NULL.
 */
int elsaa_cache_evict(const elsaa_cache *cache, const float *weight, int keep,
                      int recent, const int32_t *dst_table, int dst_pages,
                      float *weight_out, int32_t *lengths_out, int32_t *kept,
                      void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* ELSAA_CACHE_H */
