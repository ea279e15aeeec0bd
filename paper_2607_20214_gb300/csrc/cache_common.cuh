// Device helpers of the cache kernels: lengths and pages as the device finds
// them, powers of two, e4m3 conversions, the division of tiles over CTAs.
#pragma once

#include "cache.h"
#include "device_common.cuh"
#include "tc_common.cuh"

namespace elsaa {
namespace cache {

// Tokens of sequence b, clipped to its table row.
__device__ __forceinline__ int tokens(const CacheView &c, int b) {
    const int n = c.lengths[b], cap = c.max_pages * c.ps;
    if (n < 0 || n > cap) {
        report(c.status, kDevCacheLength, b, n, cap);
        return n < 0 ? 0 : cap;
    }
    return n;
}

// New tokens of sequence b.
__device__ __forceinline__ int fresh(const CacheView &c, int b) {
    if (!c.new_len) return c.T;
    const int n = c.new_len[b];
    if (n < 0 || n > c.T) {
        report(c.status, kDevCacheLength, b, n, c.T);
        return n < 0 ? 0 : c.T;
    }
    return n;
}

// A page of the pool, or -1.
__device__ __forceinline__ int checked_page(const CacheView &c, int id, int b,
                                            int p) {
    if ((unsigned)id < (unsigned)c.num_pages) return id;
    report(c.status, kDevCachePage, b, p, id);
    return -1;
}
__device__ __forceinline__ int page_id(const CacheView &c, int b, int p) {
    return checked_page(c, c.table[(size_t)b * c.max_pages + p], b, p);
}

// 2^e for -126 <= e <= 127.
__device__ __forceinline__ float pow2(int e) {
    return __int_as_float((e + 127) << 23);
}

// Least e in [low, high] with amax <= M 2^(e + s), M in [1, 2) given by its
// 23 mantissa bits `top`: 448 = 1.75 * 2^8 and 127 = 1.984375 * 2^6.
__device__ __forceinline__ int least_exponent(float amax, uint32_t top, int s,
                                              int low, int high) {
    if (!(amax > 0.0f)) return low;
    const uint32_t u = __float_as_uint(amax);
    // a subnormal lies far below 2^low: its exponent does not matter
    const int e = (int)(u >> 23) - 127 - s + ((u & 0x7fffffu) > top ? 1 : 0);
    return min(max(e, low), high);
}
__device__ __forceinline__ int page_exponent(float amax) {
    return least_exponent(amax, 0x600000u, 8, kCacheExpLow, kCacheExpHigh);
}
__device__ __forceinline__ int query_exponent(float amax) {
    return least_exponent(amax, 0x7e0000u, 6, kQueryExpLow, kCacheExpHigh);
}
// Exponent of a scale that is a power of two.
__device__ __forceinline__ int scale_exponent(float s) {
    return (int)((__float_as_uint(s) >> 23) & 0xffu) - 127;
}
// |x| for a page's extreme: NaN counts as 0, an infinity as the largest
// float.
__device__ __forceinline__ float magnitude(float x) {
    return fminf(fmaxf(fabsf(x), 0.0f), 3.402823466e38f);
}

// Two floats to two e4m3 codes (nearest even, saturating, NaN kept): lo in
// the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;"
        : "=h"(r)
        : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c,
                                           float d) {
    return e4m3x2(a, b) | (e4m3x2(c, d) << 16);
}
// The two e4m3 codes in the low half of w.
__device__ __forceinline__ float2 from_e4m3x2(uint32_t w) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)w));
    float lo, hi;
    tc::unpack_f16x2(h, lo, hi);
    return make_float2(lo, hi);
}
__device__ __forceinline__ void from_e4m3x4(uint32_t w, float *x) {
    const float2 a = from_e4m3x2(w & 0xffffu), b = from_e4m3x2(w >> 16);
    x[0] = a.x;
    x[1] = a.y;
    x[2] = b.x;
    x[3] = b.y;
}

// Rows of 8 elements of the caller's type.
__device__ __forceinline__ void load8(const float *p, float *x) {
    const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float *x) {
    const uint4 a = *(const uint4 *)p;
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// --------------------------------------------------- attention: the division
//
// Every K/V head and column group of a sequence is an item of
// ceil(tokens / kCacheTile) tiles (one at least, so that a query without keys
// gets its row). The tiles of all items, one after the other, are cut into
// `ctas` equal ranges, so that ragged lengths load the SMs evenly; an item
// that a cut crosses is written as pieces and merged afterwards.

// Tokens (or listed rows) that sequence b's heads walk, and its tiles.
__device__ __forceinline__ int walk(const CacheAttn &A, int b) {
    if (fresh(A.c, b) == 0) return -1;
    const int n = tokens(A.c, b);
    if (!A.pages) return n;
    const int np = (n + A.c.ps - 1) / A.c.ps;
    return min(np, A.n_sel) * A.c.ps;
}
__device__ __forceinline__ int walk_tiles(int n) {
    return n < 0 ? 0 : max(1, (n + kCacheTile - 1) / kCacheTile);
}

// prefix[b] = tiles of one head's items of the sequences before b, by the
// first warp; the CTA synchronises afterwards.
__device__ __forceinline__ void sum_tiles(const CacheAttn &A, int *prefix) {
    const int lane = threadIdx.x & 31;
    if (threadIdx.x >= 32) return;
    int base = 0;
    for (int b0 = 0; b0 < A.c.B; b0 += 32) {
        const int b = b0 + lane;
        int x = b < A.c.B ? walk_tiles(walk(A, b)) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (b < A.c.B) prefix[b + 1] = base + x;
        base += __shfl_sync(0xffffffffu, x, 31);
    }
    if (lane == 0) prefix[0] = 0;
}

struct Range {
    long total, n;  // tiles of the call, CTAs that have some
    long t0, t1;    // of this CTA
};
__device__ __forceinline__ Range cta_range(const CacheAttn &A,
                                           const int *prefix, int cta) {
    Range r;
    r.total = (long)prefix[A.c.B] * A.c.Hkv * A.groups;
    r.n = min((long)A.ctas, r.total);
    r.t0 = cta < r.n ? r.total * cta / r.n : r.total;
    r.t1 = cta < r.n ? r.total * (cta + 1) / r.n : r.total;
    return r;
}

// The item that tile t belongs to.
struct Item {
    int b, h, group;   // sequence, K/V head, column group
    long a;            // its first tile
    int tiles;
    int len, n;        // tokens held, new ones
    int walk;          // rows walked
    int col0, cols;    // its columns of the head's G T
};
__device__ __forceinline__ Item find_item(const CacheAttn &A,
                                          const int *prefix, long t) {
    const int HC = A.c.Hkv * A.groups;
    int lo = 0, hi = A.c.B;  // prefix[lo] HC <= t < prefix[hi] HC
    while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if ((long)prefix[m] * HC <= t)
            lo = m;
        else
            hi = m;
    }
    Item it;
    it.b = lo;
    it.tiles = prefix[lo + 1] - prefix[lo];
    const long first = (long)prefix[lo] * HC;
    const int hc = (int)((t - first) / it.tiles);
    it.a = first + (long)hc * it.tiles;
    it.h = hc / A.groups;
    it.group = hc % A.groups;
    it.n = fresh(A.c, lo);
    it.len = tokens(A.c, lo);
    it.walk = walk(A, lo);
    it.col0 = it.group * A.cols;
    it.cols = min(A.cols, A.c.G * A.c.T - it.col0);
    return it;
}

// The last position that column `col` (g T + t) of an item sees, -1 if none
// or if the column is no query.
__device__ __forceinline__ int last_seen(const CacheAttn &A, const Item &it,
                                         int col) {
    const int t = col % A.c.T;
    return t < it.n ? it.len - it.n + t : -1;
}
// Row of q, o and lse of column `col`.
__device__ __forceinline__ size_t query_row(const CacheAttn &A, int b, int h,
                                            int col) {
    const int g = col / A.c.T, t = col % A.c.T;
    return ((size_t)b * A.c.H + (size_t)h * A.c.G + g) * A.c.T + t;
}

__device__ __forceinline__ float *piece(const CacheAttn &A, long cta,
                                        int slot, int col) {
    return A.part + (((size_t)cta * 2 + slot) * A.cols + col) * (A.c.d + 2);
}

__device__ __forceinline__ void store_o(const CacheAttn &A, size_t row, int i,
                                        float x) {
    if (A.c.dtype == ELSAA_FP32)
        ((float *)A.o)[row * A.c.d + i] = x;
    else
        ((__nv_bfloat16 *)A.o)[row * A.c.d + i] = __float2bfloat16_rn(x);
}
// lse of a finished column from its maximum (log2) and sum.
__device__ __forceinline__ void store_lse(const CacheAttn &A, const Item &it,
                                          int col, float m, float l) {
    const float l2 = l > 0.0f ? m + log2f(l) : -INFINITY;
    if (A.lse2)
        A.lse2[((size_t)it.b * A.c.Hkv + it.h) * A.c.G * A.c.T + col] = l2;
    if (A.lse && col % A.c.T < it.n)
        A.lse[query_row(A, it.b, it.h, col)] = l2 * 0.6931471805599453f;
}

}  // namespace cache
}  // namespace elsaa
