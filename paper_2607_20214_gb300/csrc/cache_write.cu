// Writes into the 8-bit cache: elsaa_cache_append (rows of new tokens) and
// the second half of elsaa_cache_evict (the kept rows to other pages).
//
// A CTA owns one page of one head, keys or values, so the page's exponent is
// one block reduction away and every byte moves once: the page's new rows are
// read into registers (at most 32 KB a CTA), their largest magnitude gives
// the exponent e, and codes e4m3(x 2^-e) go out. Scaling by a power of two is
// exact, so the only rounding is the conversion's.
#include "cache_common.cuh"

namespace elsaa {

namespace {

using namespace cache;

constexpr int kWrThreads = 256;

// Largest of all threads' x.
__device__ __forceinline__ float block_max(float x, float *tmp) {
    x = warp_max(x);
    if ((threadIdx.x & 31) == 0) tmp[threadIdx.x >> 5] = x;
    __syncthreads();
    float m = tmp[0];
#pragma unroll
    for (int i = 1; i < kWrThreads / 32; ++i) m = fmaxf(m, tmp[i]);
    return m;
}

// Channel extremes of the codes: thread (row group, chunk of 8 channels)
// holds hi[8], lo[8] of its rows; afterwards thread i < D has channel i's.
template <int D>
__device__ __forceinline__ void channel_extremes(float *hi, float *lo,
                                                 float (*sh)[2][D], float &h,
                                                 float &l) {
    constexpr int C = D / 8;
    const int tid = threadIdx.x;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int o = C; o < 32; o <<= 1) {
            hi[i] = fmaxf(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], o));
            lo[i] = fminf(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], o));
        }
    }
    if ((tid & 31) < C) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            sh[tid >> 5][0][(tid & 31) * 8 + i] = hi[i];
            sh[tid >> 5][1][(tid & 31) * 8 + i] = lo[i];
        }
    }
    __syncthreads();
    h = -INFINITY;
    l = INFINITY;
    if (tid < D) {
#pragma unroll
        for (int w = 0; w < kWrThreads / 32; ++w) {
            h = fmaxf(h, sh[w][0][tid]);
            l = fminf(l, sh[w][1][tid]);
        }
    }
}

// One byte of bounds: a whole number in [-112, 112] (448 / 4) wherever the
// channel has a number; clipped for one that has none.
__device__ __forceinline__ int8_t bound(float x) {
    return (int8_t)fminf(fmaxf(x, -112.0f), 112.0f);
}

// 8 values times f as codes; extremes of what the codes stand for.
__device__ __forceinline__ uint2 encode8(const float *x, float f, bool ext,
                                         float *hi, float *lo) {
    uint2 w;
    w.x = e4m3x4(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
    w.y = e4m3x4(x[4] * f, x[5] * f, x[6] * f, x[7] * f);
    if (ext) {
        float y[8];
        from_e4m3x4(w.x, y);
        from_e4m3x4(w.y, y + 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {  // NaN is left out
            hi[i] = fmaxf(hi[i], y[i]);
            lo[i] = fminf(lo[i], y[i]);
        }
    }
    return w;
}

template <typename T>
struct Raw8 {
    uint4 w[sizeof(T) * 8 / 16];
};

template <typename T, int D>
__global__ void __launch_bounds__(kWrThreads)
    k_cache_append(CacheView c, const T *__restrict__ kn,
                   const T *__restrict__ vn) {
    wait_for_stream();
    constexpr int C = D / 8, R = kWrThreads / C, NP = kCacheTile / R;
    __shared__ float tmp[kWrThreads / 32];
    __shared__ float sh[kWrThreads / 32][2][D];
    const int tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z >> 1;
    const bool keys = (blockIdx.z & 1) == 0;
    const int end = tokens(c, b), start = end - fresh(c, b);
    const int p = max(start, 0) / c.ps + blockIdx.x, p0 = p * c.ps;
    if (p0 >= end || start >= end) return;
    // rows [r0, r1) of the page are new, [0, r0) older
    const int r0 = max(max(start, 0) - p0, 0), r1 = min(c.ps, end - p0);
    const int id = page_id(c, b, p);
    if (id < 0) return;
    const size_t ph = (size_t)id * c.Hkv + h;
    uint8_t *codes = (keys ? c.k : c.v) + ph * c.ps * D;
    float *scale = (keys ? c.ks : c.vs) + ph;
    const T *x = (keys ? kn : vn) + ((size_t)b * c.Hkv + h) * c.T * D;
    const int ch = tid % C, rr = tid / C;

    Raw8<T> raw[NP];
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = i * R + rr;
        if (r >= r0 && r < r1) {
            const uint4 *src =
                (const uint4 *)(x + (size_t)(p0 + r - start) * D + ch * 8);
#pragma unroll
            for (int j = 0; j < (int)(sizeof(T) / 2); ++j) raw[i].w[j] = src[j];
        }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = i * R + rr;
        if (r >= r0 && r < r1) {
            float y[8];
            load8((const T *)&raw[i], y);
#pragma unroll
            for (int j = 0; j < 8; ++j) amax = fmaxf(amax, magnitude(y[j]));
        }
    }
    const bool had = r0 > 0;
    const int e_old =
        had ? min(max(scale_exponent(*scale), kCacheExpLow), kCacheExpHigh)
            : kCacheExpLow;
    int e = page_exponent(block_max(amax, tmp));
    if (had) e = max(e, e_old);
    const float f = pow2(-e);
    float hi[8], lo[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        hi[j] = -INFINITY;
        lo[j] = INFINITY;
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = i * R + rr;
        if (r >= r0 && r < r1) {
            float y[8];
            load8((const T *)&raw[i], y);
            *(uint2 *)(codes + (size_t)r * D + ch * 8) =
                encode8(y, f, keys, hi, lo);
        }
    }
    // older rows move to the larger exponent; 2^(e_old - e) may be far below
    // the smallest code, whose product is then 0
    const float drop = exp2f((float)(e_old - e));
    if (had && e != e_old) {
        for (int r = rr; r < r0; r += R) {
            uint2 *at = (uint2 *)(codes + (size_t)r * D + ch * 8);
            const uint2 w = *at;
            float y[8];
            from_e4m3x4(w.x, y);
            from_e4m3x4(w.y, y + 4);
            *at = encode8(y, drop, false, nullptr, nullptr);
        }
    }
    if (keys) {
        float u, l;
        channel_extremes<D>(hi, lo, sh, u, l);
        if (tid < D) {
            int8_t *at = c.bounds + ph * 2 * D + tid;
            u = ceilf(u * 0.25f);
            l = floorf(l * 0.25f);
            if (had) {
                u = fmaxf(u, ceilf((float)at[0] * drop));
                l = fminf(l, floorf((float)at[D] * drop));
            }
            at[0] = bound(u);
            at[D] = bound(l);
        }
    }
    // block_max's barrier lies between every thread's read of it and this
    if (tid == 0) *scale = pow2(e);
}

// Page j of sequence b's kept rows, one head, keys or values.
template <int D>
__global__ void __launch_bounds__(kWrThreads)
    k_cache_compact(CacheView c, const float *__restrict__ weight, int keep,
                    const int32_t *__restrict__ kept,
                    const int *__restrict__ count,
                    const int32_t *__restrict__ dst_table, int dst_pages,
                    float *__restrict__ weight_out,
                    int32_t *__restrict__ lengths_out) {
    wait_for_stream();
    constexpr int C = D / 8, R = kWrThreads / C, NP = kCacheTile / R;
    __shared__ float tmp[kWrThreads / 32];
    __shared__ float sh[kWrThreads / 32][2][D];
    const int tid = threadIdx.x, h = blockIdx.y, b = blockIdx.z >> 1;
    const bool keys = (blockIdx.z & 1) == 0;
    const int n = count[b], p = blockIdx.x, p0 = p * c.ps;
    if (keys && p == 0 && h == 0 && tid == 0) lengths_out[b] = n;
    if (p0 >= n) return;
    const size_t bh = (size_t)b * c.Hkv + h;
    const int rows = min(c.ps, n - p0);
    const int32_t *from = kept + bh * keep + p0;
    const size_t cap = (size_t)c.max_pages * c.ps;
    if (!keys && tid < rows)
        weight_out[bh * dst_pages * c.ps + p0 + tid] =
            weight[bh * cap + from[tid]];
    const int id =
        checked_page(c, dst_table[(size_t)b * dst_pages + p], b, p);
    if (id < 0) return;
    const size_t ph = (size_t)id * c.Hkv + h;
    const uint8_t *pool = keys ? c.k : c.v;
    const float *scales = keys ? c.ks : c.vs;
    const int ch = tid % C, rr = tid / C;

    uint2 raw[NP];
    float sc[NP];
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = i * R + rr;
        raw[i] = make_uint2(0, 0);
        sc[i] = 0.0f;
        if (r < rows) {
            const int j = from[r], src = page_id(c, b, j / c.ps);
            if (src >= 0) {
                const size_t sh_ = (size_t)src * c.Hkv + h;
                raw[i] = *(const uint2 *)(pool +
                                          (sh_ * c.ps + j % c.ps) * D + ch * 8);
                sc[i] = scales[sh_];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        float y[8];
        from_e4m3x4(raw[i].x, y);
        from_e4m3x4(raw[i].y, y + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            amax = fmaxf(amax, magnitude(y[j] * sc[i]));
    }
    const int e = page_exponent(block_max(amax, tmp));
    float hi[8], lo[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        hi[j] = -INFINITY;
        lo[j] = INFINITY;
    }
    uint8_t *codes = (keys ? c.k : c.v) + ph * c.ps * D;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int r = i * R + rr;
        if (r < rows) {
            float y[8];
            from_e4m3x4(raw[i].x, y);
            from_e4m3x4(raw[i].y, y + 4);
            // a code that is not 0 has sc 2^-e <= 2^17; the clip keeps 0 from
            // meeting an infinity
            *(uint2 *)(codes + (size_t)r * D + ch * 8) =
                encode8(y, fminf(sc[i] * pow2(-e), 0x1p20f), keys, hi, lo);
        }
    }
    if (keys) {
        float u, l;
        channel_extremes<D>(hi, lo, sh, u, l);
        if (tid < D) {
            int8_t *at = c.bounds + ph * 2 * D + tid;
            at[0] = bound(ceilf(u * 0.25f));
            at[D] = bound(floorf(l * 0.25f));
        }
    }
    if (tid == 0) (keys ? c.ks : c.vs)[ph] = pow2(e);
}

}  // namespace

cudaError_t launch_cache_append(const CacheView &c, const void *k,
                                const void *v, cudaStream_t st) {
    const dim3 grid((c.T + c.ps - 2) / c.ps + 1, c.Hkv, 2 * c.B);
    auto go = [&](auto t, auto dd) {
        using T = decltype(t);
        return launch_after(k_cache_append<T, decltype(dd)::value>, grid,
                            kWrThreads, 0, st, c, (const T *)k, (const T *)v);
    };
    auto by_d = [&](auto t) {
        switch (c.d) {
            case 32: return go(t, std::integral_constant<int, 32>{});
            case 64: return go(t, std::integral_constant<int, 64>{});
            default: return go(t, std::integral_constant<int, 128>{});
        }
    };
    return c.dtype == ELSAA_FP32 ? by_d(0.0f) : by_d(__nv_bfloat16{});
}

cudaError_t launch_cache_compact(const CacheView &c, const float *weight,
                                 int keep, const int32_t *kept,
                                 const int *count, const int32_t *dst_table,
                                 int dst_pages, float *weight_out,
                                 int32_t *lengths_out, cudaStream_t st) {
    const dim3 grid((keep + c.ps - 1) / c.ps, c.Hkv, 2 * c.B);
    auto go = [&](auto dd) {
        return launch_after(k_cache_compact<decltype(dd)::value>, grid,
                            kWrThreads, 0, st, c, weight, keep, kept, count,
                            dst_table, dst_pages, weight_out, lengths_out);
    };
    switch (c.d) {
        case 32: return go(std::integral_constant<int, 32>{});
        case 64: return go(std::integral_constant<int, 64>{});
        default: return go(std::integral_constant<int, 128>{});
    }
}

}  // namespace elsaa
