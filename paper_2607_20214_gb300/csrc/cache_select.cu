// Selection over the cache: the page scores and the best pages of
// elsaa_cache_select, and the tokens that elsaa_cache_evict keeps.
//
// Scores. A page's score bounds <q, k> over the box of its key codes; with
// query and bounds in 8 bits it is a sum of whole numbers below 2^24 (four
// products a lane and instruction), times powers of two: exact, so equal
// scores are equal in every order of summation and the selection is defined
// to the last page.
//
// Selection. The m largest of n keys by three counting passes over digits of
// 11, 11 and 10 bits (a digit of 11 bits takes sign, exponent and two bits of
// the mantissa of a float, so that weights of a few binades spread over many
// counters), then one ordered pass that writes the indices, increasing. Ties
// go to the lower index: every warp owns a run of indices and learns from the
// counts of the warps before it how many ties are left.
#include "cache_common.cuh"

namespace elsaa {

namespace {

using namespace cache;

constexpr int kBins = 2048;

template <int NT>
struct TopkShared {
    int hist[kBins];
    int warps[NT / 32][2];
    int bin, above;
};

// Order-preserving key of a float: larger float, larger key; -0 as 0; NaN 0.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (isnan(x)) return 0u;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
constexpr uint32_t kKeyFirst = 0xffffffffu;  // above every float's

// thr, ties: the m largest of key(0 .. n - 1), 1 <= m <= n, are those above
// thr and `ties` of those equal to it.
template <int NT, typename K>
__device__ __forceinline__ void find_threshold(K key, int n, int m,
                                               TopkShared<NT> &S,
                                               uint32_t &thr, int &ties) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int PER = kBins / NT;
    uint32_t prefix = 0, mask = 0;
    int left = m;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digit = pass == 2 ? 0x3ffu : 0x7ffu;
#pragma unroll
        for (int i = 0; i < PER; ++i) S.hist[tid + i * NT] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += NT) {
            const uint32_t u = key(i);
            if ((u & mask) == prefix)
                atomicAdd(&S.hist[(u >> shift) & digit], 1);
        }
        __syncthreads();
        // thread t owns bins top - PER t ... downwards; `before`: keys in
        // the bins above its own
        int own = 0, x;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            own += S.hist[kBins - 1 - (tid * PER + i)];
        x = own;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) S.warps[warp][0] = x;
        __syncthreads();
        int before = x - own;
        for (int w = 0; w < warp; ++w) before += S.warps[w][0];
        if (before < left && left <= before + own) {
            int a = before;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int bin = kBins - 1 - (tid * PER + i);
                const int c = S.hist[bin];
                if (a < left && left <= a + c) {
                    S.bin = bin;
                    S.above = a;
                }
                a += c;
            }
        }
        __syncthreads();
        prefix |= (uint32_t)S.bin << shift;
        mask |= digit << shift;
        left -= S.above;
        __syncthreads();
    }
    thr = prefix;
    ties = left;
}

// Writes the selected indices, increasing, to out[0 .. m).
template <int NT, typename K>
__device__ __forceinline__ void write_selected(K key, int n, uint32_t thr,
                                               int ties, TopkShared<NT> &S,
                                               int32_t *out) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int W = NT / 32;
    const int run = ((n + W - 1) / W + 31) & ~31;
    const int i0 = min(warp * run, n), i1 = min(i0 + run, n);
    int above = 0, equal = 0;
    for (int i = i0; i < i1; i += 32) {
        const uint32_t u = i + lane < i1 ? key(i + lane) : 0u;
        const bool in = i + lane < i1;
        above += __popc(__ballot_sync(0xffffffffu, in && u > thr));
        equal += __popc(__ballot_sync(0xffffffffu, in && u == thr));
    }
    if (lane == 0) {
        S.warps[warp][0] = above;
        S.warps[warp][1] = equal;
    }
    __syncthreads();
    int at = 0, eq = 0;
    for (int w = 0; w < warp; ++w) {
        at += S.warps[w][0];
        eq += S.warps[w][1];
    }
    at += min(eq, ties);
    const uint32_t below = (1u << lane) - 1;
    for (int i = i0; i < i1; i += 32) {
        const bool in = i + lane < i1;
        const uint32_t u = in ? key(i + lane) : 0u;
        const uint32_t me = __ballot_sync(0xffffffffu, in && u == thr);
        const bool take = in && (u > thr || (u == thr &&
                                             eq + __popc(me & below) < ties));
        const uint32_t mt = __ballot_sync(0xffffffffu, take);
        if (take) out[at + __popc(mt & below)] = i + lane;
        at += __popc(mt);
        eq += __popc(me);
    }
}

// -------------------------------------------------------------- page scores

constexpr int kScThreads = 128;  // one page a thread

// Queries as pairs of 8-bit rows max(qhat, 0), min(qhat, 0): with hi >= lo,
// max(q hi, q lo) = max(q, 0) hi + min(q, 0) lo.
template <typename T, int D>
__global__ void __launch_bounds__(kScThreads)
    k_cache_scores(CacheView c, const T *__restrict__ q, int first, int last,
                   uint32_t *__restrict__ keys) {
    wait_for_stream();
    extern __shared__ uint4 sq[];  // [queries][2][D / 16]
    __shared__ float qscale[128];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int h = blockIdx.y, b = blockIdx.z;
    const int n = fresh(c, b), len = tokens(c, b);
    const int pages = (len + c.ps - 1) / c.ps;
    const int p = blockIdx.x * kScThreads + tid;
    if (n == 0 || blockIdx.x * kScThreads >= pages) return;
    const int id = p < pages ? page_id(c, b, p) : -1;
    constexpr int W = D / 16;
    uint4 hi[W], lo[W];
    float ks = 0.0f;
    if (id >= 0) {
        const size_t ph = (size_t)id * c.Hkv + h;
        const uint4 *at = (const uint4 *)(c.bounds + ph * 2 * D);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            hi[i] = at[i];
            lo[i] = at[W + i];
        }
        ks = 4.0f * c.ks[ph];
    }
    // a warp quantises a query: D / 32 values a lane
    constexpr int V = D / 32;
    int rows = 0;
    for (int g = 0; g < c.G; ++g)
        for (int t = 0; t < n; ++t, ++rows) {
            if (rows % (kScThreads / 32) != warp) continue;
            const T *x = q + (((size_t)b * c.H + (size_t)h * c.G + g) * c.T + t) * D + lane * V;
            float y[V], amax = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                y[i] = to_f32(x[i]);
                amax = fmaxf(amax, magnitude(y[i]));
            }
            const int e = query_exponent(warp_max(amax));
            const float f = pow2(-e);
            int8_t *at = (int8_t *)&sq[rows * 2 * W] + lane * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int v = __float2int_rn(
                    fminf(fmaxf(y[i] * f, -127.0f), 127.0f));
                const int z = isnan(y[i]) ? 0 : v;
                at[i] = (int8_t)max(z, 0);
                at[D + i] = (int8_t)min(z, 0);
            }
            if (lane == 0) qscale[rows] = pow2(e);
        }
    __syncthreads();
    if (p >= pages) return;
    float best = -INFINITY;
    if (id >= 0) {
        for (int r = 0; r < rows; ++r) {
            int s = 0;
            const uint4 *a = sq + r * 2 * W;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const uint4 u = a[i], v = a[W + i];
                s = __dp4a((int)u.x, (int)hi[i].x, s);
                s = __dp4a((int)u.y, (int)hi[i].y, s);
                s = __dp4a((int)u.z, (int)hi[i].z, s);
                s = __dp4a((int)u.w, (int)hi[i].w, s);
                s = __dp4a((int)v.x, (int)lo[i].x, s);
                s = __dp4a((int)v.y, (int)lo[i].y, s);
                s = __dp4a((int)v.z, (int)lo[i].z, s);
                s = __dp4a((int)v.w, (int)lo[i].w, s);
            }
            best = fmaxf(best, (float)s * qscale[r] * ks);
        }
    }
    const bool must = p < first || p >= pages - last;
    keys[((size_t)b * c.Hkv + h) * c.max_pages + p] =
        must ? kKeyFirst : order_key(best);
}

constexpr int kSpThreads = 256;

__global__ void __launch_bounds__(kSpThreads)
    k_cache_pages(CacheView c, const uint32_t *__restrict__ keys, int n_sel,
                  int32_t *__restrict__ pages) {
    wait_for_stream();
    __shared__ TopkShared<kSpThreads> S;
    const int h = blockIdx.x, b = blockIdx.y;
    const size_t bh = (size_t)b * c.Hkv + h;
    const int n = fresh(c, b) > 0 ? (tokens(c, b) + c.ps - 1) / c.ps : 0;
    const int m = min(n, n_sel);
    int32_t *out = pages + bh * n_sel;
    for (int i = m + threadIdx.x; i < n_sel; i += kSpThreads) out[i] = -1;
    if (m == 0) return;
    const uint32_t *kk = keys + bh * c.max_pages;
    if (m == n) {
        for (int i = threadIdx.x; i < n; i += kSpThreads) out[i] = i;
        return;
    }
    auto key = [=](int i) { return kk[i]; };
    uint32_t thr;
    int ties;
    find_threshold<kSpThreads>(key, n, m, S, thr, ties);
    write_selected<kSpThreads>(key, n, thr, ties, S, out);
}

// ------------------------------------------------------------- kept tokens

constexpr int kKpThreads = 1024;

__global__ void __launch_bounds__(kKpThreads)
    k_cache_keep(CacheView c, const float *__restrict__ weight, int keep,
                 int recent, int32_t *__restrict__ kept,
                 int *__restrict__ count) {
    wait_for_stream();
    __shared__ TopkShared<kKpThreads> S;
    const int h = blockIdx.x, b = blockIdx.y;
    const size_t bh = (size_t)b * c.Hkv + h;
    const int n = tokens(c, b), m = min(n, keep), safe = n - recent;
    int32_t *out = kept + bh * keep;
    if (h == 0 && threadIdx.x == 0) count[b] = m;
    for (int i = m + threadIdx.x; i < keep; i += kKpThreads) out[i] = -1;
    if (m == 0) return;
    if (m == n) {
        for (int i = threadIdx.x; i < n; i += kKpThreads) out[i] = i;
        return;
    }
    const float *w = weight + bh * c.max_pages * c.ps;
    auto key = [=](int i) { return i < safe ? order_key(w[i]) : kKeyFirst; };
    uint32_t thr;
    int ties;
    find_threshold<kKpThreads>(key, n, m, S, thr, ties);
    write_selected<kKpThreads>(key, n, thr, ties, S, out);
}

}  // namespace

cudaError_t launch_cache_select(const CacheView &c, const void *q, int n_sel,
                                int first, int last, int32_t *pages,
                                float *scores, cudaStream_t st) {
    const dim3 grid((c.max_pages + kScThreads - 1) / kScThreads, c.Hkv, c.B);
    const size_t smem = (size_t)c.G * c.T * 2 * c.d;
    uint32_t *keys = (uint32_t *)scores;
    auto go = [&](auto t, auto dd) {
        using T = decltype(t);
        return launch_after(k_cache_scores<T, decltype(dd)::value>, grid,
                            kScThreads, smem, st, c, (const T *)q, first,
                            last, keys);
    };
    auto by_d = [&](auto t) {
        switch (c.d) {
            case 32: return go(t, std::integral_constant<int, 32>{});
            case 64: return go(t, std::integral_constant<int, 64>{});
            default: return go(t, std::integral_constant<int, 128>{});
        }
    };
    const cudaError_t e =
        c.dtype == ELSAA_FP32 ? by_d(0.0f) : by_d(__nv_bfloat16{});
    if (e != cudaSuccess) return e;
    return launch_after(k_cache_pages, dim3(c.Hkv, c.B), kSpThreads, 0, st, c,
                        (const uint32_t *)keys, n_sel, pages);
}

cudaError_t launch_cache_keep(const CacheView &c, const float *weight,
                              int keep, int recent, int32_t *kept, int *count,
                              cudaStream_t st) {
    return launch_after(k_cache_keep, dim3(c.Hkv, c.B), kKpThreads, 0, st, c,
                        weight, keep, recent, kept, count);
}

}  // namespace elsaa
