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

// put(k, i) for the k-th selected index i, increasing.
template <int NT, typename K, typename P>
__device__ __forceinline__ void write_selected(K key, int n, uint32_t thr,
                                               int ties, TopkShared<NT> &S,
                                               P put) {
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
        if (take) put(at + __popc(mt & below), i + lane);
        at += __popc(mt);
        eq += __popc(me);
    }
}

// -------------------------------------------------------------- page scores
//
// A cluster per sequence and head: its CTAs score the pages, one a thread (the
// bounds of a page are 2 d bytes, sixteen 16-byte loads in flight a thread at
// d = 128), and leave the keys in the first CTA's shared memory, which
// selects. One launch; with the keys in HBM between two it was 10 us longer.
constexpr int kScThreads = 512;
constexpr int kScShared = 32768;  // keys that fit there
// Up to as many pages the rank of every key is counted directly.
constexpr int kScDirect = 128;

__device__ __forceinline__ void put_remote(uint32_t addr, uint32_t v) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(addr));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v)
                 : "memory");
}

// Queries as pairs of 8-bit rows max(qhat, 0), min(qhat, 0): with hi >= lo,
// max(q hi, q lo) = max(q, 0) hi + min(q, 0) lo.
template <typename T, int D>
__global__ void __launch_bounds__(kScThreads, 1)
    k_cache_select(const __grid_constant__ CacheView c,
                   const T *__restrict__ q, int n_sel, int first, int last,
                   int32_t *__restrict__ pages, uint32_t *__restrict__ keys,
                   int shared_keys) {
    wait_for_stream();
    extern __shared__ uint4 sq[];  // [queries][2][D / 16], then the keys
    __shared__ TopkShared<kScThreads> S;
    __shared__ float qscale[128];
    // a CTA's shared memory is written only once it runs
    if (gridDim.x > 1) tc::cluster_sync();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    const size_t bh = (size_t)b * c.Hkv + h;
    const int n = fresh(c, b), len = tokens(c, b);
    const int np = n == 0 ? 0 : (len + c.ps - 1) / c.ps;
    constexpr int W = D / 16;
    uint32_t *own = (uint32_t *)(sq + (size_t)c.G * c.T * 2 * W);
    uint4 hi[W], lo[W];
    float ks = 0.0f;
    int id = -1;
    auto fetch = [&](int p) {
        id = p < np ? page_id(c, b, p) : -1;
        if (id < 0) return;
        const size_t ph = (size_t)id * c.Hkv + h;
        const uint4 *at = (const uint4 *)(c.bounds + ph * 2 * D);
#pragma unroll
        for (int i = 0; i < W; ++i) {
            hi[i] = at[i];
            lo[i] = at[W + i];
        }
        ks = 4.0f * c.ks[ph];
    };
    int p = rank * kScThreads + tid;
    const int step = gridDim.x * kScThreads;
    if (rank * kScThreads < np) {
        fetch(p);
        // a warp quantises a query: D / 32 values a lane
        constexpr int V = D / 32;
        for (int r = warp; r < c.G * c.T; r += kScThreads / 32) {
            const T *x = q + ((bh * c.G) * c.T + r) * D + lane * V;
            float y[V], amax = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                y[i] = to_f32(x[i]);
                amax = fmaxf(amax, magnitude(y[i]));
            }
            const int e = query_exponent(warp_max(amax));
            const float f = pow2(-e);
            int8_t *at = (int8_t *)&sq[r * 2 * W] + lane * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int v = __float2int_rn(
                    fminf(fmaxf(y[i] * f, -127.0f), 127.0f));
                const int z = isnan(y[i]) ? 0 : v;
                at[i] = (int8_t)max(z, 0);
                at[D + i] = (int8_t)min(z, 0);
            }
            if (lane == 0) qscale[r] = r % c.T < n ? pow2(e) : -1.0f;
        }
        __syncthreads();
        while (p < np) {
            float best = -INFINITY;
            if (id >= 0) {
                for (int r = 0; r < c.G * c.T; ++r) {
                    const float f = qscale[r];
                    if (f < 0.0f) continue;  // no query
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
                    best = fmaxf(best, (float)s * f * ks);
                }
            }
            const bool must = p < first || p >= np - last;
            const uint32_t key = must ? kKeyFirst : order_key(best);
            if (!shared_keys)
                keys[bh * c.max_pages + p] = key;
            else if (rank == 0)
                own[p] = key;
            else
                put_remote(tc::smem_u32(own + p), key);
            p += step;
            fetch(p);
        }
    }
    if (gridDim.x > 1)
        tc::cluster_sync();
    else
        __syncthreads();
    if (rank > 0) return;
    const int m = min(np, n_sel);
    int32_t *out = pages + bh * n_sel;
    for (int i = m + tid; i < n_sel; i += kScThreads) out[i] = -1;
    if (m == 0) return;
    if (m == np) {
        for (int i = tid; i < np; i += kScThreads) out[i] = i;
        return;
    }
    const uint32_t *kk = shared_keys ? own : keys + bh * c.max_pages;
    auto key = [=](int i) { return kk[i]; };
    if (np <= kScDirect) {
        // rank of every key: the larger ones, and the equal ones before it
        bool take = false;
        if (tid < np) {
            const uint32_t mine = kk[tid];
            int above = 0;
            for (int i = 0; i < np; ++i) {
                const uint32_t x = kk[i];
                above += x > mine || (x == mine && i < tid);
            }
            take = above < m;
        }
        const uint32_t votes = __ballot_sync(0xffffffffu, take);
        if (lane == 0) S.warps[warp][0] = __popc(votes);
        __syncthreads();
        int at = __popc(votes & ((1u << lane) - 1));
        for (int w = 0; w < warp; ++w) at += S.warps[w][0];
        if (take) out[at] = tid;
        return;
    }
    uint32_t thr;
    int ties;
    find_threshold<kScThreads>(key, np, m, S, thr, ties);
    write_selected<kScThreads>(key, np, thr, ties, S,
                               [=](int k, int i) { out[k] = i; });
}

// ------------------------------------------------------------- kept tokens
//
// A CTA per sequence and head. The weights are read once, as many at a time
// as there are registers for, and their keys kept in shared memory (up to
// kKpShared tokens; longer rows are read again by every pass).
constexpr int kKpThreads = 1024;
constexpr int kKpShared = 49152;

__global__ void __launch_bounds__(kKpThreads)
    k_cache_keep(const __grid_constant__ CacheView c,
                 const float *__restrict__ weight, int keep, int recent,
                 const CacheKept out, int shared_keys) {
    wait_for_stream();
    extern __shared__ uint32_t own[];
    __shared__ TopkShared<kKpThreads> S;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const size_t bh = (size_t)b * c.Hkv + h;
    const int n = tokens(c, b), m = min(n, keep), safe = n - recent;
    const float *w = weight + bh * c.max_pages * c.ps;
    int32_t *kept = out.kept ? out.kept + bh * keep : nullptr;
    int32_t *rows = out.rows + bh * keep;
    float *wout = out.weight_out + bh * out.dst_pages * c.ps;
    if (h == 0 && tid == 0) out.count[b] = m;
    if (kept)
        for (int i = m + tid; i < keep; i += kKpThreads) kept[i] = -1;
    if (m == 0) return;
    // the rows' places are found here, where the reads of the table overlap
    auto put = [&](int k, int i) {
        const int id = page_id(c, b, i / c.ps);
        rows[k] = id < 0 ? -1 : id * c.ps + i % c.ps;
        wout[k] = w[i];
        if (kept) kept[k] = i;
    };
    if (m == n) {
        for (int i = tid; i < n; i += kKpThreads) put(i, i);
        return;
    }
    uint32_t thr;
    int ties;
    if (shared_keys) {
        constexpr int U = 8;
        for (int i0 = tid; i0 < n; i0 += U * kKpThreads) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kKpThreads;
                x[u] = i < n ? w[i] : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * kKpThreads;
                if (i < n) own[i] = i < safe ? order_key(x[u]) : kKeyFirst;
            }
        }
        __syncthreads();
        const uint32_t *kk = own;
        auto key = [=](int i) { return kk[i]; };
        find_threshold<kKpThreads>(key, n, m, S, thr, ties);
        write_selected<kKpThreads>(key, n, thr, ties, S, put);
    } else {
        auto key = [=](int i) {
            return i < safe ? order_key(w[i]) : kKeyFirst;
        };
        find_threshold<kKpThreads>(key, n, m, S, thr, ties);
        write_selected<kKpThreads>(key, n, thr, ties, S, put);
    }
}

// launch_after with clusters of `cluster` CTAs along x.
template <typename... K, typename... A>
cudaError_t launch_clusters(void (*kern)(K...), dim3 grid, int threads,
                            size_t smem, int cluster, cudaStream_t st,
                            A... args) {
    cudaError_t e = cudaFuncSetAttribute(
        kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return taken(e);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return taken(cudaLaunchKernelEx(&cfg, kern, K(args)...));
}

}  // namespace

cudaError_t launch_cache_select(const CacheView &c, const void *q, int n_sel,
                                int first, int last, int32_t *pages,
                                float *scores, cudaStream_t st) {
    // as many CTAs as have pages and SMs
    int cluster = 1;
    while (cluster < 8 && cluster * kScThreads < c.max_pages &&
           2L * cluster * c.B * c.Hkv <= 152)
        cluster *= 2;
    const int shared_keys = c.max_pages <= kScShared;
    const size_t smem = (size_t)c.G * c.T * 2 * c.d +
                        (shared_keys ? sizeof(uint32_t) * c.max_pages : 0);
    auto go = [&](auto t, auto dd) {
        using T = decltype(t);
        return launch_clusters(k_cache_select<T, decltype(dd)::value>,
                               dim3(cluster, c.Hkv, c.B), kScThreads, smem,
                               cluster, st, c, (const T *)q, n_sel, first,
                               last, pages, (uint32_t *)scores, shared_keys);
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

cudaError_t launch_cache_keep(const CacheView &c, const float *weight,
                              int keep, int recent, const CacheKept &out,
                              cudaStream_t st) {
    const long slots = (long)c.max_pages * c.ps;
    const int shared_keys = slots <= kKpShared;
    return launch_clusters(k_cache_keep, dim3(c.Hkv, c.B), kKpThreads,
                           shared_keys ? sizeof(uint32_t) * slots : 0, 1, st,
                           c, weight, keep, recent, out, shared_keys);
}

}  // namespace elsaa
