// Selection over the cache: the page scores and the best pages of
// elsaa_cache_select, and the tokens that elsaa_cache_evict keeps.
//
// Scores. A page's score bounds <q, k> over the box of its key codes; with
// query and bounds in 8 bits it is a sum of whole numbers below 2^24, times
// powers of two: exact in fp32, so equal scores are equal in every order of
// summation and the selection is defined to the last page.
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
    alignas(16) int hist[2][kBins];  // of a pass, and of the next
    int warps[NT / 32][2];
    int bin, above, count;  // the threshold's bin, keys above it and in it
    alignas(8) int taken[2];  // this CTA's keys above the threshold, equal
};

// Two neighbouring words of CTA `rank`'s shared memory.
__device__ __forceinline__ int2 get_remote(const int *p, int rank) {
    int2 v;
    asm volatile(
        "{\n .reg .b32 a;\n mapa.shared::cluster.u32 a, %2, %3;\n"
        " ld.shared::cluster.v2.s32 {%0, %1}, [a];\n}\n"
        : "=r"(v.x), "=r"(v.y)
        : "r"(tc::smem_u32(p)), "r"(rank));
    return v;
}
// Sum of v over the warps before this one, and over all; v: [W] of [2], the
// `which`-th. A whole warp.
template <int W>
__device__ __forceinline__ int sum_warps(const int (*v)[2], int which,
                                         int &all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = lane < W ? v[lane][which] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    all = __shfl_sync(0xffffffffu, x, 31);
    const int before = __shfl_sync(0xffffffffu, x, warp - 1);
    return warp == 0 ? 0 : before;
}
constexpr int kMaxCluster = 8;
// All threads of the cluster's `cs` CTAs.
__device__ __forceinline__ void sync_all(int cs) {
    if (cs > 1)
        tc::cluster_sync();
    else
        __syncthreads();
}

// Order-preserving key of a float: larger float, larger key; -0 as 0; NaN 0.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (isnan(x)) return 0u;
    const uint32_t u = __float_as_uint(x + 0.0f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
constexpr uint32_t kKeyFirst = 0xffffffffu;  // above every float's

// thr, ties: the m largest keys are those above thr and `ties` of those equal
// to it. n keys are this CTA's; the `cs` CTAs of a cluster (1: this one alone)
// count together and find the same threshold.
template <int NT, typename K>
__device__ __forceinline__ void find_threshold(K key, int n, int m, int cs,
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
        int *hist = S.hist[pass & 1];
#pragma unroll
        for (int i = 0; i < PER; ++i) hist[tid + i * NT] = 0;
        __syncthreads();
#pragma unroll 4
        for (int i = tid; i < n; i += NT) {
            const uint32_t u = key(i);
            if ((u & mask) == prefix)
                atomicAdd(&hist[(u >> shift) & digit], 1);
        }
        sync_all(cs);
        // thread t owns bins top - PER t ... downwards; `before`: keys in
        // the bins above its own. (The next pass counts elsewhere: another
        // CTA may still read here.)
        static_assert(PER % 2 == 0, "bins in pairs");
        int bins[PER], own = 0;  // top - PER t - i
        if (cs > 1) {
            int2 got[PER / 2][kMaxCluster];
#pragma unroll
            for (int i = 0; i < PER / 2; ++i)
#pragma unroll
                for (int r = 0; r < kMaxCluster; ++r)
                    got[i][r] =
                        r < cs ? get_remote(
                                     &hist[kBins - 2 - tid * PER - 2 * i], r)
                               : make_int2(0, 0);
#pragma unroll
            for (int i = 0; i < PER / 2; ++i) {
                bins[2 * i] = bins[2 * i + 1] = 0;
#pragma unroll
                for (int r = 0; r < kMaxCluster; ++r) {
                    bins[2 * i] += got[i][r].y;
                    bins[2 * i + 1] += got[i][r].x;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i)
                bins[i] = hist[kBins - 1 - (tid * PER + i)];
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) own += bins[i];
        int x = own, all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        if (lane == 31) S.warps[warp][0] = x;
        __syncthreads();
        const int before =
            x - own + sum_warps<NT / 32>(S.warps, 0, all);
        if (before < left && left <= before + own) {
            int a = before;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (a < left && left <= a + bins[i]) {
                    S.bin = kBins - 1 - (tid * PER + i);
                    S.above = a;
                    S.count = bins[i];
                }
                a += bins[i];
            }
        }
        __syncthreads();
        prefix |= (uint32_t)S.bin << shift;
        mask |= digit << shift;
        left -= S.above;
        if (S.count == left) {
            // the whole bin is selected: with distinct keys nearly always
            // before the last pass (there are other keys below: m < all)
            thr = prefix - 1;
            ties = 0;
            return;
        }
        __syncthreads();
    }
    thr = prefix;
    ties = left;
}

// put(k, i) for the k-th selected key i of this CTA's, increasing; k counts on
// from the selected keys of the cluster's CTAs before it. [k0, k1): this CTA's.
template <int NT, typename K, typename P>
__device__ __forceinline__ void write_selected(K key, int n, uint32_t thr,
                                               int ties, int cs, int rank,
                                               TopkShared<NT> &S, int &k0,
                                               int &k1, P put) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    constexpr int W = NT / 32;
    const int run = ((n + W - 1) / W + 31) & ~31;
    const int i0 = min(warp * run, n), i1 = min(i0 + run, n);
    int above = 0, equal = 0;
#pragma unroll 4
    for (int i = i0; i < i1; i += 32) {
        const bool in = i + lane < i1;
        const uint32_t u = in ? key(i + lane) : 0u;
        above += in && u > thr;
        equal += in && u == thr;
    }
    above = __reduce_add_sync(0xffffffffu, above);
    equal = __reduce_add_sync(0xffffffffu, equal);
    if (lane == 0) {
        S.warps[warp][0] = above;
        S.warps[warp][1] = equal;
    }
    __syncthreads();
    int all, alleq;
    int at = sum_warps<W>(S.warps, 0, all);
    int eq = sum_warps<W>(S.warps, 1, alleq);
    int a0 = 0, e0 = 0;  // of the CTAs before
    if (cs > 1) {
        if (threadIdx.x == 0) {
            S.taken[0] = all;
            S.taken[1] = alleq;
        }
        sync_all(cs);
        int2 got[kMaxCluster];
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r)
            got[r] = r < rank ? get_remote(S.taken, r) : make_int2(0, 0);
#pragma unroll
        for (int r = 0; r < kMaxCluster; ++r) {
            a0 += got[r].x;
            e0 += got[r].y;
        }
    }
    k0 = a0 + min(e0, ties);
    k1 = a0 + all + min(e0 + alleq, ties);
    eq += e0;
    at += a0 + min(eq, ties);
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
// A cluster per sequence and head: its CTAs score the pages, kScPages at a
// time, and leave the keys in the first CTA's shared memory, which selects.
// One launch, 9 us for 1024 pages of 64 heads of 128 (17 MB: dependent loads,
// the cluster's barrier and the counting bound it); with the keys in HBM
// between two launches it was 10 us longer. The bounds of a page are 2 d
// neighbouring bytes: they come by 16-byte asynchronous copies, so that a warp
// reads whole lines (a page a thread, straight into registers, took 7000
// cycles for 512 pages instead of 2000).
//
// The sums are small matrix products (16 pages x 8 queries x 2 d) of fp16
// numbers, which hold 8-bit ones and add up exactly in fp32: 4-byte integer
// products run at 16 lanes a cycle here, 3800 cycles for 256 pages and 4
// queries. The order along 2 d is free as long as both operands share it: a
// lane takes 16 neighbouring bytes for four steps.
constexpr int kScThreads = 512;
constexpr int kScPages = kScThreads / 2;
constexpr int kScShared = 16384;  // keys that fit in shared memory
// Up to as many pages the rank of every key is counted directly.
constexpr int kScDirect = 128;

// Four 8-bit integers as fp16 pairs: 1024 + u has u = v + 128 in its last bits.
__device__ __forceinline__ void halves(uint32_t w, uint32_t &a, uint32_t &b) {
    const uint32_t u = w ^ 0x80808080u;
    constexpr uint32_t k = 0xe480e480u;  // -(1024 + 128) twice
    asm("add.rn.f16x2 %0, %1, %2;"
        : "=r"(a)
        : "r"(__byte_perm(u, 0x64646464u, 0x4140)), "r"(k));
    asm("add.rn.f16x2 %0, %1, %2;"
        : "=r"(b)
        : "r"(__byte_perm(u, 0x64646464u, 0x4342)), "r"(k));
}
// c (16 x 8) += a (16 x 16) b (16 x 8).
__device__ __forceinline__ void mma_16x8(float (&c)[4], uint32_t a0,
                                         uint32_t a1, uint32_t a2, uint32_t a3,
                                         uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 "
        "{%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cluster_arrive() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void put_remote(uint32_t addr, uint32_t v) {
    uint32_t at;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(at) : "r"(addr));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v)
                 : "memory");
}

// Bytes between rows of 2 d bytes in shared memory: 64 more than a multiple of
// 128, so that eight lanes that read four pieces of two rows meet no bank
// twice.
__host__ __device__ constexpr int score_row(int d) {
    return d == 32 ? 64 : 2 * d + 64;
}

// Queries as pairs of 8-bit rows max(qhat, 0), min(qhat, 0): with hi >= lo,
// max(q hi, q lo) = max(q, 0) hi + min(q, 0) lo.
template <typename T, int D>
__global__ void __launch_bounds__(kScThreads, 2)
    k_cache_select(const __grid_constant__ CacheView c,
                   const T *__restrict__ q, int n_sel, int first, int last,
                   int32_t *__restrict__ pages, uint32_t *__restrict__ keys,
                   int shared_keys) {
    // the other CTAs' shared memory is written only once they run
    if (gridDim.x > 1) cluster_arrive();
    wait_for_stream();
    let_next_launch();
    // queries, a tile of bounds (rows of 2 D bytes), keys
    extern __shared__ uint4 sq[];
    __shared__ TopkShared<kScThreads> S;
    __shared__ float qscale[128], pscale[kScPages];
    __shared__ int ids[kScPages];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
    const size_t bh = (size_t)b * c.Hkv + h;
    const auto [len, n] = lengths(c, b);
    const int np = n == 0 ? 0 : (len + c.ps - 1) / c.ps;
    constexpr int W = D / 16, ROW = score_row(D) / 16;  // 16-byte pieces
    const int GT = c.G * c.T, GT8 = (GT + 7) & ~7;
    uint4 *tile = sq + GT8 * ROW;
    uint32_t *own = (uint32_t *)(tile + kScPages * ROW);
    const int step = gridDim.x * kScPages;
    for (int p0 = rank * kScPages; p0 < np; p0 += step) {
        if (tid < kScPages)
            ids[tid] = p0 + tid < np ? page_id(c, b, p0 + tid) : -1;
        __syncthreads();
        const int here = min(kScPages, np - p0);
        for (int i = tid; i < here * 2 * W; i += kScThreads) {
            const int id = ids[i / (2 * W)];
            if (id >= 0)
                tc::cp_async16(
                    tc::smem_u32(tile + i / (2 * W) * ROW + i % (2 * W)),
                    c.bounds + ((size_t)id * c.Hkv + h) * 2 * D +
                        i % (2 * W) * 16);
        }
        tc::cp_async_commit();
        if (tid < kScPages)
            pscale[tid] = ids[tid] < 0
                              ? 0.0f
                              : 4.0f * c.ks[(size_t)ids[tid] * c.Hkv + h];
        if (p0 == rank * kScPages) {
            // meanwhile a warp quantises a query: D / 32 values a lane
            constexpr int V = D / 32;
            for (int r = warp; r < GT; r += kScThreads / 32) {
                const T *x = q + (bh * GT + r) * D + lane * V;
                float y[V], amax = 0.0f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    y[i] = to_f32(x[i]);
                    amax = fmaxf(amax, magnitude(y[i]));
                }
                const int e = query_exponent(warp_max(amax));
                const float f = pow2(-e);
                int8_t *at = (int8_t *)&sq[r * ROW] + lane * V;
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
        }
        tc::cp_async_wait<0>();
        __syncthreads();
        if (p0 == rank * kScPages && gridDim.x > 1) cluster_wait();
        // a warp has 16 pages: a lane rows g and g + 8, columns 2 t, 2 t + 1
        const int g = lane >> 2, t = lane & 3, row = warp * 16 + g;
        float best[2] = {-INFINITY, -INFINITY};
        if (warp * 16 < here) {
            for (int r0 = 0; r0 < GT; r0 += 8) {
                float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
                for (int k = 0; k < 2 * W; k += 4) {
                    const uint4 a = tile[row * ROW + k + t];
                    const uint4 z = tile[(row + 8) * ROW + k + t];
                    const uint4 y = sq[(r0 + g) * ROW + k + t];
                    const uint32_t aw[4] = {a.x, a.y, a.z, a.w};
                    const uint32_t zw[4] = {z.x, z.y, z.z, z.w};
                    const uint32_t yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t a0, a1, a2, a3, b0, b1;
                        halves(aw[j], a0, a2);
                        halves(zw[j], a1, a3);
                        halves(yw[j], b0, b1);
                        mma_16x8(acc, a0, a1, a2, a3, b0, b1);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = r0 + 2 * t + (j & 1);
                    const float f = r < GT ? qscale[r] : -1.0f;
                    // the smaller factor first: what overflows then is larger
                    // than fp32 holds as a whole
                    const float s = pscale[row + 8 * (j >> 1)];
                    if (f >= 0.0f)
                        best[j >> 1] =
                            fmaxf(best[j >> 1],
                                  acc[j] * fminf(f, s) * fmaxf(f, s));
                }
            }
        }
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            best[x] = fmaxf(best[x], __shfl_xor_sync(0xffffffffu, best[x], 1));
            best[x] = fmaxf(best[x], __shfl_xor_sync(0xffffffffu, best[x], 2));
            const int i = row + 8 * x, p = p0 + i;
            if (t == 0 && p < np) {
                if (ids[i] < 0) best[x] = -INFINITY;
                const bool must = p < first || p >= np - last;
                const uint32_t key = must ? kKeyFirst : order_key(best[x]);
                if (!shared_keys)
                    keys[bh * c.max_pages + p] = key;
                else if (rank == 0)
                    own[p] = key;
                else
                    put_remote(tc::smem_u32(own + p), key);
            }
        }
        __syncthreads();
    }
    if (gridDim.x > 1) {
        if (rank * kScPages >= np) cluster_wait();  // of the start
        tc::cluster_sync();
    } else {
        __syncthreads();
    }
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
    int ties, k0, k1;
    find_threshold<kScThreads>(key, np, m, 1, S, thr, ties);
    write_selected<kScThreads>(key, np, thr, ties, 1, 0, S, k0, k1,
                               [=](int k, int i) { out[k] = i; });
}

// ------------------------------------------------------------- kept tokens
//
// A CTA per sequence and head, or for long rows of few sequences a cluster,
// whose CTAs have a run of the tokens each. Counting together costs a CTA 3500
// cycles a pass, as much as the keys of 16384 tokens by itself, so only longer
// rows are shared. The weights are read once, as many at a time as
// there are registers for, and their keys kept in shared memory (up to
// kKpShared a CTA; longer runs are read again by every pass). 32 rows of 16384
// weights take 13 us, a chain of barriers and dependent shared-memory reads.
constexpr int kKpThreads = 1024;
constexpr int kKpShared = 49152;

__global__ void __launch_bounds__(kKpThreads)
    k_cache_keep(const __grid_constant__ CacheView c,
                 const float *__restrict__ weight, int keep, int recent,
                 const CacheKept out, int shared_keys) {
    wait_for_stream();
    let_next_launch();
    extern __shared__ uint32_t own[];
    __shared__ TopkShared<kKpThreads> S;
    const int cs = gridDim.x, rank = blockIdx.x;
    const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const size_t bh = (size_t)b * c.Hkv + h;
    const int n = lengths(c, b).len, m = min(n, keep);
    const float *w = weight + bh * c.max_pages * c.ps;
    int32_t *kept = out.kept ? out.kept + bh * keep : nullptr;
    int32_t *rows = out.rows + bh * keep;
    float *wout = out.weight_out + bh * out.dst_pages * c.ps;
    if (h == 0 && rank == 0 && tid == 0) out.count[b] = m;
    if (kept && rank == 0)
        for (int i = m + tid; i < keep; i += kKpThreads) kept[i] = -1;
    // this CTA's tokens [j0, j1)
    const int run = ((n + cs - 1) / cs + 31) & ~31;
    const int j0 = min(rank * run, n), j1 = min(j0 + run, n);
    const int own_n = j1 - j0, safe = n - recent - j0;
    int k0 = j0, k1 = j1;
    auto put = [=](int k, int i) { rows[k] = j0 + i; };
    if (m == n) {
        for (int i = tid; i < own_n; i += kKpThreads) put(j0 + i, i);
    } else {
        uint32_t thr;
        int ties;
        const float *wj = w + j0;
        if (shared_keys) {
            constexpr int U = 8;
            for (int i0 = tid; i0 < own_n; i0 += U * kKpThreads) {
                float x[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * kKpThreads;
                    x[u] = i < own_n ? wj[i] : 0.0f;
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i0 + u * kKpThreads;
                    if (i < own_n)
                        own[i] = i < safe ? order_key(x[u]) : kKeyFirst;
                }
            }
            __syncthreads();
            const uint32_t *kk = own;
            auto key = [=](int i) { return kk[i]; };
            find_threshold<kKpThreads>(key, own_n, m, cs, S, thr, ties);
            write_selected<kKpThreads>(key, own_n, thr, ties, cs, rank, S, k0,
                                       k1, put);
        } else {
            auto key = [=](int i) {
                return i < safe ? order_key(wj[i]) : kKeyFirst;
            };
            find_threshold<kKpThreads>(key, own_n, m, cs, S, thr, ties);
            write_selected<kKpThreads>(key, own_n, thr, ties, cs, rank, S, k0,
                                       k1, put);
        }
    }
    __syncthreads();
    // positions to places in the pool, with the weights, several at a time
    constexpr int U = 4;
    for (int q = k0 + tid; q < k1; q += U * kKpThreads) {
        int i[U], id[U];
        float x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = q + u * kKpThreads;
            i[u] = k < k1 ? rows[k] : 0;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            id[u] = c.table[(size_t)b * c.max_pages + i[u] / c.ps];
            x[u] = w[i[u]];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = q + u * kKpThreads;
            if (k >= k1) break;
            id[u] = checked_page(c, id[u], b, i[u] / c.ps);
            rows[k] = id[u] < 0 ? -1 : id[u] * c.ps + i[u] % c.ps;
            wout[k] = x[u];
            if (kept) kept[k] = i[u];
        }
    }
    // another CTA may still read this one's counts
    if (cs > 1) tc::cluster_sync();
}

}  // namespace

cudaError_t launch_cache_select(const CacheView &c, const void *q, int n_sel,
                                int first, int last, int32_t *pages,
                                float *scores, cudaStream_t st) {
    // as many CTAs as have pages and, two an SM, find a place
    int cluster = 1;
    while (cluster < kMaxCluster && cluster * kScPages < c.max_pages &&
           2L * cluster * c.B * c.Hkv <= 304)
        cluster *= 2;
    const int shared_keys = c.max_pages <= kScShared;
    const size_t smem = (size_t)(((c.G * c.T + 7) & ~7) + kScPages) *
                            score_row(c.d) +
                        (shared_keys ? sizeof(uint32_t) * c.max_pages : 0);
    auto go = [&](auto t, auto dd) {
        using T = decltype(t);
        constexpr int D = decltype(dd)::value;
        return launch_cache<k_cache_select<T, D>>(
            dim3(cluster, c.Hkv, c.B), kScThreads, smem,
            (128 + kScPages) * score_row(D) + sizeof(uint32_t) * kScShared,
            cluster, st, c, (const T *)q, n_sel, first, last, pages,
            (uint32_t *)scores, shared_keys);
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
    int cluster = 1;
    while (cluster < kMaxCluster && 16384L * cluster < slots &&
           2L * cluster * c.B * c.Hkv <= 152)
        cluster *= 2;
    const long run = ((slots + cluster - 1) / cluster + 31) / 32 * 32;
    const int shared_keys = run <= kKpShared;
    return launch_cache<k_cache_keep>(
        dim3(cluster, c.Hkv, c.B), kKpThreads,
        shared_keys ? sizeof(uint32_t) * run : 0, sizeof(uint32_t) * kKpShared,
        cluster, st, c, weight, keep, recent, out, shared_keys);
}

}  // namespace elsaa
