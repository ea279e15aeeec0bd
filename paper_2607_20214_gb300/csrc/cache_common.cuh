// Device helpers of the cache kernels: lengths and pages as the device finds
// them, powers of two, e4m3 conversions, the division of tiles over CTAs.
#pragma once

#include <atomic>

#include "cache.h"
#include "cache_division.h"
#include "device_common.cuh"
#include "tc_common.cuh"

namespace elsaa {
namespace cache {

// Launch of kernel K as launch_after does it, in clusters of `cluster` CTAs
// along x. `most`: the largest dynamic shared memory that it is launched with,
// allowed once for every device (asking each time is a tenth of a launch).
template <auto K, typename... A>
cudaError_t launch_cache(dim3 grid, int threads, size_t smem, size_t most,
                         int cluster, cudaStream_t st, A... args) {
    static std::atomic<unsigned long long> allowed{0};
    if (most > 0) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return taken(e);
        const unsigned long long bit = 1ull << (dev & 63);
        if (dev > 63 || !(allowed.load(std::memory_order_relaxed) & bit)) {
            e = cudaFuncSetAttribute(
                K, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
            if (e != cudaSuccess) return taken(e);
            allowed.fetch_or(bit, std::memory_order_relaxed);
        }
    }
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
    return taken(cudaLaunchKernelEx(&cfg, K, args...));
}

// The launch behind this one may be set up once every CTA of this one runs: it
// finds what this one left behind its own wait_for_stream(). The kernels begin
// with it (one K/V head of 16384 tokens: 11.6 -> 11.2 us, page selection with
// its attention 23.8 -> 23.1, eviction 32.4 -> 31.1), except k_cache_append,
// and k_cache_attn_simt with its merge: behind those the waiting CTAs cost more
// than their start (append 4.6 -> 4.7, fp32 attention 10.2 -> 10.9).
__device__ __forceinline__ void let_next_launch() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Out of line: faults are rare, and the code before a kernel's first loads is
// fetched while nothing else runs.
static __device__ __noinline__ void report_rare(DeviceStatus *st, int code,
                                                int where, int a, int b) {
    report(st, code, where, a, b);
}

// Tokens of sequence b, clipped to its table row, and its new tokens. Both
// loads are issued before one is looked at: a kernel's first loads are on its
// critical path.
struct Lengths {
    int len, n;
};
__device__ __forceinline__ Lengths lengths(const CacheView &c, int b) {
    Lengths x = {c.lengths[b], c.new_len ? c.new_len[b] : c.T};
    const int cap = c.max_pages * c.ps;
    if (x.len < 0 || x.len > cap) {
        report_rare(c.status, kDevCacheLength, b, x.len, cap);
        x.len = x.len < 0 ? 0 : cap;
    }
    if (x.n < 0 || x.n > c.T) {
        report_rare(c.status, kDevCacheLength, b, x.n, c.T);
        x.n = x.n < 0 ? 0 : c.T;
    }
    return x;
}

// A page of the pool, or -1.
__device__ __forceinline__ int checked_page(const CacheView &c, int id, int b,
                                            int p) {
    if ((unsigned)id < (unsigned)c.num_pages) return id;
    report_rare(c.status, kDevCachePage, b, p, id);
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

// Shared-memory lines of LINE = 32, 64 or 128 bytes with the swizzle of that
// width: where the 16-byte chunk c of line r lies.
template <int LINE>
__host__ __device__ __forceinline__ uint32_t line_offset(int r, int c) {
    constexpr int PER = LINE / 16;  // chunks of a line; 8 / PER lines a row
    return (uint32_t)(r * LINE + ((c ^ ((r / (8 / PER)) & (PER - 1))) << 4));
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
// ceil(rows / kCacheTile) tiles (one at least, so that a query without keys
// gets its row). An item costs its tiles and, for its queries and its end,
// about as much as kItemCost more (8000 cycles where a tile of 16 columns
// takes 2000): 8 drafted sequences, some of a single token, took 35 us with
// ranges of equal tiles, whose slowest CTA had six items. So the units tiles +
// kItemCost of all items, one after the other, are cut into equal ranges, one
// per CTA; an item that a cut crosses is written as pieces and merged
// afterwards. Every CTA finds its range by itself from the lengths: a launch
// that did it for all cost more than the B loads and the scan. (Cuts at whole
// steps of two tiles only were a wash: 8 heads of 1024 tokens 8.9 -> 8.5 us, 32
// of 16384 tokens 30.1 -> 30.4.)

// What a sequence's heads walk.
struct Seq {
    int len, n;  // tokens held, new ones
    int walk;    // tokens, or rows of listed pages
    int tiles;   // of a head's item; 0 without queries
};
__device__ __forceinline__ Seq sequence(const CacheAttn &A, int b) {
    const Lengths x = lengths(A.c, b);
    Seq s;
    s.len = x.len;
    s.n = x.n;
    s.walk = A.pages ? min((s.len + A.c.ps - 1) / A.c.ps, A.n_sel) * A.c.ps
                     : s.len;
    s.tiles =
        s.n == 0 ? 0 : max(1, (s.walk + kCacheTile - 1) / kCacheTile);
    return s;
}

// Whole items (A.whole) are a unit each instead, and none is cut.
__device__ __forceinline__ int units(const CacheAttn &A, int tiles) {
    return tiles == 0 ? 0 : A.whole ? 1 : tiles + kItemCost;
}

struct Start {
    int b, hc, off;  // sequence, head and group, first tile of that item
    int count;       // tiles of this CTA
};

// The sequences from the CTA's first on, as far as they fit.
constexpr int kNearSeqs = 32;

// The cuts of a call whose sequences have `sum` units in all for each of their
// items, `items` of them some.
__device__ __forceinline__ Cut cuts(const CacheAttn &A, int sum, int items) {
    return Cut((unsigned)sum, (unsigned)items,
               (unsigned)(A.c.Hkv * A.groups), (unsigned)A.ctas, A.whole);
}
// Unit u in a sequence with items of n > 0 tiles, whose units begin at a:
// its item there (HC: the one behind the last), tiles of that item before u,
// and tiles of all items before u; `before`: those of the sequences before.
struct Place {
    unsigned hc, off, tiles;
    __device__ __forceinline__ Place(const CacheAttn &A, int n, unsigned a,
                                     unsigned u, unsigned before) {
        const unsigned each = units(A, n), in = u - a;
        hc = in / each;
        const unsigned r = in - hc * each;
        off = r > kItemCost ? r - kItemCost : 0;
        tiles = before + hc * n + off;
    }
};
// The item that goes on behind the range, if it begins in it: the thread's
// sequence has the range's end u1 (a < u1 <= its end), the range begins at u0.
__device__ __forceinline__ CacheSplit split_in(const CacheAttn &A,
                                               const Cut &cut, int b,
                                               const Seq &s, unsigned a,
                                               unsigned u0, unsigned u1) {
    const Place end(A, s.tiles, a, u1, 0);
    const unsigned each = units(A, s.tiles), i0 = a + end.hc * each;
    // its first tile is unit i0 + kItemCost; a range that begins before it
    // begins the item
    if (end.off == 0 || u0 > i0 + kItemCost) return {0, 0, 0, 0};
    return {b, (int)end.hc,
            (int)(cut.owner(i0 + each - 1) - blockIdx.x) + 1, s.n};
}
// Sums up to the lane's, over the warp.
__device__ __forceinline__ int upto_lane(int x) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    return x;
}

// More than 32 sequences: all NT threads of the CTA together, a sequence a
// thread (several, one after the other, beyond NT); near: kNearSeqs entries.
template <int NT>
__device__ __noinline__ Start divide_many(const CacheAttn &A, Seq *near) {
    __shared__ int warps[NT / 32], some[NT / 32];
    __shared__ Start mine;  // its count: tiles before the range
    __shared__ int to;      // and before its end
    const CacheView &c = A.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rounds = (c.B + NT - 1) / NT, HC = c.Hkv * A.groups;
    Seq own = {0, 0, 0, 0};
    int done = 0;  // tiles of the round's sequences up to the thread's
    // their units
    auto sum = [&](int round) {
        const int b = round * NT + tid;
        own = {0, 0, 0, 0};
        if (b < c.B) own = sequence(A, b);
        const int live = __popc(__ballot_sync(0xffffffffu, own.tiles > 0));
        int x = upto_lane(units(A, own.tiles));
        done = upto_lane(own.tiles);
        __syncthreads();  // the round before has read
        if (lane == 31) {
            warps[warp] = x;
            some[warp] = live;
        }
        __syncthreads();
        for (int w = 0; w < warp; ++w) {
            x += warps[w];
            done += warps[w] - some[w] * kItemCost;
        }
        return x;
    };
    if (tid == 0) {
        mine = {0, 0, 0, 0};
        to = 0;
        A.split[blockIdx.x] = {0, 0, 0, 0};
    }
    int total = 0, items = 0, upto = 0;
    for (int r = 0; r < rounds; ++r) {
        upto = sum(r);
        for (int w = 0; w < NT / 32; ++w) {
            total += warps[w];
            items += some[w];
        }
    }
    const Cut cut = cuts(A, total, items);
    const unsigned k = blockIdx.x;
    const unsigned u0 = k < cut.n ? cut.at(k) : 0;
    const unsigned u1 = k < cut.n ? cut.at(k + 1) : 0;
    int base = 0, tiles = 0;
    for (int r = 0; r < rounds && k < cut.n; ++r) {
        if (rounds > 1) upto = sum(r);
        const unsigned z = (unsigned)(base + upto) * HC;
        const unsigned a = z - (unsigned)units(A, own.tiles) * HC;
        const unsigned before = (unsigned)(tiles + done - own.tiles) * HC;
        const int b = r * NT + tid;
        if (a <= u0 && u0 < z) {
            const Place p(A, own.tiles, a, u0, before);
            mine = {b, (int)p.hc, (int)p.off, (int)p.tiles};
        }
        if (a < u1 && u1 <= z) {
            to = (int)Place(A, own.tiles, a, u1, before).tiles;
            A.split[k] = split_in(A, cut, b, own, a, u0, u1);
        }
        if (rounds > 1)
            for (int w = 0; w < NT / 32; ++w) {
                base += warps[w];
                tiles += warps[w] - some[w] * kItemCost;
            }
    }
    __syncthreads();
    Start s = mine;
    s.count = to - s.count;
    if (tid < kNearSeqs && s.b + tid < c.B) near[tid] = sequence(A, s.b + tid);
    __syncthreads();
    return s;
}

// The CTA's range; its entry of A.split is written. Up to 32 sequences every
// warp finds it by itself, a sequence a lane (`own`, which Walk asks), so that
// no warp waits for another.
template <int NT>
__device__ __forceinline__ Start divide(const CacheAttn &A, Seq *near,
                                        Seq &own) {
    const CacheView &c = A.c;
    own = {0, 0, 0, 0};
    if (c.B > 32) return divide_many<NT>(A, near);
    const int lane = threadIdx.x & 31, HC = c.Hkv * A.groups;
    if (lane < c.B) own = sequence(A, lane);
    const int upto = upto_lane(units(A, own.tiles));
    const int done = upto_lane(own.tiles);
    const Cut cut = cuts(A, __shfl_sync(0xffffffffu, upto, 31),
                         __popc(__ballot_sync(0xffffffffu, own.tiles > 0)));
    const unsigned k = blockIdx.x;
    if (k >= cut.n) {
        if (threadIdx.x == 0) A.split[k] = {0, 0, 0, 0};
        return {0, 0, 0, 0};
    }
    const unsigned u0 = cut.at(k), u1 = cut.at(k + 1);
    const unsigned z = (unsigned)upto * HC;
    const unsigned a = z - (unsigned)units(A, own.tiles) * HC;
    const unsigned before = (unsigned)(done - own.tiles) * HC;
    if (threadIdx.x < 32 && a < u1 && u1 <= z)
        A.split[k] = split_in(A, cut, lane, own, a, u0, u1);
    // every lane evaluates both ends in the sequence that has them
    auto place = [&](unsigned u, int b) {
        return Place(A, __shfl_sync(0xffffffffu, own.tiles, b),
                     __shfl_sync(0xffffffffu, a, b), u,
                     __shfl_sync(0xffffffffu, before, b));
    };
    const int b0 = __ffs(__ballot_sync(0xffffffffu, a <= u0 && u0 < z)) - 1;
    const int b1 = __ffs(__ballot_sync(0xffffffffu, a < u1 && u1 <= z)) - 1;
    const Place p0 = place(u0, b0), p1 = place(u1, b1);
    return {b0, (int)p0.hc, (int)p0.off, (int)(p1.tiles - p0.tiles)};
}

// A CTA's share of one item.
struct alignas(16) Item {
    int b, h, col0, cols;   // sequence, K/V head, its columns of the G T
    int len, n, walk;       // as in Seq
    int off, count;         // tiles [off, off + count) of it
    int slot;               // -1: the whole item; else 0 if it began in an
                            // earlier CTA, 1 if here
};
// Walks the items of a CTA's range. Whole warps.
struct Walk {
    const Seq *near;
    Seq own;
    int b0, b, hc, off, left;
    __device__ __forceinline__ Walk(const Start &s, const Seq *n, const Seq &o)
        : near(n), own(o), b0(s.b), b(s.b), hc(s.hc), off(s.off),
          left(s.count) {}
    __device__ __forceinline__ Seq at(const CacheAttn &A, int b) const {
        if (A.c.B <= 32)
            return {__shfl_sync(0xffffffffu, own.len, b),
                    __shfl_sync(0xffffffffu, own.n, b),
                    __shfl_sync(0xffffffffu, own.walk, b),
                    __shfl_sync(0xffffffffu, own.tiles, b)};
        return b - b0 < kNearSeqs ? near[b - b0] : sequence(A, b);
    }
    __device__ __forceinline__ Item next(const CacheAttn &A) {
        Seq s = at(A, b);
        while (s.tiles == 0) s = at(A, ++b);  // left > 0: there is one
        Item it;
        it.b = b;
        it.h = hc / A.groups;
        it.col0 = hc % A.groups * A.cols;
        it.cols = min(A.cols, A.c.G * A.c.T - it.col0);
        it.len = s.len;
        it.n = s.n;
        it.walk = s.walk;
        it.off = off;
        it.count = min(s.tiles - off, left);
        it.slot = it.count == s.tiles ? -1 : off > 0 ? 0 : 1;
        left -= it.count;
        off = 0;
        if (++hc == A.c.Hkv * A.groups) {
            hc = 0;
            ++b;
        }
        return it;
    }
};

// The new token of column `col` < 128 (T at most 64: the product's error stays
// below 1 / T).
__device__ __forceinline__ int token_of(const CacheAttn &A, int col) {
    return col - A.c.T * (int)((unsigned)col * A.per_t >> 16);
}
// The last position that column `col` (g T + t) of an item sees, -1 if none
// or if the column is no query.
__device__ __forceinline__ int last_seen(const CacheAttn &A, int len, int n,
                                         int col) {
    const int t = token_of(A, col);
    return t < n ? len - n + t : -1;
}
// Row of q, o and lse of column `col`: a head's columns lie side by side.
__device__ __forceinline__ size_t query_row(const CacheAttn &A, int b, int h,
                                            int col) {
    return ((size_t)b * A.c.H + (size_t)h * A.c.G) * A.c.T + col;
}

__device__ __forceinline__ float *piece(const CacheAttn &A, int cta, int slot,
                                        int col) {
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
__device__ __forceinline__ void store_lse(const CacheAttn &A, int b, int h,
                                          int n, int col, float m, float l) {
    const float l2 = l == 0.0f ? -INFINITY : m + log2f(l);
    if (A.lse2)
        A.lse2[((size_t)b * A.c.Hkv + h) * A.c.G * A.c.T + col] = l2;
    if (A.lse && token_of(A, col) < n)
        A.lse[query_row(A, b, h, col)] = l2 * 0.6931471805599453f;
}

}  // namespace cache
}  // namespace elsaa
