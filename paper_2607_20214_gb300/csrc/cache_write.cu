// Writes into the 8-bit cache: elsaa_cache_append (rows of new tokens) and
// the second half of elsaa_cache_evict (the kept rows to other pages).
//
// A page of one head, keys or values, belongs to ps d / 64 threads of a CTA,
// each with E channels of 64 / E rows, so the page's exponent is one reduction
// away and every byte moves once: rows are read into registers, their largest
// magnitude gives the exponent e, and codes e4m3(x 2^-e) go out. Scaling by a
// power of two is exact, so the only rounding is the conversion's. What bounds
// it is HBM, if enough pages are in flight: small pages share a CTA, and every
// dependent read (length, table entry, position) is issued for all four rows
// before one is used. A prompt of 2 x 16 heads x 16384 rows of 128: 65 us, 6.1
// TB/s (8 channels a thread; with 16, read in two loads, 99 when this took 81).
// Compaction of 2 x 16 heads to 4096 rows: 16 us, bound by its issue slots
// (decoding, extremes) and by the reads that wait for one another.
#include "cache_common.cuh"

namespace elsaa {

namespace {

using namespace cache;
using tc::pack_bf16x2;
using tc::pack_f16x2;
using tc::unpack_f16x2;

constexpr int kWrThreads = 256;

// The threads of a page: E channels each, in 64 / E rows.
template <int D, int E>
struct Page {
    static constexpr int C = D / E;      // threads of a row
    static constexpr int ROWS = 64 / E;  // rows of a thread
    int size;                            // threads of the page
    int t;                               // this one
    int ch, row, step;                   // channels E ch.., rows row + i step
    int index;                           // which of the CTA's pages
    __device__ __forceinline__ explicit Page(int ps) {
        size = ps * D / 64;
        t = threadIdx.x & (size - 1);
        index = threadIdx.x / size;
        ch = t % C;
        row = t / C;
        step = ps / ROWS;
    }
};

// Extremes of neighbouring channels, in the type that the rows come in
// (rounding is monotonous, so the extremes of the codes are the codes of the
// extremes). NaN is left out.
#define ELSAA_EXTREME(NAME, OP)                                       \
    __device__ __forceinline__ uint32_t NAME(uint32_t a, uint32_t b) { \
        uint32_t r;                                                   \
        asm(OP " %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));            \
        return r;                                                     \
    }
ELSAA_EXTREME(bf16x2_max, "max.bf16x2")
ELSAA_EXTREME(bf16x2_min, "min.bf16x2")
ELSAA_EXTREME(f16x2_max, "max.f16x2")
ELSAA_EXTREME(f16x2_min, "min.f16x2")
// of the magnitudes; the sign means nothing
ELSAA_EXTREME(f16x2_abs_max, "max.xorsign.abs.f16x2")
#undef ELSAA_EXTREME

struct Bf16Rows {  // 8 channels, bf16 pairs
    static constexpr int P = 4, PER = 2;  // words, channels a word
    static constexpr uint32_t kNoHigh = 0xff80ff80u, kNoLow = 0x7f807f80u;
    static constexpr uint32_t kAbs = 0x7fff7fffu;
    static __device__ uint32_t max2(uint32_t a, uint32_t b) {
        return bf16x2_max(a, b);
    }
    static __device__ uint32_t min2(uint32_t a, uint32_t b) {
        return bf16x2_min(a, b);
    }
    static __device__ float2 get(uint32_t w) {
        return make_float2(__uint_as_float(w << 16),
                           __uint_as_float(w & 0xffff0000u));
    }
};
struct F16Rows {  // 16 channels, fp16 pairs
    static constexpr int P = 8, PER = 2;
    static constexpr uint32_t kNoHigh = 0xfc00fc00u, kNoLow = 0x7c007c00u;
    static constexpr uint32_t kAbs = 0x7fff7fffu;
    static __device__ uint32_t max2(uint32_t a, uint32_t b) {
        return f16x2_max(a, b);
    }
    static __device__ uint32_t min2(uint32_t a, uint32_t b) {
        return f16x2_min(a, b);
    }
    static __device__ float2 get(uint32_t w) {
        float2 x;
        unpack_f16x2(w, x.x, x.y);
        return x;
    }
};
struct F32Rows {  // 8 channels
    static constexpr int P = 8, PER = 1;
    static constexpr uint32_t kNoHigh = 0xff800000u, kNoLow = 0x7f800000u;
    static constexpr uint32_t kAbs = 0x7fffffffu;
    static __device__ uint32_t max2(uint32_t a, uint32_t b) {
        return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    }
    static __device__ uint32_t min2(uint32_t a, uint32_t b) {
        return __float_as_uint(fminf(__uint_as_float(a), __uint_as_float(b)));
    }
    static __device__ float2 get(uint32_t w) {
        return make_float2(__uint_as_float(w), __uint_as_float(w));
    }
};

// Largest magnitude in the P words of a row (any sign), joined with `m`.
template <typename R>
__device__ __forceinline__ uint32_t abs_max(uint32_t m, const uint32_t *w) {
#pragma unroll
    for (int i = 0; i < R::P; ++i) m = R::max2(m, w[i] & R::kAbs);
    return m;
}

// Largest x of the page's threads. All threads of the CTA.
template <int D, int E>
__device__ __forceinline__ float page_max(const Page<D, E> &g, float x,
                                          float *tmp) {
    // x >= 0: its bits are in the same order
    if (g.size >= 32)
        x = __uint_as_float(
            __reduce_max_sync(0xffffffffu, __float_as_uint(x)));
    else
        for (int o = 1; o < g.size; o <<= 1)
            x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
    if (g.size > 32) {
        if ((threadIdx.x & 31) == 0) tmp[threadIdx.x >> 5] = x;
        __syncthreads();
        const float *at = tmp + g.index * g.size / 32;
#pragma unroll
        for (int w = 0; w < kWrThreads / 32; ++w)
            if (w < g.size / 32) x = fmaxf(x, at[w]);
    }
    return x;
}

// Four bytes of bounds: the extremes' codes (of x f) over 4, rounded outwards,
// joined with the page's older ones times `drop`. sign: 1 for the largest, -1
// for the smallest. Whole numbers in [-112, 112] (448 / 4).
template <typename R>
__device__ __forceinline__ uint32_t bound_word(const uint32_t *x, float sign,
                                               float f, bool had,
                                               uint32_t old, float drop) {
    uint32_t out = 0;
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const float2 a = R::get(x[i / R::PER]);
        const float b = R::PER == 2 ? a.y : R::get(x[(i + 1) / R::PER]).x;
        const float2 c = from_e4m3x2(e4m3x2(a.x * f, b * f));
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float u = ceilf((k ? c.y : c.x) * 0.25f * sign);
            if (had)
                u = fmaxf(u, ceilf((float)(int8_t)(old >> 8 * (i + k)) * drop *
                                   sign));
            out |= ((uint32_t)(int)(u * sign) & 0xffu) << 8 * (i + k);
        }
    }
    return out;
}

// A channel in which the page holds no number may hold anything: its bounds are
// the widest. It has both extremes' first values, -inf for the largest and
// inf for the smallest (one of them may be a key's). `out`: the four bytes as
// bound_word has them, from the extremes `own`; `other`: the other side's.
template <int W>
struct Words {
    uint32_t w[W];
};
template <typename R, int W>
__device__ __noinline__ uint32_t widest(uint32_t out, Words<W> own,
                                        Words<W> other, bool low) {
    const float no = low ? INFINITY : -INFINITY;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 a = R::get(own.w[k / R::PER]);
        const float2 b = R::get(other.w[k / R::PER]);
        const bool y = R::PER == 2 && (k & 1);
        if ((y ? a.y : a.x) == no && (y ? b.y : b.x) == -no)
            out = (out & ~(0xffu << 8 * k)) | (low ? 0x90u : 0x70u) << 8 * k;
    }
    return out;
}
// Whether one of the four bytes is what bound_word makes of such an extreme.
__device__ __forceinline__ bool may_be_none(uint32_t out, bool low) {
    const uint32_t z = out ^ (low ? 0x70707070u : 0x90909090u);
    return ((z - 0x01010101u) & ~z & 0x80808080u) != 0;
}

// The page's channel extremes into its bounds (`bounds`: where the page's
// begin, or NULL: values, or nothing to write). All threads of the CTA; sh:
// [warps][2][D / 4][W] words. The lanes that share channels exchange halves of
// them, so that each ends with four channels; then two warps of the page, one
// for the largest and one for the smallest, join the warps' (one warp for both,
// and whole rows exchanged: a prompt 68 us instead of 65, a step 4.6 instead
// of 4.0, eviction 31 instead of 29.6).
template <typename R, int D, int E>
__device__ __forceinline__ void page_bounds(const Page<D, E> &g, uint32_t *hi,
                                            uint32_t *lo, uint32_t *sh,
                                            int8_t *bounds, float f, bool had,
                                            float drop) {
    constexpr int C = Page<D, E>::C, P = R::P, PARTS = E / 4, W = P / PARTS;
    constexpr int N = D / 4;  // words of bounds
    static_assert(P * R::PER == E && PARTS <= 32 / C && N <= 32, "channels");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // a whole warp without keys has nothing to exchange
    const bool any = __any_sync(0xffffffffu, bounds != nullptr);
    int o = min(g.size, 32) / 2, part = 0;
#pragma unroll
    for (int n = P / 2; n >= W; n /= 2, o /= 2) {
        const bool up = (g.t & o) != 0;
        part = 2 * part + up;
        if (any)
#pragma unroll
            for (int i = 0; i < n; ++i) {
                const uint32_t h = up ? hi[i] : hi[n + i];
                const uint32_t l = up ? lo[i] : lo[n + i];
                hi[i] = R::max2(up ? hi[n + i] : hi[i],
                                __shfl_xor_sync(0xffffffffu, h, o));
                lo[i] = R::min2(up ? lo[n + i] : lo[i],
                                __shfl_xor_sync(0xffffffffu, l, o));
            }
    }
    const bool writes = bounds && (g.t & (2 * o - 1)) < C;
    for (; o >= C; o >>= 1)
        if (any)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                hi[i] = R::max2(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], o));
                lo[i] = R::min2(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], o));
            }
    const int word = g.ch * PARTS + part;
    uint32_t *to = (uint32_t *)bounds;
    if (g.size > 32) {
        uint32_t *at = sh + warp * 2 * N * W;
        if (writes)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                at[word * W + i] = hi[i];
                at[(N + word) * W + i] = lo[i];
            }
        const bool low = g.t >= 32, mine = bounds && g.t < 64 && lane < N;
        to += low * N + lane;
        const uint32_t old = mine && had ? *to : 0u;
        __syncthreads();
        if (!mine) return;
        // the page's first warp
        const uint32_t *from = sh + (warp - low) * 2 * N * W + lane * W;
        auto join = [&](bool l) {
            Words<W> x;
#pragma unroll
            for (int w = 0; w < kWrThreads / 32; ++w)
                if (w < g.size / 32)
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const uint32_t y = from[(w * 2 + l) * N * W + i];
                        x.w[i] = w == 0 ? y
                                 : l    ? R::min2(x.w[i], y)
                                        : R::max2(x.w[i], y);
                    }
            return x;
        };
        const Words<W> x = join(low);
        uint32_t out =
            bound_word<R>(x.w, low ? -1.0f : 1.0f, f, had, old, drop);
        if (!had && may_be_none(out, low))
            out = widest<R, W>(out, x, join(!low), low);
        *to = out;
    } else if (writes) {
        to += word;
        const uint32_t old[2] = {had ? to[0] : 0u, had ? to[N] : 0u};
        uint32_t out[2] = {bound_word<R>(hi, 1.0f, f, had, old[0], drop),
                           bound_word<R>(lo, -1.0f, f, had, old[1], drop)};
        if (!had && may_be_none(out[0], false)) {
            Words<W> h, l;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                h.w[i] = hi[i];
                l.w[i] = lo[i];
            }
            out[0] = widest<R, W>(out[0], h, l, false);
            out[1] = widest<R, W>(out[1], l, h, true);
        }
        to[0] = out[0];
        to[N] = out[1];
    }
}

// 8 neighbouring elements as read, and times f as codes.
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
    using Rows = Bf16Rows;
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) {
        a = *(const uint4 *)p;
    }
    __device__ __forceinline__ const uint32_t *words() const { return &a.x; }
    __device__ __forceinline__ uint2 codes(float f) const {
        // a power of two times a bf16 number is a bf16 number (or far too
        // small for a code)
        const uint32_t ff = pack_bf16x2(f, f);
        uint32_t c[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t y;
            asm("mul.rn.bf16x2 %0, %1, %2;"
                : "=r"(y)
                : "r"(words()[i]), "r"(ff));
            const float2 x = Bf16Rows::get(y);
            c[i] = e4m3x2(x.x, x.y);
        }
        return make_uint2(c[0] | c[1] << 16, c[2] | c[3] << 16);
    }
};
template <>
struct Raw8<float> {
    using Rows = F32Rows;
    uint4 a[2];
    __device__ __forceinline__ void load(const float *p) {
        a[0] = ((const uint4 *)p)[0];
        a[1] = ((const uint4 *)p)[1];
    }
    __device__ __forceinline__ const uint32_t *words() const {
        return &a[0].x;
    }
    __device__ __forceinline__ uint2 codes(float f) const {
        const float *x = (const float *)a;
        return make_uint2(e4m3x4(x[0] * f, x[1] * f, x[2] * f, x[3] * f),
                          e4m3x4(x[4] * f, x[5] * f, x[6] * f, x[7] * f));
    }
};

// blockIdx: (pages of the window, keys and values in turn; head; sequence)
template <typename T, int D>
__global__ void __launch_bounds__(kWrThreads, sizeof(T) == 2 ? 4 : 2)
    k_cache_append(const __grid_constant__ CacheView c,
                   const T *__restrict__ kn, const T *__restrict__ vn) {
    wait_for_stream();
    using G = Page<D, 8>;
    using R = typename Raw8<T>::Rows;
    __shared__ float tmp[kWrThreads / 32];
    __shared__ uint32_t sh[kWrThreads / 32 * G::C * 2 * R::P];
    const G g(c.ps);
    const int h = blockIdx.y, b = blockIdx.z;
    const int q = blockIdx.x * (kWrThreads / g.size) + g.index;
    const bool keys = (q & 1) == 0;
    const auto [end, fresh] = lengths(c, b);
    const int start = end - fresh;
    const int p = max(start, 0) / c.ps + (q >> 1), p0 = p * c.ps;
    // rows [r0, r1) of the page are new, [0, r0) older; they are read while
    // the table entry is on its way
    const int r0 = max(max(start, 0) - p0, 0);
    const int r1 = p0 < end && start < end ? min(c.ps, end - p0) : 0;
    const int entry = r1 > 0 ? c.table[(size_t)b * c.max_pages + p] : -1;
    const T *x = (keys ? kn : vn) + ((size_t)b * c.Hkv + h) * c.T * D +
                 g.ch * 8;
    Raw8<T> raw[G::ROWS];
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i) {
        const int r = g.row + i * g.step;
        if (r >= r0 && r < r1)
            raw[i].load(x + (size_t)(p0 + r - start) * D);
    }
    const int id = r1 > 0 ? checked_page(c, entry, b, p) : -1;
    const bool had = id >= 0 && r0 > 0;
    const size_t ph = (size_t)max(id, 0) * c.Hkv + h;
    uint8_t *codes = (keys ? c.k : c.v) + ph * c.ps * D + g.ch * 8;
    float *scale = (keys ? c.ks : c.vs) + ph;
    const int e_old =
        had ? min(max(scale_exponent(*scale), kCacheExpLow), kCacheExpHigh)
            : kCacheExpLow;
    uint32_t hi[R::P], lo[R::P], top = 0;
#pragma unroll
    for (int j = 0; j < R::P; ++j) {
        hi[j] = R::kNoHigh;
        lo[j] = R::kNoLow;
    }
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i) {
        const int r = g.row + i * g.step;
        if (r >= r0 && r < r1) {
            const uint32_t *w = raw[i].words();
            if (keys) {
#pragma unroll
                for (int j = 0; j < R::P; ++j) {
                    hi[j] = R::max2(hi[j], w[j]);
                    lo[j] = R::min2(lo[j], w[j]);
                }
            } else {
                top = abs_max<R>(top, w);
            }
        }
    }
    if (keys) {
        // a channel without a number holds infinities of the wrong sign
#pragma unroll
        for (int j = 0; j < R::P; ++j)
            top = R::max2(top, R::max2(R::max2(hi[j], 0u),
                                       R::min2(lo[j], 0u) & R::kAbs));
    }
    const float2 t2 = R::get(top);
    int e = page_exponent(page_max(g, magnitude(fmaxf(t2.x, t2.y)), tmp));
    if (had) e = max(e, e_old);
    const float f = pow2(-e);
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i) {
        const int r = g.row + i * g.step;
        if (r >= r0 && r < r1 && id >= 0)
            *(uint2 *)(codes + (size_t)r * D) = raw[i].codes(f);
    }
    // older rows move to the larger exponent; 2^(e_old - e) may be far below
    // the smallest code, whose product is then 0
    const float drop = exp2f((float)(e_old - e));
    if (had && e != e_old) {
        for (int r = g.row; r < r0; r += g.step) {
            uint2 *at = (uint2 *)(codes + (size_t)r * D);
            const uint2 old = *at;
            float y[8];
            from_e4m3x4(old.x, y);
            from_e4m3x4(old.y, y + 4);
            *at = make_uint2(e4m3x4(y[0] * drop, y[1] * drop, y[2] * drop,
                                    y[3] * drop),
                             e4m3x4(y[4] * drop, y[5] * drop, y[6] * drop,
                                    y[7] * drop));
        }
    }
    page_bounds<R>(g, hi, lo, sh,
                   keys && id >= 0 ? c.bounds + ph * 2 * D : nullptr, f, had,
                   drop);
    // every thread of the page has read the scale: a barrier of page_max's lies
    // between, or the page is in one warp
    __syncwarp();
    if (id >= 0 && g.t == 0) *scale = pow2(e);
}

__device__ __forceinline__ uint32_t h2_of_e4m3(uint32_t w) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
    return r;
}
// 2^k as an fp16 pair, 0 below 2^-24.
__device__ __forceinline__ uint32_t pow2_h2(int k) {
    const float x = k < -24 ? 0.0f : pow2(min(k, 15));
    return pack_f16x2(x, x);
}
__device__ __forceinline__ uint32_t mul_h2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// The codes of four fp16 numbers.
__device__ __forceinline__ uint32_t e4m3x4_of(uint32_t a, uint32_t b) {
    uint16_t x, y;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(x) : "r"(a));
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(y) : "r"(b));
    return (uint32_t)x | (uint32_t)y << 16;
}

// Codes times 4, for a factor beyond fp16's 2^15 (448 is 2^-9 2^17 at most).
static __device__ __noinline__ uint4 times_four(uint4 w) {
    const uint32_t f = pow2_h2(2);
    auto four = [=](uint32_t c) {
        return e4m3x4_of(mul_h2(h2_of_e4m3(c), f),
                         mul_h2(h2_of_e4m3(c >> 16), f));
    };
    return make_uint4(four(w.x), four(w.y), four(w.z), four(w.w));
}

__device__ __forceinline__ uint32_t word(const uint4 &w, int m) {
    return m == 0 ? w.x : m == 1 ? w.y : m == 2 ? w.z : w.w;
}

// 16 channels a thread, rows of a page's own exponent copied as they are.
// blockIdx: (pages of the kept rows, keys and values in turn; head; sequence)
template <int D>
__global__ void __launch_bounds__(kWrThreads, 4)
    k_cache_compact(const __grid_constant__ CacheView c, int keep,
                    const int32_t *__restrict__ rows,
                    const int *__restrict__ count,
                    const int32_t *__restrict__ dst_table, int dst_pages,
                    int32_t *__restrict__ lengths_out) {
    wait_for_stream();
    let_next_launch();
    using G = Page<D, 16>;
    using R = F16Rows;
    __shared__ float tmp[kWrThreads / 32];
    __shared__ uint32_t sh[kWrThreads / 32 * G::C * 2 * R::P];
    const G g(c.ps);
    const int h = blockIdx.y, b = blockIdx.z;
    const int q = blockIdx.x * (kWrThreads / g.size) + g.index;
    const bool keys = (q & 1) == 0;
    const int p = q >> 1, p0 = p * c.ps;
    const int32_t *from = rows + ((size_t)b * c.Hkv + h) * keep + p0;
    const uint8_t *pool = keys ? c.k : c.v;
    const float *scales = keys ? c.ks : c.vs;
    // where the rows are, then codes and scales, each read for all of them
    // before one is used
    int src[G::ROWS];
    uint4 raw[G::ROWS];
    int ex[G::ROWS];  // exponents
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i) {
        const int r = g.row + i * g.step;
        src[i] = p0 + r < keep ? from[r] : -1;
    }
    const int n = count[b];
    const int entry =
        p < dst_pages ? dst_table[(size_t)b * dst_pages + p] : -1;
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) lengths_out[b] = n;
    const int held = max(0, min(c.ps, n - p0));
    const int shift = __ffs(c.ps) - 1;
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i) {
        raw[i] = make_uint4(0, 0, 0, 0);
        ex[i] = 0;
        if (g.row + i * g.step < held && src[i] >= 0) {
            // rows of the pool fit in an int: the host's check
            const int sp = (src[i] >> shift) * c.Hkv + h;
            const int at = (sp << shift) + (src[i] & (c.ps - 1));
            raw[i] = *(const uint4 *)(pool + (size_t)at * D + g.ch * 16);
            ex[i] = __float_as_int(scales[sp]);
        }
    }
    const int id = held > 0 ? checked_page(c, entry, b, p) : -1;
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i) {
        // the largest code of the row's 16 times its scale
        uint32_t top = 0;
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const uint32_t w = word(raw[i], m);
            top = f16x2_abs_max(top, h2_of_e4m3(w));
            top = f16x2_abs_max(top, h2_of_e4m3(w >> 16));
        }
        const float2 x = R::get(top & R::kAbs);
        const float sc = __int_as_float(ex[i]);
        amax = fmaxf(amax, magnitude(fmaxf(x.x, x.y) * sc));
        ex[i] = scale_exponent(sc);
    }
    const int e = page_exponent(page_max(g, amax, tmp));
    uint32_t hi[R::P], lo[R::P];
#pragma unroll
    for (int k = 0; k < R::P; ++k) {
        hi[k] = R::kNoHigh;
        lo[k] = R::kNoLow;
    }
    const size_t ph = (size_t)max(id, 0) * c.Hkv + h;
    uint8_t *codes = (keys ? c.k : c.v) + ph * c.ps * D + g.ch * 16;
#pragma unroll
    for (int i = 0; i < G::ROWS; ++i) {
        const int r = g.row + i * g.step;
        if (r < held && id >= 0) {
            // code 2^k in fp16: exact wherever it does not end below half
            // the smallest code
            const int k = ex[i] - e;
            if (k > 15) raw[i] = times_four(raw[i]);
            // the page's own exponent, that of most rows: the codes stay
            uint32_t o[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
            if (keys || k != 0) {
                const uint32_t f = pow2_h2(k > 15 ? k - 2 : k);
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    const uint32_t x = mul_h2(h2_of_e4m3(o[m]), f);
                    const uint32_t y = mul_h2(h2_of_e4m3(o[m] >> 16), f);
                    if (keys) {
                        hi[2 * m] = R::max2(hi[2 * m], x);
                        lo[2 * m] = R::min2(lo[2 * m], x);
                        hi[2 * m + 1] = R::max2(hi[2 * m + 1], y);
                        lo[2 * m + 1] = R::min2(lo[2 * m + 1], y);
                    }
                    if (k != 0) o[m] = e4m3x4_of(x, y);
                }
            }
            *(uint4 *)(codes + (size_t)r * D) =
                make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
    page_bounds<R>(g, hi, lo, sh,
                   keys && id >= 0 ? c.bounds + ph * 2 * D : nullptr, 1.0f,
                   false, 1.0f);
    if (id >= 0 && g.t == 0) (keys ? c.ks : c.vs)[ph] = pow2(e);
}

// CTAs for `pages` pages of keys and of values.
unsigned page_ctas(const CacheView &c, long pages) {
    const int per = kWrThreads / (c.ps * c.d / 64);
    return (unsigned)((2 * pages + per - 1) / per);
}

}  // namespace

cudaError_t launch_cache_append(const CacheView &c, const void *k,
                                const void *v, cudaStream_t st) {
    // T rows touch at most this many pages
    const dim3 grid(page_ctas(c, ((long)c.T + c.ps - 2) / c.ps + 1), c.Hkv,
                    c.B);
    auto go = [&](auto t, auto dd) {
        using T = decltype(t);
        return launch_cache<k_cache_append<T, decltype(dd)::value>>(
            grid, kWrThreads, 0, 0, 1, st, c, (const T *)k, (const T *)v);
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

cudaError_t launch_cache_compact(const CacheView &c, int keep,
                                 const int32_t *rows, const int *count,
                                 const int32_t *dst_table, int dst_pages,
                                 int32_t *lengths_out, cudaStream_t st) {
    const dim3 grid(page_ctas(c, ((long)keep + c.ps - 1) / c.ps), c.Hkv, c.B);
    auto go = [&](auto dd) {
        return launch_cache<k_cache_compact<decltype(dd)::value>>(
            grid, kWrThreads, 0, 0, 1, st, c, keep, rows, count, dst_table,
            dst_pages, lengths_out);
    };
    switch (c.d) {
        case 32: return go(std::integral_constant<int, 32>{});
        case 64: return go(std::integral_constant<int, 64>{});
        default: return go(std::integral_constant<int, 128>{});
    }
}

}  // namespace elsaa
