// From the rows of the Q/K/V projections to heads and back
// (include/elsaa_heads.h): the norm of every query and key head, the rotation
// by position and the change of layout in one pass; kernels and C ABI.
//
// A warp takes one token's heads of one kind (queries, keys or values);
// D / VE lanes of 16 bytes hold a head, so that it works on 32 VE / D heads at
// once, which lie side by side in the row. What belongs to the token alone is
// made once: two pairs' sine and cosine a lane, handed round, and multiplied
// by the norm's weights:
//     out = r (x A + x' B),  A = w cos a,  B = +-w' sin a,
// x' the pair's other channel (of lane +- dim / 2 VE, or next to x), r the
// head's 1 / sqrt(mean x^2 + eps). Memory bound: every row is read once and
// every head written once. B2 H16 N16384 d128 bf16 136 us, 5.9 TB/s, 0.88 of the
// measured copy rate; backward B8 H12 N8192 d64 from fp32 gradients 210 us, 0.79.
#include <stdlib.h>

#include <type_traits>

#include "../../include/elsaa_heads.h"
#include "cache.h"
#include "device_common.cuh"
#include "tc_common.cuh"

using namespace elsaa;

namespace elsaa {
namespace {

constexpr int kHeadWarps = 8;
// CTAs of the backward kernel at most, each of which leaves a partial of dw:
// six of 8 warps for each of the 152 SMs of a GB300. Fixed, so that the
// workspace does not depend on the device.
constexpr int kHeadCtas = 912;

struct RowsView {
    char *p;
    int64_t batch, row, head;  // in bytes
};

struct HeadsArgs {
    int B, H, Hkv, N, G;
    int heads[3];   // of q, k, v that the call handles: H, Hkv, Hkv or 0
    int copies;     // of a K/V head: G with expand
    int norm, grad_fp32;
    // a warp handles a group of heads at a time; the groups of each kind are
    // divided among splits[kind] CTAs of per_split each
    int groups[3], splits[3], per_split;
    float eps;
    RowsView x[3];  // rows (forward), rows of q and k (backward)
    RowsView dx[3];
    char *out[3];   // heads, or their gradients
    const float *w[2];
    const int32_t *positions, *lengths, *new_len;
    float *part;    // [CTAs of queries, then of keys][D]
    int dim;
    uint64_t turns[ELSAA_MAX_PAIRS];
    uint8_t axis[ELSAA_MAX_PAIRS];
};

template <typename T>
struct Vec;  // 16 bytes of T
template <>
struct Vec<float> {
    static constexpr int n = 4;
    static __device__ __forceinline__ void unpack(const uint4 &u, float *x) {
        x[0] = __uint_as_float(u.x);
        x[1] = __uint_as_float(u.y);
        x[2] = __uint_as_float(u.z);
        x[3] = __uint_as_float(u.w);
    }
    static __device__ __forceinline__ uint4 pack(const float *x) {
        return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]),
                          __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int n = 8;
    static __device__ __forceinline__ void unpack(const uint4 &u, float *x) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ uint4 pack(const float *x) {
        return make_uint4(
            tc::pack_bf16x2(x[0], x[1]), tc::pack_bf16x2(x[2], x[3]),
            tc::pack_bf16x2(x[4], x[5]), tc::pack_bf16x2(x[6], x[7]));
    }
};

// What a lane needs of the rotation: the lane that holds its channels' other
// halves (HALVES), and per channel cos a and the signed sine.
template <int VE>
struct Turn {
    int partner;
    bool on;  // the lane has rotated channels
    float c[VE], s[VE];
};

// Sine and cosine of h half turns, h in [-1, 1). For heads of bf16 the
// hardware's, 2^-21.41 and 2^-21.19 off for arguments up to pi, which are off
// themselves by 2^-21.6 (h, pi and their product as fp32): 2^-20.4, where heads
// and rows are rounded to 2^-8. dw, in fp32, is off by that times its terms'
// sizes, as by a dozen roundings, of the many that its sum has. (With sincospif
// the backward pass of B8 H12 N8192 d64 took 5 us more.)
template <typename T>
__device__ __forceinline__ void half_turns(float h, float *s, float *c) {
    if (sizeof(T) == 4) {
        sincospif(h, s, c);
    } else {
        const float x = h * 3.14159265f;
        *s = __sinf(x);
        *c = __cosf(x);
    }
}

// Sines and cosines of the token at (b, n), a pair a lane or two (D = 128),
// handed to the lanes whose channels they turn.
template <typename T, int D, int VE, int LPH, bool IL>
__device__ __forceinline__ void make_turn(const HeadsArgs &a, int b, int n,
                                          int n_new, int lane,
                                          Turn<VE> &t) {
    constexpr int PL = D > 64 ? 2 : 1;
    float c0[PL], s0[PL];
    const int pairs = a.dim >> 1;
    int64_t start = n;
    if (a.lengths) start += (int64_t)a.lengths[b] - n_new;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
        const int p = PL * lane + i;
        c0[i] = 1.0f;
        s0[i] = 0.0f;
        if (p < pairs) {
            int64_t pos = start;
            if (a.positions)
                pos = a.positions[((size_t)a.axis[p] * a.B + b) * a.N + n];
            const uint64_t f = (uint64_t)pos * a.turns[p];
            // the 32 leading bits of the fraction
            const float h = (float)(int32_t)(f >> 32) * 0x1p-31f;
            half_turns<T>(h, &s0[i], &c0[i]);
        }
    }
    const int ch = (lane % LPH) * VE;
    int base;
    float sign = 1.0f;
    t.partner = lane;
    t.on = ch < a.dim;
    if (IL) {
        base = ch >> 1;
    } else {
        const bool lo = ch < pairs;
        base = lo ? ch : ch - pairs;
        sign = lo ? -1.0f : 1.0f;
        if (t.on) t.partner = lo ? lane + pairs / VE : lane - pairs / VE;
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        // the pair of channel ch + e, in lane pair / PL
        const int q = IL ? e >> 1 : e;
        const int src = ((base + q) / PL) & 31;
        const float c = __shfl_sync(~0u, c0[q % PL], src);
        const float s = __shfl_sync(~0u, s0[q % PL], src);
        const bool rot = IL ? ch + e < a.dim : t.on;
        t.c[e] = rot ? c : 1.0f;
        t.s[e] = rot ? (IL ? (e & 1 ? s : -s) : sign * s) : 0.0f;
    }
}

// 1 / sqrt(m), a Newton step behind the approximation
__device__ __forceinline__ float inv_sqrt(float m) {
    const float r = rsqrtf(m);
    if (!(m < INFINITY)) return r;
    return fmaf(0.5f * r, fmaf(-m * r, r, 1.0f), r);
}

template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
    for (int o = LPH / 2; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

__device__ __forceinline__ uint4 shfl4(const uint4 &u, int src) {
    return make_uint4(__shfl_sync(~0u, u.x, src), __shfl_sync(~0u, u.y, src),
                      __shfl_sync(~0u, u.z, src), __shfl_sync(~0u, u.w, src));
}

// blockIdx.y: kind (0 queries, 1 keys, 2 values) and split of its groups.
__device__ __forceinline__ int which_kind(const HeadsArgs &a, int &split) {
    int y = blockIdx.y, kind = 0;
    while (kind < 2 && y >= a.splits[kind]) y -= a.splits[kind++];
    split = y;
    return kind;
}

// Pairs of channels as packed fp32.
template <int VE>
__device__ __forceinline__ float2 two(const float (&x)[VE], int i) {
    return make_float2(x[2 * i], x[2 * i + 1]);
}

// Five CTAs an SM: B2 H16 N16384 d128 bf16 142 us, with four 149, with six and
// two groups a time 146.
template <typename T, int D, bool IL>
__global__ void __launch_bounds__(kHeadWarps * 32, 5)
    k_heads_forward(const __grid_constant__ HeadsArgs a) {
    wait_for_stream();
    using V = Vec<T>;
    constexpr int VE = V::n, LPH = D / VE, HPW = 32 / LPH, U = 4;
    const int lane = threadIdx.x & 31;
    const long row = (long)blockIdx.x * kHeadWarps + (threadIdx.x >> 5);
    if (row >= (long)a.B * a.N) return;
    const int b = (int)(row / a.N), n = (int)(row - (long)b * a.N);
    const int n_new = a.new_len ? min(max(a.new_len[b], 0), a.N) : a.N;
    if (n >= n_new) return;
    int split;
    const int kind = which_kind(a, split);
    const int ch = (lane % LPH) * VE;
    const int heads = a.heads[kind], cp = kind ? a.copies : 1;
    // this lane's head of group g is g HPW + lane / LPH
    const int h0 = split * a.per_split * HPW + lane / LPH;
    const int h1 = min(heads, (split + 1) * a.per_split * HPW);
    const RowsView &X = a.x[kind];
    const int64_t in_step = X.head * HPW;
    const char *in = X.p + b * X.batch + n * X.row + h0 * X.head + ch * sizeof(T);
    const size_t out_head = (size_t)a.N * D * sizeof(T);
    const size_t out_step = out_head * HPW * cp;
    char *out = a.out[kind] +
                ((((size_t)b * heads + h0) * cp * a.N + n) * D + ch) *
                    sizeof(T);

    if (kind == 2) {  // values are copied
        for (int h = h0; h < h1; h += HPW * U) {
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (h + u * HPW < h1)
                    raw[u] = *reinterpret_cast<const uint4 *>(in +
                                                              u * in_step);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (h + u * HPW < h1)
                    for (int i = 0; i < cp; ++i)
                        *reinterpret_cast<uint4 *>(out + u * out_step +
                                                   i * out_head) = raw[u];
            in += U * in_step;
            out += U * out_step;
        }
        return;
    }
    // A = w cos a, B = +-w' sin a
    float A[VE], Bs[VE];
    int partner;
    bool rot;
    {
        Turn<VE> t;
        make_turn<T, D, VE, LPH, IL>(a, b, n, n_new, lane, t);
        float w[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e)
            w[e] = a.norm && a.w[kind] ? a.w[kind][ch + e] : 1.0f;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float wp =
                IL ? w[e ^ 1] : __shfl_sync(~0u, w[e], t.partner);
            A[e] = w[e] * t.c[e];
            Bs[e] = wp * t.s[e];
        }
        partner = t.partner;
        rot = t.on;
    }
    // lanes take part in the shuffles until the warp's last head is done
    const int warp_h = split * a.per_split * HPW;
    for (int g = 0; warp_h + g < h1; g += HPW * U) {
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u] = make_uint4(0, 0, 0, 0);
            if (h0 + g + u * HPW < h1)
                raw[u] = *reinterpret_cast<const uint4 *>(in + u * in_step);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (warp_h + g + u * HPW >= h1) break;
            float x[VE], xp[VE], y[VE];
            V::unpack(raw[u], x);
            float r = 1.0f;
            if (a.norm) {
                float2 ss = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int e = 0; e < VE / 2; ++e)
                    ss = tc::fma2(two(x, e), two(x, e), ss);
                r = inv_sqrt(
                    fmaf(head_sum<LPH>(ss.x + ss.y), 1.0f / D, a.eps));
            }
            if (IL) {
#pragma unroll
                for (int e = 0; e < VE; ++e) xp[e] = x[e ^ 1];
            } else {
                V::unpack(shfl4(raw[u], partner), xp);
            }
            const float2 rr = make_float2(r, r);
#pragma unroll
            for (int e = 0; e < VE / 2; ++e) {
                const float2 z = tc::mul2(two(x, e), two(A, e));
                float2 o = tc::fma2(two(xp, e), two(Bs, e), z);
                // no product with a sine of 0: x' may be infinite
                if (IL ? ch + 2 * e >= a.dim : !rot) o = z;
                o = tc::mul2(o, rr);
                y[2 * e] = o.x;
                y[2 * e + 1] = o.y;
            }
            if (h0 + g + u * HPW < h1) {
                const uint4 y4 = V::pack(y);
                for (int i = 0; i < cp; ++i)
                    *reinterpret_cast<uint4 *>(out + u * out_step +
                                               i * out_head) = y4;
            }
        }
        in += U * in_step;
        out += U * out_step;
    }
}

// VE gradients of one lane, fp32 or T
template <typename T, typename GT>
__device__ __forceinline__ void load_grad(const char *p, float *g) {
    constexpr int VE = Vec<T>::n, n = Vec<GT>::n;
#pragma unroll
    for (int i = 0; i < VE / n; ++i)
        Vec<GT>::unpack(*reinterpret_cast<const uint4 *>(p + 16 * i),
                        g + n * i);
}

// The gradients of copies 1 .. cp - 1, three loads at a time.
template <typename T, typename GT>
__device__ __forceinline__ void add_copies(const char *p, size_t step, int cp,
                                           float (&g)[Vec<T>::n]) {
    constexpr int VE = Vec<T>::n;
    for (int i = 1; i < cp; i += 3) {
        float m[3][VE];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
#pragma unroll
            for (int e = 0; e < VE; ++e) m[k][e] = 0.0f;
            if (i + k < cp) load_grad<T, GT>(p + (i + k) * step, m[k]);
        }
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int e = 0; e < VE; ++e) g[e] += m[k][e];
    }
}

// Groups of heads that a warp of the backward kernel reads at a time, and CTAs
// an SM, by the bytes of a lane's gradients: fp32 ones of bf16 rows (32) fill
// the registers of two CTAs, and three groups in flight serve memory better than
// more warps (B8 H12 N8192 d64 214 us; two groups 251, one group and three CTAs
// 240; half the channels a lane 287; asking for the next groups before working
// on those at hand 219). 16-bit ones do best the other way (padded B2 H16 H_kv4
// N2047 d128, copied heads: 35 us; two groups and two CTAs 42).
template <typename T, typename GT>
constexpr bool kWide = sizeof(GT) * Vec<T>::n > 16;

// The backward pass. A CTA's warps walk the tokens; dw is summed in
// registers, then over the CTA's warps, and leaves as one partial of the CTA
// that k_heads_weights adds up in order.
template <typename T, typename GT, int D, bool IL>
__global__ void __launch_bounds__(kHeadWarps * 32, (kWide<T, GT> ? 2 : 3))
    k_heads_backward(const __grid_constant__ HeadsArgs a) {
    wait_for_stream();
    using V = Vec<T>;
    constexpr int VE = V::n, LPH = D / VE, HPW = 32 / LPH, U = kWide<T, GT> ? 3 : 1;
    __shared__ float sums[kHeadWarps][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int ch = (lane % LPH) * VE;
    const long rows = (long)a.B * a.N;
    int split;
    const int kind = which_kind(a, split);
    const int heads = a.heads[kind], cp = kind ? a.copies : 1;
    const int warp_h = split * a.per_split * HPW, h0 = warp_h + lane / LPH;
    const int h1 = min(heads, (split + 1) * a.per_split * HPW);
    const bool norm = a.norm && kind < 2;
    const RowsView &X = a.x[norm ? kind : 0], &Y = a.dx[kind];
    const size_t g_head = (size_t)a.N * D * sizeof(GT);
    const size_t g_step = g_head * HPW * cp;
    float w[VE], dw[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        w[e] = norm && a.w[kind] ? a.w[kind][ch + e] : 1.0f;
        dw[e] = 0.0f;
    }
    for (long row = (long)blockIdx.x * kHeadWarps + warp; row < rows;
         row += (long)gridDim.x * kHeadWarps) {
        const int b = (int)(row / a.N), n = (int)(row - (long)b * a.N);
        const int n_new = a.new_len ? min(max(a.new_len[b], 0), a.N) : a.N;
        if (n >= n_new) continue;
        Turn<VE> t;
        if (kind < 2) make_turn<T, D, VE, LPH, IL>(a, b, n, n_new, lane, t);
        const char *gp = a.out[kind] +
                         ((((size_t)b * heads + h0) * cp * a.N + n) * D + ch) *
                             sizeof(GT);
        const char *xp = X.p + b * X.batch + n * X.row + h0 * X.head +
                         ch * sizeof(T);
        char *yp = Y.p + b * Y.batch + n * Y.row + h0 * Y.head +
                   ch * sizeof(T);
        for (int g = 0; warp_h + g < h1; g += HPW * U) {
            float gr[U][VE];
            uint4 raw[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                raw[u] = make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < VE; ++e) gr[u][e] = 0.0f;
                if (h0 + g + u * HPW < h1) {
                    load_grad<T, GT>(gp + u * g_step, gr[u]);
                    if (norm)
                        raw[u] = *reinterpret_cast<const uint4 *>(
                            xp + u * X.head * HPW);
                }
            }
            if (cp > 1) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (h0 + g + u * HPW < h1)
                        add_copies<T, GT>(gp + u * g_step, g_head, cp, gr[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (warp_h + g + u * HPW >= h1) break;
                if (kind < 2) {
                    float uu[VE];
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        const float p =
                            IL ? gr[u][e ^ 1]
                               : __shfl_sync(~0u, gr[u][e], t.partner);
                        const bool rot = IL ? ch + e < a.dim : t.on;
                        const float z = gr[u][e] * t.c[e];
                        uu[e] = rot ? fmaf(-p, t.s[e], z) : z;
                    }
                    if (norm) {
                        float x[VE];
                        float2 s2 = make_float2(0.0f, 0.0f), t2 = s2;
                        V::unpack(raw[u], x);
#pragma unroll
                        for (int e = 0; e < VE / 2; ++e) {
                            s2 = tc::fma2(two(x, e), two(x, e), s2);
                            t2 = tc::fma2(tc::mul2(two(uu, e), two(w, e)),
                                          two(x, e), t2);
                        }
                        const float ss = head_sum<LPH>(s2.x + s2.y);
                        const float tx = head_sum<LPH>(t2.x + t2.y);
                        const float r = inv_sqrt(fmaf(ss, 1.0f / D, a.eps));
                        // of xh = x r: mean(t xh) = r mean(t x)
                        const float m = tx * (1.0f / D) * r;
#pragma unroll
                        for (int e = 0; e < VE; ++e) {
                            const float xh = x[e] * r;
                            dw[e] = fmaf(uu[e], xh, dw[e]);
                            uu[e] = r * fmaf(-xh, m, uu[e] * w[e]);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < VE; ++e) gr[u][e] = uu[e];
                }
                if (h0 + g + u * HPW < h1)
                    *reinterpret_cast<uint4 *>(yp + u * Y.head * HPW) =
                        V::pack(gr[u]);
            }
            gp += U * g_step;
            xp += U * X.head * HPW;
            yp += U * Y.head * HPW;
        }
    }
    if (!a.part || kind == 2) return;
#pragma unroll
    for (int e = 0; e < VE; ++e) {
        float v = dw[e];
#pragma unroll
        for (int o = LPH; o < 32; o <<= 1) v += __shfl_xor_sync(~0u, v, o);
        if (lane < LPH) sums[warp][ch + e] = v;
    }
    __syncthreads();
    const long cta =
        (long)((kind ? a.splits[0] : 0) + split) * gridDim.x + blockIdx.x;
    for (int i = threadIdx.x; i < D; i += kHeadWarps * 32) {
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < kHeadWarps; ++q) v += sums[q][i];
        a.part[cta * D + i] = v;
    }
}

// dw: 32 columns of the partials a CTA, 32 rows of threads, in one order.
__global__ void __launch_bounds__(1024)
    k_heads_weights(const float *__restrict__ part, int ctas_q, int ctas_k,
                    int d, float *__restrict__ dw_q,
                    float *__restrict__ dw_k) {
    wait_for_stream();
    __shared__ float s[32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const bool keys = (int)blockIdx.x * 32 >= d;
    const int col = blockIdx.x * 32 + x - (keys ? d : 0);
    const int first = keys ? ctas_q : 0, last = first + (keys ? ctas_k : ctas_q);
    float v = 0.0f;
    for (int c = first + y; c < last; c += 32) v += part[(size_t)c * d + col];
    s[y][x] = v;
    __syncthreads();
    if (y > 0) return;
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v += s[i][x];
    float *o = keys ? dw_k : dw_q;
    if (o) o[col] = v;
}

int bad(const char *m) {
    return set_last_error(ELSAA_ERR_INVALID_ARG, "%s", m);
}
int no(const char *m) {
    return set_last_error(ELSAA_ERR_UNSUPPORTED, "%s", m);
}
bool misaligned(const void *p, size_t a) { return (uintptr_t)p % a != 0; }

int check_heads(const elsaa_heads *p) {
    if (!p) return bad("heads is NULL");
    if (p->B <= 0 || p->H <= 0 || p->H_kv <= 0 || p->N <= 0)
        return bad("B, H, H_kv and N must be positive");
    if (p->H % p->H_kv != 0) return bad("H must be a multiple of H_kv");
    if (p->dtype != ELSAA_BF16 && p->dtype != ELSAA_FP32)
        return bad("dtype must be ELSAA_BF16 or ELSAA_FP32");
    for (int f : {p->norm, p->expand, p->grad_fp32})
        if (f != 0 && f != 1) return bad("norm, expand and grad_fp32 must be "
                                         "0 or 1");
    if (p->norm && !(p->eps > 0.0f && isfinite(p->eps)))
        return bad("eps must be finite and > 0");
    if (p->d_h != 32 && p->d_h != 64 && p->d_h != 128)
        return no("d_h must be 32, 64 or 128");
    if (p->H > 65535) return no("H must be at most 65535");
    if ((long)p->B * p->N > 1L << 30) return no("B * N must be at most 2^30");
    const elsaa_rotary &r = p->rotary;
    if (r.interleaved != 0 && r.interleaved != 1)
        return bad("rotary.interleaved must be 0 or 1");
    if (r.dim < 0 || r.dim > p->d_h)
        return bad("rotary.dim must be in [0, d_h]");
    if (r.dim % (r.interleaved ? 2 : 16) != 0)
        return no("rotary.dim must be a multiple of 16, or of 2 when "
                  "interleaved");
    if (r.axes < 1 || r.axes > ELSAA_MAX_AXES)
        return bad("rotary.axes must be 1 to 4");
    for (int i = 0; i < r.dim / 2; ++i)
        if (r.axis[i] >= r.axes)
            return bad("rotary.axis entries must be below rotary.axes");
    return ELSAA_OK;
}

// The view of one tensor of rows; `write`: no two rows share an element.
int check_rows(const elsaa_rows *r, const elsaa_heads *p, int heads,
               bool write, RowsView *v) {
    if (!r->data) return bad("rows without data");
    if (misaligned(r->data, 16)) return bad("rows must be 16-byte aligned");
    const int64_t el = p->dtype == ELSAA_FP32 ? 4 : 2;
    const int64_t size[3] = {p->B, p->N, heads};
    int64_t st[3] = {r->batch, r->row, r->head};
    for (int i = 0; i < 3; ++i) {
        if (size[i] == 1) st[i] = 0;
        if (st[i] > (1L << 50) || st[i] < -(1L << 50))
            return bad("strides of rows must be below 2^50");
        if (st[i] * el % 16 != 0)
            return bad("strides of rows must be multiples of 16 bytes");
    }
    if (write) {
        // from the smallest stride up, each steps over what is below it
        int64_t below = p->d_h;
        bool used[3] = {};
        for (int k = 0; k < 3; ++k) {
            int m = -1;
            for (int i = 0; i < 3; ++i)
                if (!used[i] && (m < 0 || llabs(st[i]) < llabs(st[m]))) m = i;
            used[m] = true;
            if (size[m] == 1) continue;
            if (llabs(st[m]) < below)
                return bad("rows that are written must not overlap");
            below += (size[m] - 1) * llabs(st[m]);
        }
    }
    *v = RowsView{(char *)r->data, st[0] * el, st[1] * el, st[2] * el};
    return ELSAA_OK;
}

int check_tokens(const elsaa_heads *p, const float *w_q, const float *w_k,
                 const int32_t *positions, const int32_t *lengths) {
    if (!p->norm && (w_q || w_k)) return bad("w_q and w_k need norm = 1");
    if (positions && lengths)
        return bad("positions and lengths exclude one another");
    return ELSAA_OK;
}

void fill(const elsaa_heads *p, HeadsArgs *a) {
    a->B = p->B;
    a->H = p->H;
    a->Hkv = p->H_kv;
    a->N = p->N;
    a->G = p->H / p->H_kv;
    a->copies = p->expand ? a->G : 1;
    a->norm = p->norm;
    a->grad_fp32 = p->grad_fp32;
    a->eps = p->eps;
    a->dim = p->rotary.dim;
    for (int i = 0; i < ELSAA_MAX_PAIRS; ++i) {
        a->turns[i] = p->rotary.turns[i];
        a->axis[i] = p->rotary.axis[i];
    }
}

// Groups of heads of a CTA: those of one K/V set, four at least (the token's
// sines are made for each), fewer where the tokens alone do not give every
// SM's warps work. Returns the CTAs of a token, at most `most`.
int divide_groups(HeadsArgs *a, int d, int el, long tokens, int most) {
    const int per_warp = 32 / (d * el / 16);
    int all = 0, least = 0;
    for (int i = 0; i < 3; ++i) {
        a->groups[i] = (a->heads[i] + per_warp - 1) / per_warp;
        all += a->groups[i];
        if (a->groups[i] && (!least || a->groups[i] < least))
            least = a->groups[i];
    }
    const long units = 152 * 16;
    long per = tokens * all / units;
    if (per > least) per = least > 4 ? least : (per < 4 ? per : 4);
    if (per < 1) per = 1;
    for (;; per *= 2) {
        int n = 0;
        for (int i = 0; i < 3; ++i) {
            a->splits[i] = (int)((a->groups[i] + per - 1) / per);
            n += a->splits[i];
        }
        a->per_split = (int)per;
        if (n <= most) return n;
    }
}

int bwd_ctas(long tokens, int splits) {
    long x = (tokens + kHeadWarps - 1) / kHeadWarps;
    long most = kHeadCtas / splits;
    if (most < 1) most = 1;
    return (int)(x < most ? x : most);
}

template <typename F>
cudaError_t timed(const char *name, cudaStream_t st, F fn) {
    return timed_launch(
        name, st, [](void *f) { return (*(F *)f)(); }, &fn);
}

template <typename T, int D>
cudaError_t launch_fwd(const HeadsArgs &a, bool il, dim3 grid,
                       cudaStream_t st) {
    auto go = [&](auto kern) {
        return launch_after(kern, grid, kHeadWarps * 32, 0, st, a);
    };
    return il ? go(k_heads_forward<T, D, true>)
              : go(k_heads_forward<T, D, false>);
}
template <typename T, typename GT, int D>
cudaError_t launch_bwd(const HeadsArgs &a, bool il, dim3 grid,
                       cudaStream_t st) {
    auto go = [&](auto kern) {
        return launch_after(kern, grid, kHeadWarps * 32, 0, st, a);
    };
    return il ? go(k_heads_backward<T, GT, D, true>)
              : go(k_heads_backward<T, GT, D, false>);
}

}  // namespace
}  // namespace elsaa

extern "C" int elsaa_heads_workspace_size(const elsaa_heads *heads,
                                          size_t *bytes) {
    clear_last_error();
    if (!bytes) return bad("bytes is NULL");
    const int rc = check_heads(heads);
    if (rc != ELSAA_OK) return rc;
    *bytes = sizeof(float) * heads->d_h * kHeadCtas;
    return ELSAA_OK;
}

extern "C" int elsaa_heads_forward(
    const elsaa_heads *heads, const elsaa_rows *q, const elsaa_rows *k,
    const elsaa_rows *v, const float *w_q, const float *w_k,
    const int32_t *positions, const int32_t *lengths, const int32_t *new_len,
    void *q_out, void *k_out, void *v_out, void *stream) {
    clear_last_error();
    int rc = check_heads(heads);
    if (rc == ELSAA_OK) rc = check_tokens(heads, w_q, w_k, positions, lengths);
    if (rc != ELSAA_OK) return rc;
    HeadsArgs a = {};
    fill(heads, &a);
    const elsaa_rows *rows[3] = {q, k, v};
    void *out[3] = {q_out, k_out, v_out};
    for (int i = 0; i < 3; ++i) {
        if (!rows[i] != !out[i])
            return bad("rows and heads of q, k and v go together");
        if (!rows[i]) continue;
        if (misaligned(out[i], 16))
            return bad("q_out, k_out and v_out must be 16-byte aligned");
        a.heads[i] = i ? a.Hkv : a.H;
        a.out[i] = (char *)out[i];
        rc = check_rows(rows[i], heads, a.heads[i], false, &a.x[i]);
        if (rc != ELSAA_OK) return rc;
    }
    if (!q && !k && !v) return bad("one of q, k and v must be given");
    a.w[0] = w_q;
    a.w[1] = w_k;
    a.positions = positions;
    a.lengths = lengths;
    a.new_len = new_len;
    const bool f32 = heads->dtype == ELSAA_FP32;
    const long tokens = (long)a.B * a.N;
    const int splits =
        divide_groups(&a, heads->d_h, f32 ? 4 : 2, tokens, 65535);
    const dim3 grid((unsigned)((tokens + kHeadWarps - 1) / kHeadWarps),
                    splits);
    const bool il = heads->rotary.interleaved != 0;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = timed("heads_forward", st, [&] {
        switch (heads->d_h) {
            case 32:
                return f32 ? launch_fwd<float, 32>(a, il, grid, st)
                           : launch_fwd<__nv_bfloat16, 32>(a, il, grid, st);
            case 64:
                return f32 ? launch_fwd<float, 64>(a, il, grid, st)
                           : launch_fwd<__nv_bfloat16, 64>(a, il, grid, st);
            default:
                return f32 ? launch_fwd<float, 128>(a, il, grid, st)
                           : launch_fwd<__nv_bfloat16, 128>(a, il, grid, st);
        }
    });
    if (e != cudaSuccess)
        return set_last_error(ELSAA_ERR_CUDA, "heads_forward: %s",
                              cudaGetErrorString(e));
    return ELSAA_OK;
}

extern "C" int elsaa_heads_backward(
    const elsaa_heads *heads, const void *dq, const void *dk, const void *dv,
    const elsaa_rows *q, const elsaa_rows *k, const float *w_q,
    const float *w_k, const int32_t *positions, const int32_t *lengths,
    const int32_t *new_len, const elsaa_rows *dq_rows,
    const elsaa_rows *dk_rows, const elsaa_rows *dv_rows, float *dw_q,
    float *dw_k, void *workspace, size_t workspace_bytes, void *stream) {
    clear_last_error();
    int rc = check_heads(heads);
    if (rc == ELSAA_OK) rc = check_tokens(heads, w_q, w_k, positions, lengths);
    if (rc != ELSAA_OK) return rc;
    HeadsArgs a = {};
    fill(heads, &a);
    const void *grad[3] = {dq, dk, dv};
    const elsaa_rows *x[3] = {q, k, nullptr};
    const elsaa_rows *dx[3] = {dq_rows, dk_rows, dv_rows};
    float *dw[2] = {dw_q, dw_k};
    for (int i = 0; i < 3; ++i) {
        if (!grad[i] != !dx[i])
            return bad("gradients of heads and of rows of q, k and v go "
                       "together");
        if (i < 2 && dw[i] && (!heads->norm || !grad[i]))
            return bad("dw_q and dw_k need norm = 1 and their heads' "
                       "gradients");
        if (!grad[i]) continue;
        if (misaligned(grad[i], 16))
            return bad("dq, dk and dv must be 16-byte aligned");
        a.heads[i] = i ? a.Hkv : a.H;
        a.out[i] = (char *)grad[i];
        rc = check_rows(dx[i], heads, a.heads[i], true, &a.dx[i]);
        if (rc == ELSAA_OK && i < 2 && heads->norm) {
            if (!x[i]) return bad("the backward pass of the norm needs the "
                                  "rows");
            rc = check_rows(x[i], heads, a.heads[i], false, &a.x[i]);
        }
        if (rc != ELSAA_OK) return rc;
    }
    if (!dq && !dk && !dv) return bad("one of dq, dk and dv must be given");
    const int d = heads->d_h;
    const bool sums = dw_q || dw_k;
    if (sums) {
        if (!workspace)
            return set_last_error(ELSAA_ERR_WORKSPACE, "workspace is NULL");
        if (misaligned(workspace, 256))
            return set_last_error(ELSAA_ERR_WORKSPACE,
                                  "workspace must be 256-byte aligned");
        const size_t need = sizeof(float) * d * kHeadCtas;
        if (workspace_bytes < need)
            return set_last_error(ELSAA_ERR_WORKSPACE,
                                  "workspace too small: %zu bytes given, %zu "
                                  "needed",
                                  workspace_bytes, need);
        a.part = (float *)workspace;
    }
    a.w[0] = w_q;
    a.w[1] = w_k;
    a.positions = positions;
    a.lengths = lengths;
    a.new_len = new_len;
    const bool f32 = heads->dtype == ELSAA_FP32;
    const bool g32 = f32 || heads->grad_fp32;
    const long tokens = (long)a.B * a.N;
    const int splits =
        divide_groups(&a, d, f32 ? 4 : 2, tokens, kHeadCtas);
    const dim3 grid(bwd_ctas(tokens, splits), splits);
    const bool il = heads->rotary.interleaved != 0;
    cudaStream_t st = (cudaStream_t)stream;
    using bf = __nv_bfloat16;
    auto run = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        if (f32) return launch_bwd<float, float, D>(a, il, grid, st);
        return g32 ? launch_bwd<bf, float, D>(a, il, grid, st)
                   : launch_bwd<bf, bf, D>(a, il, grid, st);
    };
    cudaError_t e = timed("heads_backward", st, [&] {
        return d == 32   ? run(std::integral_constant<int, 32>{})
               : d == 64 ? run(std::integral_constant<int, 64>{})
                         : run(std::integral_constant<int, 128>{});
    });
    if (e == cudaSuccess && sums)
        e = timed("heads_weights", st, [&] {
            return launch_after(k_heads_weights, dim3(2 * d / 32), 1024, 0,
                                st, (const float *)a.part,
                                (int)grid.x * a.splits[0],
                                (int)grid.x * a.splits[1], d, dw_q, dw_k);
        });
    if (e != cudaSuccess)
        return set_last_error(ELSAA_ERR_CUDA, "heads_backward: %s",
                              cudaGetErrorString(e));
    return ELSAA_OK;
}
