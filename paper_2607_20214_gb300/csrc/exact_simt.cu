// Exact attention on the CUDA cores, in fp32 (include/elsaa_exact.h): fp32
// tensors, and bf16 ones with impl = SIMT. One pass over the keys with the
// running maximum and sum of the softmax; the backward pass as two kernels of
// one shape, one with query rows held and keys passing (dQ), one with keys
// held and query rows passing (dK, dV), so that every sum has one order.
//
// A CTA of 128 threads holds kHeld rows and walks tiles of kPass rows, all
// operands in shared memory as fp32. Thread (y, x) of 8 x 16 computes the
// scores of rows 4 y .. 4 y + 3 with x, x + 16, x + 32, x + 48, and of the sums
// the same rows with d / 16 channels. Every four channels cost 8 16-byte reads
// from shared memory for 64 multiply-adds (32 packed ones). Shared memory's
// wavefronts run at 64 % of their peak, the multiply-adds at 46 %: B8 H8 N1000
// d64 fp32 464 us forward, 35 TFLOP/s of 74; its backward pass 1559, 26. (8 rows a
// thread, or warps of 4 x 8, save wavefronts and were no faster.) With few
// tiles of held rows the walks are divided into chunks, and k_exact_join and
// k_exact_add add up, in order, what these leave.
#include <type_traits>

#include "device_common.cuh"
#include "exact.h"
#include "tc_common.cuh"

namespace elsaa {
namespace {

constexpr int kHeld = 32, kPass = 64, kThreads = 128;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <typename T>
__device__ __forceinline__ float4 load4(const T *p);
template <>
__device__ __forceinline__ float4 load4<float>(const float *p) {
    return *reinterpret_cast<const float4 *>(p);
}
template <>
__device__ __forceinline__ float4
load4<__nv_bfloat16>(const __nv_bfloat16 *p) {
    const uint2 u = *reinterpret_cast<const uint2 *>(p);
    return make_float4(__uint_as_float(u.x << 16),
                       __uint_as_float(u.x & 0xffff0000u),
                       __uint_as_float(u.y << 16),
                       __uint_as_float(u.y & 0xffff0000u));
}

// Rows [0, n) of `src` into `rows` rows of shared memory, `pitch` floats
// apart, zeros behind them. ok(i): row i has data.
template <typename T, int D, typename F>
__device__ __forceinline__ void load_rows(float *dst, int pitch,
                                          const T *src, int rows, F ok) {
    for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (ok(r)) x = load4(src + (size_t)r * D + c);
        *reinterpret_cast<float4 *>(dst + r * pitch + c) = x;
    }
}

// s[a][e] = <held row 4 y + a, passing row x + 16 e>
template <int D>
__device__ __forceinline__ void scores(const float *held, const float *pass,
                                       int y, int x, float (&s)[4][4]) {
    using tc::fma2;
    float2 acc[4][4];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[a][e] = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
        float4 h[4], p[4];
#pragma unroll
        for (int a = 0; a < 4; ++a)
            h[a] = *reinterpret_cast<const float4 *>(held +
                                                     (4 * y + a) * D + c);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            p[e] = *reinterpret_cast<const float4 *>(
                pass + (x + 16 * e) * (D + 4) + c);
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                acc[a][e] = fma2(make_float2(h[a].x, h[a].y),
                                 make_float2(p[e].x, p[e].y), acc[a][e]);
                acc[a][e] = fma2(make_float2(h[a].z, h[a].w),
                                 make_float2(p[e].z, p[e].w), acc[a][e]);
            }
    }
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[a][e] = acc[a][e].x + acc[a][e].y;
}

// Channels of thread x: pairs 2 x + 32 c, 2 x + 32 c + 1 (D = 32: one pair).
// acc[a][c] += sum over the passing rows of w[4 y + a][row] pass[row].
template <int D>
__device__ __forceinline__ void weighted(const float *w, const float *pass,
                                         int y, int x,
                                         float2 (&acc)[4][D / 32]) {
    using tc::fma2;
#pragma unroll 2
    for (int j = 0; j < kPass; j += 4) {
        float4 p[4];
#pragma unroll
        for (int a = 0; a < 4; ++a)
            p[a] = *reinterpret_cast<const float4 *>(w + (4 * y + a) * kPass +
                                                     j);
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                const float2 v = *reinterpret_cast<const float2 *>(
                    pass + (j + q) * (D + 4) + 2 * x + 32 * c);
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    const float f = q == 0   ? p[a].x
                                    : q == 1 ? p[a].y
                                    : q == 2 ? p[a].z
                                             : p[a].w;
                    acc[a][c] = fma2(make_float2(f, f), v, acc[a][c]);
                }
            }
    }
}

template <typename T>
__device__ __forceinline__ void store2(T *p, float2 v);
template <>
__device__ __forceinline__ void store2<float>(float *p, float2 v) {
    *reinterpret_cast<float2 *>(p) = v;
}
template <>
__device__ __forceinline__ void store2<__nv_bfloat16>(__nv_bfloat16 *p,
                                                      float2 v) {
    *reinterpret_cast<uint32_t *>(p) = tc::pack_bf16x2(v.x, v.y);
}

// over the 16 lanes of a row
__device__ __forceinline__ float row_max(float v) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
        v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

// How walks are divided: `splits` chunks at most, of `chunk` keys, or (dK, dV) of
// `chunk` passing rows over all heads. What a chunk leaves of held row r (over
// all heads): the sums in o[part][r][D], of the forward pass those of e^(z - m) v
// with (m, sum of e^(z - m)) in ml[part][r], z and m base 2; of dK and dV
// [part][r][2][D].
struct Split {
    int splits, chunk;
    size_t rows;
    float *o;
    float2 *ml;
};

// Tile `t` (the last ones first: they see most) of K/V head `kvh`, b-major.
struct Item {
    int b, kvh, tile, part;
    __device__ Item(const ExactView &a, int tiles, int splits = 1) {
        const int heads = a.B * a.Hkv;
        const int h = blockIdx.x % heads, t = (int)(blockIdx.x / heads);
        tile = tiles - 1 - t / splits;
        part = t % splits;
        b = h / a.Hkv;
        kvh = h % a.Hkv;
    }
};

template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
    k_exact_fwd(const __grid_constant__ ExactView a,
                const __grid_constant__ Split split, int tiles) {
    wait_for_stream();
    extern __shared__ __align__(16) float sm[];
    float *sQ = sm, *sK = sQ + kHeld * D, *sV = sK + kPass * (D + 4);
    float *sP = sV + kPass * (D + 4);
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
    if (blockIdx.x == 0 && threadIdx.x < 4) (&a.status->code)[threadIdx.x] = 0;
    const Item it(a, tiles, split.splits);
    const ExactSeq seq(a, it.b);
    const int rows = a.G * a.Nq, r0 = it.tile * kHeld;
    const int r1 = min(r0 + kHeld, rows);
    const size_t head0 = (size_t)it.b * a.H + (size_t)it.kvh * a.G;
    const T *q = (const T *)a.q + (head0 * a.Nq + r0) * D;
    const size_t kv = ((size_t)it.b * a.Hkv + it.kvh) * a.Nk;
    const int all = exact_most(seq, r0, r1, a.Nq);
    const int first = it.part * split.chunk;
    if (it.part > 0 && first >= all) return;
    const int most = min(all, first + split.chunk);
    load_rows<T, D>(sQ, D, q, kHeld, [&](int r) {
        return r0 + r < r1 && (r0 + r) % a.Nq < seq.ql;
    });
    int seen[4];
    float m[4], l[4];
    float2 acc[4][D / 32];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 4 * y + i;
        seen[i] = r < r1 ? seq.seen(r % a.Nq) : 0;
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) acc[i][c] = make_float2(0.f, 0.f);
    }
    const float sl2 = a.scale * kLog2e;
    for (int j0 = first; j0 < most; j0 += kPass) {
        __syncthreads();
        auto have = [&](int r) { return j0 + r < most; };
        load_rows<T, D>(sK, D + 4, (const T *)a.k + (kv + j0) * D, kPass, have);
        load_rows<T, D>(sV, D + 4, (const T *)a.v + (kv + j0) * D, kPass, have);
        __syncthreads();
        float s[4][4];
        scores<D>(sQ, sK, y, x, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float z = -INFINITY;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // (rounded before the maximum, itself one of them, is
                // subtracted: large scores' weights stay below 1)
                s[i][e] = j0 + x + 16 * e < seen[i] ? __fmul_rn(s[i][e], sl2)
                                                    : -INFINITY;
                z = fmaxf(z, s[i][e]);
            }
            z = fmaxf(row_max(z), m[i]);
            const float ref = z == -INFINITY ? 0.f : z;
            const float f = exp2f(m[i] - ref);
            m[i] = z;
            float t = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = exp2f(s[i][e] - ref);
                t += p;
                sP[(4 * y + i) * kPass + x + 16 * e] = p;
            }
            l[i] = fmaf(l[i], f, row_sum(t));
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
                acc[i][c] = tc::mul2(acc[i][c], make_float2(f, f));
        }
        __syncwarp();  // a warp reads the rows that it wrote
        weighted<D>(sP, sV, y, x, acc);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 4 * y + i;
        if (r >= r1 || r % a.Nq >= seq.ql) continue;
        if (all > split.chunk) {
            const size_t to = it.part * split.rows + head0 * a.Nq + r;
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
                store2(split.o + to * D + 2 * x + 32 * c, acc[i][c]);
            if (x == 0) split.ml[to] = make_float2(m[i], l[i]);
            continue;
        }
        const float inv = l[i] > 0.f ? 1.0f / l[i] : l[i] == 0.f ? 0.f : l[i];
        T *o = (T *)a.out + (head0 * a.Nq + r) * D + 2 * x;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
            store2(o + 32 * c, tc::mul2(acc[i][c], make_float2(inv, inv)));
        if (a.lse && x == 0)
            a.lse[head0 * a.Nq + r] =
                l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * kLn2;
    }
}

// Joins the chunks of the rows that have more than one: D / 4 lanes a row.
template <typename T, int D>
__global__ void __launch_bounds__(256)
    k_exact_join(const __grid_constant__ ExactView a,
                 const __grid_constant__ Split split) {
    wait_for_stream();
    constexpr int L = D / 4;
    const size_t row = ((size_t)blockIdx.x * 256 + threadIdx.x) / L;
    const int c = threadIdx.x % L * 4;
    if (row >= split.rows) return;
    const int group = a.G * a.Nq, r = (int)(row % group);
    const ExactSeq seq(a, (int)(row / group) / a.Hkv);
    if (r % a.Nq >= seq.ql) return;
    const int r0 = r / kHeld * kHeld;
    const int all = exact_most(seq, r0, min(r0 + kHeld, group), a.Nq);
    if (all <= split.chunk) return;
    const int parts = (all + split.chunk - 1) / split.chunk;
    float m = -INFINITY;
    for (int p = 0; p < parts; ++p)
        m = fmaxf(m, split.ml[p * split.rows + row].x);
    const float ref = m == -INFINITY ? 0.f : m;
    float l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = 0; p < parts; ++p) {
        const float2 ml = split.ml[p * split.rows + row];
        const float f = exp2f(ml.x - ref);
        const float4 v = *reinterpret_cast<const float4 *>(
            split.o + (p * split.rows + row) * D + c);
        l = fmaf(ml.y, f, l);
        o.x = fmaf(v.x, f, o.x);
        o.y = fmaf(v.y, f, o.y);
        o.z = fmaf(v.z, f, o.z);
        o.w = fmaf(v.w, f, o.w);
    }
    const float inv = l > 0.f ? 1.0f / l : l == 0.f ? 0.f : l;
    T *to = (T *)a.out + row * D + c;
    store2(to, make_float2(o.x * inv, o.y * inv));
    store2(to + 2, make_float2(o.z * inv, o.w * inv));
    if (a.lse && c == 0)
        a.lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// KEYS = 0: query rows held; dQ, and D_i = <dO_i, O_i> for the other kernel.
// KEYS = 1: key rows held; dK, dV.
template <typename T, int D, bool KEYS>
__global__ void __launch_bounds__(kThreads)
    k_exact_bwd(const __grid_constant__ ExactView a,
                const __grid_constant__ Split split, int tiles) {
    wait_for_stream();
    extern __shared__ __align__(16) float sm[];
    // held: Q, dO or K, V; passing: K, V or Q, dO
    float *sA = sm, *sB = sA + kHeld * D;
    float *sC = sB + kHeld * D, *sE = sC + kPass * (D + 4);
    float *sW = sE + kPass * (D + 4);  // [held][passing] dS
    float *sP = sW + kHeld * kPass;    // KEYS: P
    float *sL = sP + (KEYS ? kHeld * kPass : 0), *sD = sL + kPass;
    int *sN = (int *)(sD + kPass);
    const int x = threadIdx.x & 15, y = threadIdx.x >> 4;
    if (!KEYS && blockIdx.x == 0 && threadIdx.x < 4)
        (&a.status->code)[threadIdx.x] = 0;
    const Item it(a, tiles, split.splits);
    const ExactSeq seq(a, it.b);
    const size_t head0 = (size_t)it.b * a.H + (size_t)it.kvh * a.G;
    const size_t qrow = head0 * a.Nq;
    const size_t kv = ((size_t)it.b * a.Hkv + it.kvh) * a.Nk;
    // causal: the last query rows see most, the first key rows are seen most
    const int r0 = (KEYS ? tiles - 1 - it.tile : it.tile) * kHeld;
    const T *Q = (const T *)a.q + qrow * D, *dO = (const T *)a.d_o + qrow * D;
    const T *K = (const T *)a.k + kv * D, *V = (const T *)a.v + kv * D;
    const float sl2 = a.scale * kLog2e;
    float2 acc[4][D / 32], acc2[4][KEYS ? D / 32 : 1];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            acc[i][c] = make_float2(0.f, 0.f);
            if (KEYS) acc2[i][KEYS ? c : 0] = make_float2(0.f, 0.f);
        }
    if constexpr (!KEYS) {
        const int rows = a.G * a.Nq, r1 = min(r0 + kHeld, rows);
        const int all = exact_most(seq, r0, r1, a.Nq);
        const int begin = it.part * split.chunk;
        if (it.part > 0 && begin >= all) return;
        const int most = min(all, begin + split.chunk);
        auto valid = [&](int r) {
            return r0 + r < r1 && (r0 + r) % a.Nq < seq.ql;
        };
        load_rows<T, D>(sA, D, Q + (size_t)r0 * D, kHeld, valid);
        load_rows<T, D>(sB, D, dO + (size_t)r0 * D, kHeld, valid);
        // O, for a moment where the keys will be
        load_rows<T, D>(sC, D + 4, (const T *)a.o + (qrow + r0) * D, kHeld,
                        valid);
        __syncthreads();
        float lse2[4], edge[4], delta[4];
        int seen[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 4 * y + i;
            float t = 0.f;
            for (int c = x; c < D; c += 16)
                t = fmaf(sB[r * D + c], sC[r * (D + 4) + c], t);
            delta[i] = row_sum(t);
            seen[i] = 0;
            lse2[i] = 0.f;
            if (valid(r)) {
                seen[i] = seq.seen((r0 + r) % a.Nq);
                lse2[i] = exact_lse(a.lse + qrow + r0 + r) * kLog2e;
                if (x == 0 && it.part == 0)
                    a.delta[qrow + r0 + r] = delta[i];
            }
            edge[i] = exact_edge(lse2[i]);
        }
        for (int j0 = begin; j0 < most; j0 += kPass) {
            __syncthreads();
            auto have = [&](int r) { return j0 + r < most; };
            load_rows<T, D>(sC, D + 4, K + (size_t)j0 * D, kPass, have);
            load_rows<T, D>(sE, D + 4, V + (size_t)j0 * D, kPass, have);
            __syncthreads();
            float s[4][4], dp[4][4];
            scores<D>(sA, sC, y, x, s);
            scores<D>(sB, sE, y, x, dp);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = exp2f(exact_exponent(
                        fmaf(s[i][e], sl2, -lse2[i]), edge[i]));
                    sW[(4 * y + i) * kPass + x + 16 * e] =
                        j0 + x + 16 * e < seen[i]
                            ? p * (dp[i][e] - delta[i]) : 0.f;
                }
            __syncwarp();
            weighted<D>(sW, sC, y, x, acc);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = r0 + 4 * y + i;
            if (!valid(4 * y + i)) continue;
            if (all > split.chunk) {
                float *o = split.o + (it.part * split.rows + qrow + r) * D +
                           2 * x;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) store2(o + 32 * c, acc[i][c]);
                continue;
            }
            T *o = (T *)a.dq + (qrow + r) * D + 2 * x;
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
                store2(o + 32 * c, tc::mul2(acc[i][c], make_float2(
                                                           a.scale, a.scale)));
        }
    } else {
        if (r0 >= seq.kl) return;
        auto valid = [&](int r) { return r0 + r < seq.kl; };
        load_rows<T, D>(sA, D, K + (size_t)r0 * D, kHeld, valid);
        load_rows<T, D>(sB, D, V + (size_t)r0 * D, kHeld, valid);
        // passing tiles of a head, of all heads, of this chunk
        const int first = seq.first_row(r0);
        const int per = (seq.ql - first + kPass - 1) / kPass;
        const int all = a.G * per, t0 = it.part * (split.chunk / kPass);
        if (it.part > 0 && t0 >= all) return;
        const int t1 = min(all, t0 + split.chunk / kPass);
        if (t0 < t1) {
            int g = t0 / per, i0 = first + t0 % per * kPass;
            for (int t = t0; t < t1; ++t) {
                const size_t at = (size_t)g * a.Nq + i0;
                __syncthreads();
                auto have = [&](int r) { return i0 + r < seq.ql; };
                load_rows<T, D>(sC, D + 4, Q + at * D, kPass, have);
                load_rows<T, D>(sE, D + 4, dO + at * D, kPass, have);
                if (threadIdx.x < kPass) {
                    const int r = threadIdx.x;
                    sL[r] = have(r) ? exact_lse(a.lse + qrow + at + r) * kLog2e
                                    : 0.f;
                    sD[r] = have(r) ? a.delta[qrow + at + r] : 0.f;
                    sN[r] = seq.seen(i0 + r);
                }
                __syncthreads();
                float s[4][4], dp[4][4];
                scores<D>(sA, sC, y, x, s);
                scores<D>(sB, sE, y, x, dp);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = x + 16 * e;
                    const float edge = exact_edge(sL[j]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool on = r0 + 4 * y + i < sN[j];
                        const float p =
                            on ? exp2f(exact_exponent(
                                     fmaf(s[i][e], sl2, -sL[j]), edge))
                               : 0.f;
                        sP[(4 * y + i) * kPass + j] = p;
                        sW[(4 * y + i) * kPass + j] =
                            on ? p * (dp[i][e] - sD[j]) : 0.f;
                    }
                }
                __syncwarp();
                weighted<D>(sW, sC, y, x, acc);
                weighted<D>(sP, sE, y, x, acc2);
                i0 += kPass;
                if (i0 >= seq.ql) {
                    i0 = first;
                    ++g;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!valid(4 * y + i)) continue;
            if (all * kPass > split.chunk) {
                float *o = split.o + (it.part * split.rows + kv + r0 + 4 * y +
                                      i) * 2 * D + 2 * x;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    store2(o + 32 * c, acc[i][c]);
                    store2(o + D + 32 * c, acc2[i][c]);
                }
                continue;
            }
            const size_t at = (kv + r0 + 4 * y + i) * D + 2 * x;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) {
                store2((T *)a.dk + at + 32 * c,
                       tc::mul2(acc[i][c], make_float2(a.scale, a.scale)));
                store2((T *)a.dv + at + 32 * c, acc2[i][c]);
            }
        }
    }
}

// The sums of dQ's rows, or of dK's and dV's, that were divided: D / 4 lanes a
// row.
template <typename T, int D, bool KEYS>
__global__ void __launch_bounds__(256)
    k_exact_add(const __grid_constant__ ExactView a,
                const __grid_constant__ Split split) {
    wait_for_stream();
    constexpr int L = D / 4, n = KEYS ? 2 : 1;
    const size_t row = ((size_t)blockIdx.x * 256 + threadIdx.x) / L;
    const int c = threadIdx.x % L * 4;
    if (row >= split.rows) return;
    int parts;
    if constexpr (KEYS) {
        const int j = (int)(row % a.Nk);
        const ExactSeq seq(a, (int)(row / a.Nk) / a.Hkv);
        if (j >= seq.kl) return;
        const int first = seq.first_row(j / kHeld * kHeld);
        const int all =
            a.G * ((seq.ql - first + kPass - 1) / kPass) * kPass;
        parts = (all + split.chunk - 1) / split.chunk;
    } else {
        const int group = a.G * a.Nq, r = (int)(row % group);
        const ExactSeq seq(a, (int)(row / group) / a.Hkv);
        if (r % a.Nq >= seq.ql) return;
        const int r0 = r / kHeld * kHeld;
        const int all = exact_most(seq, r0, min(r0 + kHeld, group), a.Nq);
        parts = (all + split.chunk - 1) / split.chunk;
    }
    if (parts < 2) return;
#pragma unroll
    for (int w = 0; w < n; ++w) {
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int p = 0; p < parts; ++p) {
            const float4 v = *reinterpret_cast<const float4 *>(
                split.o + ((p * split.rows + row) * n + w) * D + c);
            o.x += v.x;
            o.y += v.y;
            o.z += v.z;
            o.w += v.w;
        }
        const float f = w ? 1.0f : a.scale;
        T *to = (T *)(w ? a.dv : KEYS ? a.dk : a.dq) + row * D + c;
        store2(to, make_float2(o.x * f, o.y * f));
        store2(to + 2, make_float2(o.z * f, o.w * f));
    }
}

template <typename F>
cudaError_t by_type(const ExactView &a, F f) {
    using bf = __nv_bfloat16;
    const bool f32 = a.dtype == ELSAA_FP32;
    using I32 = std::integral_constant<int, 32>;
    using I64 = std::integral_constant<int, 64>;
    using I128 = std::integral_constant<int, 128>;
    switch (a.d) {
        case 32: return f32 ? f(0.f, I32{}) : f(bf{}, I32{});
        case 64: return f32 ? f(0.f, I64{}) : f(bf{}, I64{});
        default: return f32 ? f(0.f, I128{}) : f(bf{}, I128{});
    }
}

}  // namespace

namespace {

// Walks of `passing` rows of `rows` held ones in `tiles` tiles: chunks so that
// there are eight CTAs for each of a GB300's 152 SMs, of two tiles at least. (By
// the sizes alone: the workspace does not depend on the device.)
Split divide(long tiles, long passing, size_t rows) {
    const long passes = (passing + kPass - 1) / kPass;
    long n = (8 * 152 + tiles - 1) / tiles;
    if (n > passes / 2) n = passes / 2;
    if (n < 1) n = 1;
    Split s = {};
    s.chunk = (int)((passes + n - 1) / n) * kPass;
    s.splits = (int)((passing + s.chunk - 1) / s.chunk);
    s.rows = rows;
    return s;
}
long query_tiles(const ExactView &a) {
    return ((long)a.G * a.Nq + kHeld - 1) / kHeld;
}
Split divide_keys(const ExactView &a) {
    return divide(query_tiles(a) * a.B * a.Hkv, a.Nk,
                  (size_t)a.B * a.H * a.Nq);
}
// dK, dV: the rows of every head in tiles of their own
Split divide_queries(const ExactView &a) {
    return divide((long)((a.Nk + kHeld - 1) / kHeld) * a.B * a.Hkv,
                  a.G * (((long)a.Nq + kPass - 1) / kPass) * kPass,
                  (size_t)a.B * a.Hkv * a.Nk);
}

}  // namespace

size_t exact_chunk_bytes(const ExactView &a) {
    const Split s = divide_keys(a);
    return s.splits > 1 ? sizeof(float) * (a.d + 2) * s.splits * s.rows : 0;
}

cudaError_t launch_exact_fwd_simt(const ExactView &a, float *part,
                                  cudaStream_t st) {
    Split split = divide_keys(a);
    split.o = part;
    split.ml = (float2 *)(part + split.rows * split.splits * a.d);
    const int tiles = (int)(((long)a.G * a.Nq + kHeld - 1) / kHeld);
    const dim3 grid((unsigned)((long)tiles * a.B * a.Hkv * split.splits));
    const size_t smem = sizeof(float) * (kHeld * a.d + 2 * kPass * (a.d + 4) +
                                         kHeld * kPass);
    return by_type(a, [&](auto t, auto dim) {
        using T = decltype(t);
        constexpr int D = decltype(dim)::value;
        cudaError_t e = launch_after(k_exact_fwd<T, D>, grid, kThreads, smem,
                                     st, a, split, tiles);
        if (e == cudaSuccess && split.splits > 1)
            e = launch_after(
                k_exact_join<T, D>,
                dim3((unsigned)((split.rows * (D / 4) + 255) / 256)), 256, 0,
                st, a, split);
        return e;
    });
}

size_t exact_add_bytes(const ExactView &a) {
    const Split q = divide_keys(a), k = divide_queries(a);
    const size_t x = q.splits > 1 ? q.splits * q.rows : 0;
    const size_t y = k.splits > 1 ? 2 * k.splits * k.rows : 0;
    return sizeof(float) * a.d * (x > y ? x : y);
}

cudaError_t launch_exact_bwd_simt(const ExactView &a, bool keys, float *part,
                                  cudaStream_t st) {
    Split split = keys ? divide_queries(a) : divide_keys(a);
    split.o = part;
    const long tiles = keys ? (a.Nk + kHeld - 1) / kHeld : query_tiles(a);
    const dim3 grid((unsigned)(tiles * a.B * a.Hkv * split.splits));
    const size_t smem =
        sizeof(float) * (2 * kHeld * a.d + 2 * kPass * (a.d + 4) +
                         (keys ? 2 : 1) * kHeld * kPass + 3 * kPass);
    return by_type(a, [&](auto t, auto dim) {
        using T = decltype(t);
        constexpr int D = decltype(dim)::value;
        const dim3 rows((unsigned)((split.rows * (D / 4) + 255) / 256));
        auto run = [&](auto which) {
            constexpr bool K = decltype(which)::value;
            cudaError_t e = launch_after(k_exact_bwd<T, D, K>, grid, kThreads,
                                         smem, st, a, split, (int)tiles);
            if (e == cudaSuccess && split.splits > 1)
                e = launch_after(k_exact_add<T, D, K>, rows, 256, 0, st, a,
                                 split);
            return e;
        };
        return keys ? run(std::true_type{}) : run(std::false_type{});
    });
}

}  // namespace elsaa
