// Attention of new tokens over the 8-bit cache: the CUDA-core kernel, the
// merge of items that several CTAs shared, and the accumulated weights.
//
// k_cache_attn_simt walks the tiles of its range once with a running maximum
// and sum. A warp takes 32 tokens of a tile: the lanes of a row hold 16
// channels each (one 16-byte load of codes), so a token's score is 16 products
// a lane and a few shuffles, its value 16 products again, and O stays in
// registers for all columns of the item. A cached byte is read once per group
// of up to 4 columns and costs 2 conversions' share and 2 fp32 products per
// column: with one column (ungrouped heads) that is below what the SMs have
// to spare while HBM delivers the byte, with more the products bound it. 4
// sequences of up to 4096 tokens, 12 fp32 heads of 64: 10 us with the merge,
// two launches' latencies above all.
#include "cache_common.cuh"

namespace elsaa {

namespace {

using namespace cache;

constexpr int kSaThreads = 128;
constexpr float kLog2eF = 1.4426950408889634f;

template <typename T, int D, int NG>
__global__ void __launch_bounds__(kSaThreads)
    k_cache_attn_simt(const __grid_constant__ CacheAttn A) {
    wait_for_stream();
    constexpr int LPR = D / 16;   // lanes per row
    constexpr int R = 32 / LPR;   // rows per warp load
    constexpr int S = 32 / R;     // loads per tile
    __shared__ float accs[4][NG][D];
    __shared__ float ms[4][NG], ls[4][NG];
    const CacheView &c = A.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int sub = lane % LPR, rg = lane / LPR;
    __shared__ Seq near[kNearSeqs];
    Seq own;
    const Start first = divide<kSaThreads>(A, near, own);
    Walk walk(first, near, own);
    const float sl2 = c.scale * kLog2eF;
    const int GT = c.G * c.T;

    while (walk.left > 0) {
        const Item it = walk.next(A);
        const size_t bh = (size_t)it.b * c.Hkv + it.h;
        float qf[NG][16], acc[NG][16], m[NG], l[NG];
        int limit[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            m[g] = -INFINITY;
            l[g] = 0.0f;
            limit[g] =
                g < it.cols ? last_seen(A, it.len, it.n, it.col0 + g) : -1;
#pragma unroll
            for (int i = 0; i < 16; ++i) qf[g][i] = acc[g][i] = 0.0f;
            if (limit[g] >= 0) {
                const T *x = (const T *)A.q +
                             query_row(A, it.b, it.h, it.col0 + g) * D +
                             sub * 16;
                load8(x, qf[g]);
                load8(x + 8, qf[g] + 8);
            }
        }
        for (int t = it.off; t < it.off + it.count; ++t) {
            // lane i: token i of the warp's 32
            const int w = t * kCacheTile + warp * 32 + lane;
            int id = -1, pos = 0;
            float ks = 0.0f, vs = 0.0f;
            if (w < it.walk) {
                int p = w / c.ps;
                if (A.pages) p = A.pages[bh * A.n_sel + p];
                pos = p * c.ps + w % c.ps;
                if (p >= 0 && p < c.max_pages && pos < it.len)
                    id = page_id(c, it.b, p);
                if (id >= 0) {
                    const size_t ph = (size_t)id * c.Hkv + it.h;
                    ks = c.ks[ph] * sl2;
                    vs = c.vs[ph];
                }
            }
            const int row = w % c.ps;
            uint4 kr[S], vr[S];
#pragma unroll
            for (int s = 0; s < S; ++s) {
                const int tk = s * R + rg;
                const int i = __shfl_sync(0xffffffffu, id, tk);
                const int ro = __shfl_sync(0xffffffffu, row, tk);
                kr[s] = vr[s] = make_uint4(0, 0, 0, 0);
                if (i >= 0) {
                    const size_t at =
                        (((size_t)i * c.Hkv + it.h) * c.ps + ro) * D + sub * 16;
                    kr[s] = *(const uint4 *)(c.k + at);
                    vr[s] = *(const uint4 *)(c.v + at);
                }
            }
            float sc[NG][S];
#pragma unroll
            for (int s = 0; s < S; ++s) {
                float x[16];
                from_e4m3x4(kr[s].x, x);
                from_e4m3x4(kr[s].y, x + 4);
                from_e4m3x4(kr[s].z, x + 8);
                from_e4m3x4(kr[s].w, x + 12);
                const int tk = s * R + rg;
                const float f = __shfl_sync(0xffffffffu, ks, tk);
                const int po = __shfl_sync(0xffffffffu, pos, tk);
                const bool in = __shfl_sync(0xffffffffu, id, tk) >= 0;
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    float d = 0.0f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) d = fmaf(qf[g][i], x[i], d);
#pragma unroll
                    for (int o = 1; o < LPR; o <<= 1)
                        d += __shfl_xor_sync(0xffffffffu, d, o);
                    sc[g][s] = in && po <= limit[g] ? d * f : -INFINITY;
                }
            }
            if (A.scores) {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    const int at = t * kCacheTile + warp * 32 + s * R + rg;
                    if (sub == 0 && at < it.walk)
#pragma unroll
                        for (int g = 0; g < NG; ++g)
                            if (g < it.cols)
                                A.scores[(bh * GT + it.col0 + g) * A.slots +
                                         at] = sc[g][s];
                }
            }
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float mx = sc[g][0];
#pragma unroll
                for (int s = 1; s < S; ++s) mx = fmaxf(mx, sc[g][s]);
#pragma unroll
                for (int o = LPR; o < 32; o <<= 1)
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                mx = fmaxf(mx, m[g]);
                const float ref = mx == -INFINITY ? 0.0f : mx;
                const float al = tc::ex2_approx(m[g] - ref);
                m[g] = mx;
                l[g] *= al;
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[g][i] *= al;
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    const bool seen = sc[g][s] != -INFINITY;
                    const float p = tc::ex2_approx(sc[g][s] - ref);
                    l[g] += p;
                    sc[g][s] = seen ? p : -1.0f;
                }
            }
#pragma unroll
            for (int s = 0; s < S; ++s) {
                float x[16];
                from_e4m3x4(vr[s].x, x);
                from_e4m3x4(vr[s].y, x + 4);
                from_e4m3x4(vr[s].z, x + 8);
                from_e4m3x4(vr[s].w, x + 12);
                const float f = __shfl_sync(0xffffffffu, vs, s * R + rg);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    // a token that a column does not see adds nothing,
                    // whatever its codes are
                    const float p = sc[g][s] * f;
                    if (!(sc[g][s] < 0.0f))
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            acc[g][i] = fmaf(p, x[i], acc[g][i]);
                }
            }
        }
        // the warp's rows, then the four warps
#pragma unroll
        for (int g = 0; g < NG; ++g) {
#pragma unroll
            for (int o = LPR; o < 32; o <<= 1) {
                l[g] += __shfl_xor_sync(0xffffffffu, l[g], o);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    acc[g][i] += __shfl_xor_sync(0xffffffffu, acc[g][i], o);
            }
            if (rg == 0)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    accs[warp][g][sub * 16 + i] = acc[g][i];
            if (lane == 0) {
                ms[warp][g] = m[g];
                ls[warp][g] = l[g];
            }
        }
        __syncthreads();
        for (int g = 0; g < it.cols; ++g) {
            float M = ms[0][g], L = 0.0f, x = 0.0f;
            for (int k = 1; k < 4; ++k) M = fmaxf(M, ms[k][g]);
            const float ref = M == -INFINITY ? 0.0f : M;
            for (int k = 0; k < 4; ++k) {
                const float f = tc::ex2_approx(ms[k][g] - ref);
                L += f * ls[k][g];
                if (tid < D) x += f * accs[k][g][tid];
            }
            const int col = it.col0 + g;
            if (it.slot >= 0) {
                float *at = piece(A, blockIdx.x, it.slot, g);
                if (tid < D) at[tid] = x;
                if (tid == 0) {
                    at[D] = M;
                    at[D + 1] = L;
                }
            } else {
                if (tid == 0) store_lse(A, it.b, it.h, it.n, col, M, L);
                if (tid < D && token_of(A, col) < it.n)
                    store_o(A, query_row(A, it.b, it.h, col), tid,
                            L == 0.0f ? 0.0f : x / L);
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------- merge
//
// The columns of an item that began in CTA blockIdx.x and went on in others:
// its pieces in order, so the result does not depend on which CTA was first.
// A thread has a channel of a column; with few columns a block the pieces are
// shared out among groups of threads, whose sums are added in order as well. A
// few dependent reads of L2 is all it takes, 700 cycles for 8 pieces a thread,
// so it is as short as its loads in flight are many: with few items, whose
// pieces are many, a block has one column (64 pieces of 4 columns: 9 us less
// than with 4 columns a block), else 4, for fewer blocks.
constexpr int kMgThreads = 512;
int merge_cols(const CacheAttn &A) {
    const long items = (long)A.c.B * A.c.Hkv * A.groups;
    return A.cols < 4 || 8 * items <= A.ctas ? 1 : 4;
}

__global__ void __launch_bounds__(kMgThreads)
    k_cache_merge(const __grid_constant__ CacheAttn A, int cols,
                  bool tensor_cores) {
    wait_for_stream();
    if (tensor_cores) let_next_launch();
    __shared__ float sm[kMgThreads], sl[kMgThreads], sx[kMgThreads];
    const CacheSplit s = A.split[blockIdx.x];
    if (s.pieces == 0) return;
    const CacheView &c = A.c;
    const int tid = threadIdx.x, d = c.d, ch = tid % d, group = tid / d;
    const int parts = kMgThreads / d / cols;
    const int g = blockIdx.y * cols + group % cols, part = group / cols;
    const int h = s.hc / A.groups, col = s.hc % A.groups * A.cols + g;
    float M = -INFINITY, L = 0.0f, x = 0.0f;
    if (part < parts) {
        constexpr int U = 8;
        for (int i0 = part; i0 < s.pieces; i0 += parts * U) {
            float m[U], l[U], y[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u * parts;
                m[u] = -INFINITY;
                l[u] = y[u] = 0.0f;
                if (i < s.pieces) {
                    const float *at = piece(A, blockIdx.x + i, i == 0, g);
                    y[u] = at[ch];
                    m[u] = at[d];
                    l[u] = at[d + 1];
                }
            }
            float top = M;
#pragma unroll
            for (int u = 0; u < U; ++u) top = fmaxf(top, m[u]);
            const float ref = top == -INFINITY ? 0.0f : top;
            const float f = exp2f(M - ref);
            x *= f;
            L *= f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float e = exp2f(m[u] - ref);
                x += e * y[u];
                L += e * l[u];
            }
            M = top;
        }
    }
    if (parts > 1) {
        sm[tid] = M;
        sl[tid] = L;
        sx[tid] = x;
        __syncthreads();
        if (part > 0) return;
        for (int p = 1; p < parts; ++p) {
            const int o = tid + p * cols * d;
            const float top = fmaxf(M, sm[o]);
            const float ref = top == -INFINITY ? 0.0f : top;
            const float f = exp2f(M - ref), e = exp2f(sm[o] - ref);
            x = x * f + sx[o] * e;
            L = L * f + sl[o] * e;
            M = top;
        }
    }
    if (part > 0 || col >= c.G * c.T) return;
    if (ch == 0) store_lse(A, s.b, h, s.n, col, M, L);
    if (token_of(A, col) < s.n)
        store_o(A, query_row(A, s.b, h, col), ch, L == 0.0f ? 0.0f : x / L);
}

// ----------------------------------------------------------------- weights
//
// weight_out_j = weight_in_j + sum over the columns of 2^(s_j - lse), from
// the scores that the attention kernel left: 4 bytes a token and column,
// where a second walk over the keys would read d bytes. Four neighbouring
// tokens a thread (they share a page), a column's in one load. The scores come
// from L2 as long as they fit; with them, 32 sequences of up to 8192 tokens, 8
// heads, 4 queries each, take 62 us, and the bytes of codes and weights 39.
constexpr int kWtThreads = 128;
constexpr int kWtTokens = 4 * kWtThreads;

__global__ void __launch_bounds__(kWtThreads)
    k_cache_weights(const __grid_constant__ CacheAttn A) {
    wait_for_stream();
    let_next_launch();
    __shared__ int slot[kWtTokens / 16];
    __shared__ float lse[128];
    const CacheView &c = A.c;
    const int h = blockIdx.y, b = blockIdx.z, GT = c.G * c.T;
    const int tid = threadIdx.x;
    const size_t bh = (size_t)b * c.Hkv + h;
    const int j0 = blockIdx.x * kWtTokens, j = j0 + 4 * tid;
    const auto [len, n] = lengths(c, b);
    if (j0 >= len) return;
    const bool any = n > 0;
    // a column that is no query adds nothing: 2^(s - inf)
    if (any && tid < GT)
        lse[tid] = token_of(A, tid) < n ? A.lse2[bh * GT + tid] : INFINITY;
    long at = j;
    if (A.pages) {
        // the list entries of this block's pages
        if (tid < kWtTokens / 16) slot[tid] = -1;
        __syncthreads();
        const int p0 = j0 / c.ps, np = kWtTokens / c.ps;
        const int listed = min(A.n_sel, (len + c.ps - 1) / c.ps);
        for (int e = tid; e < listed; e += kWtThreads) {
            const int p = A.pages[bh * A.n_sel + e] - p0;
            if (p >= 0 && p < np) slot[p] = e;
        }
        __syncthreads();
        const int e = slot[(j - j0) / c.ps];
        at = e < 0 ? -1 : (long)e * c.ps + j % c.ps;
    }
    __syncthreads();
    if (j >= len) return;
    // a row of weights is a whole number of pages long, so whole fours can be
    // read; only tokens that are held are written
    const size_t w = bh * c.max_pages * c.ps + j;
    const float4 z = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    const float4 was = A.weight_in ? *(const float4 *)(A.weight_in + w) : z;
    float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (any && at >= 0) {
        const float *s = A.scores + bh * GT * A.slots + at;
#pragma unroll 4
        for (int col = 0; col < GT; ++col) {
            const float4 v = *(const float4 *)(s + (size_t)col * A.slots);
            const float l = lse[col];
            // a masked score beside an empty row's -inf is not a number
            const float y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (y[i] != -INFINITY) x[i] += tc::ex2_approx(y[i] - l);
        }
    }
    float *out = A.weight_out + w;
    const float4 sum =
        make_float4(was.x + x[0], was.y + x[1], was.z + x[2], was.w + x[3]);
    if (j + 3 < len) {
        *(float4 *)out = sum;
    } else {
        out[0] = sum.x;
        if (j + 1 < len) out[1] = sum.y;
        if (j + 2 < len) out[2] = sum.z;
    }
}

template <typename T, int D, int NG>
cudaError_t launch_simt(const CacheAttn &A, cudaStream_t st) {
    return launch_cache<k_cache_attn_simt<T, D, NG>>(
        dim3(A.ctas), kSaThreads, 0, 0, 1, st, A);
}

template <typename T, int D>
cudaError_t launch_simt_cols(const CacheAttn &A, cudaStream_t st) {
    switch (A.cols) {
        case 1: return launch_simt<T, D, 1>(A, st);
        case 2: return launch_simt<T, D, 2>(A, st);
        default: return launch_simt<T, D, 4>(A, st);
    }
}

template <typename T>
cudaError_t launch_simt_d(const CacheAttn &A, cudaStream_t st) {
    switch (A.c.d) {
        case 32: return launch_simt_cols<T, 32>(A, st);
        case 64: return launch_simt_cols<T, 64>(A, st);
        default: return launch_simt_cols<T, 128>(A, st);
    }
}

}  // namespace

cudaError_t launch_cache_attn_simt(const CacheAttn &A, cudaStream_t st) {
    return A.c.dtype == ELSAA_FP32 ? launch_simt_d<float>(A, st)
                                   : launch_simt_d<__nv_bfloat16>(A, st);
}

cudaError_t launch_cache_merge(const CacheAttn &A, bool tensor_cores,
                               cudaStream_t st) {
    const int cols = merge_cols(A);
    return launch_cache<k_cache_merge>(dim3(A.ctas, A.cols / cols),
                                       kMgThreads, 0, 0, 1, st, A, cols,
                                       tensor_cores);
}

cudaError_t launch_cache_weights(const CacheAttn &A, cudaStream_t st) {
    const long cap = (long)A.c.max_pages * A.c.ps;
    return launch_cache<k_cache_weights>(
        dim3((unsigned)((cap + kWtTokens - 1) / kWtTokens), A.c.Hkv, A.c.B),
        kWtThreads, 0, 0, 1, st, A);
}

}  // namespace elsaa
