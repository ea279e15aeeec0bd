// Attention of new tokens over the 8-bit cache on the tensor cores: bf16
// queries, d_h 64 or 128.
//
// The cached codes are operands as they are (kind::f8f6f4, e4m3, fp32 sums):
// nothing is converted on the way from HBM to the products. With a tile of
// 128 tokens as M,
//     S^T [128 tokens x columns] = K [128 x d] Q^T         (columns: queries)
//     O^T [d x columns]          = V^T [d x 128] P^T.
// The other operand is made to fit. A bf16 query has 8 significant bits, an
// e4m3 number 4: q 2^-e = hi + lo / 16 with hi the nearest e4m3 number, and
// the remainder, at most half a step of it, again has 4 bits, so hi and lo
// hold q exactly (elements below 2^-14 of the row's largest lose bits below
// 2^-22 of it). Two columns a query; scores are as exact as fp32 products. A
// softmax weight is an fp32 number; three e4m3 numbers (256, 16 and 1 times
// the remainder so far) hold it to 2^-12 relative, and to 2^-26 of the
// tile's largest where it is smaller: a bf16 weight would have 2^-9. Each
// tile's weights are relative to the tile's own maximum, so that a flat tail
// behind one large score keeps its bits; sums and O, in registers, are
// rescaled in fp32.
//
// Scales: a page's key scale multiplies the score in fp32; its value scale,
// relative to the tile's largest (both powers of two), goes into the weight
// before it is split.
//
// d = 64: V's rows are taken in pairs, M = (parity, d), 64 pairs as K, so that
// every product has M = 128; one product for the weights of the even tokens
// (its lower 64 lanes count), one for the odd (the upper). O's halves are
// added at the end.
//
// CTA: 4 softmax warps (a token a thread for S, a channel a thread for O), a
// producer warp (page table, TMA of the pages' rows, scales), a product warp
// and two query warps, which split the next item's queries while this one is
// walked. The range's tiles run through rings of K and V buffers; S of tile
// i + 1 is issued before O of tile i, so the softmax finds its next scores
// ready. Two CTAs share an SM.
#include "cache_common.cuh"

namespace elsaa {

namespace {

using namespace cache;
using namespace tc;

constexpr int kTaThreads = 256;
// Registers: 128 a thread at launch (two CTAs); the four softmax warps take
// what the other four leave, 2 * 128 in all.
constexpr int kTaRegsSoft = 184, kTaRegsOther = 72;
constexpr float kLog2eF = 1.4426950408889634f;
constexpr int kMaxPagesPerTile = kCacheTile / 16;

template <int D, int NV>
struct Cfg {
    static constexpr int N1 = 2 * NV < 16 ? 16 : 2 * NV;  // columns of S
    static constexpr int NP = (3 * NV + 15) / 16 * 16;    // of one P product
    static constexpr int NO = D == 128 ? NP : 2 * NP;     // of O
    static constexpr int W = NP <= 32 ? 32 : 64;  // bytes of a token's P row
    static constexpr int KS = D == 64 ? (NV < 16 ? 6 : 5) : (NV < 16 ? 3 : 2);
    static constexpr int VS = D == 64 ? (NV < 16 ? 6 : 5) : 3;
    static constexpr uint32_t kTile = kCacheTile * D;
    static constexpr uint32_t kQ = N1 * D;
    static constexpr uint32_t kP = kCacheTile * W;
    static constexpr uint32_t kSmem =
        1024 + (KS + VS) * kTile + 2 * kQ + 2 * kP;
    static constexpr uint32_t kCols = 2 * N1 + 2 * NO;
    static constexpr uint32_t kTmem = kCols <= 64    ? 64
                                      : kCols <= 128 ? 128
                                                     : 256;
    static_assert(kCols <= 256, "two CTAs share tensor memory");
};

// Shared-memory descriptor of an operand whose lines are `line` = 32, 64 or
// 128 bytes, with the swizzle of that width: 8 lines are an atom.
__device__ __forceinline__ uint64_t line_desc(uint32_t start, uint32_t line) {
    uint64_t d = 0;
    d |= (uint64_t)((start >> 4) & 0x3FFF);
    d |= (uint64_t)1 << 16;                      // one atom across
    d |= (uint64_t)((line * 8) >> 4) << 32;      // atoms along the lines
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)(line == 128 ? 2 : line == 64 ? 4 : 6) << 61;
    return d;
}
// kind::f8f6f4 with e4m3 operands and fp32 sums.
__host__ __device__ constexpr uint32_t idesc_e4m3(int M, int N, bool a_mn,
                                                  bool b_mn) {
    return (1u << 4) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void mma_e4m3(uint32_t d_tmem, uint64_t a,
                                         uint64_t b, uint32_t idesc,
                                         uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n}\n" ::
            "r"(d_tmem),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate));
}

// N consecutive columns of the thread's lane, N = 2, 4, 8 or a multiple of 16.
template <int N>
__device__ __forceinline__ void tmem_read(uint32_t t, float *x) {
    if constexpr (N >= 16) {
        uint32_t r[16];
        tmem_ld16(t, r);
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(r[i]);
        if constexpr (N > 16) tmem_read<N - 16>(t + 16, x + 16);
    } else if constexpr (N == 8) {
        uint32_t r[8];
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x8.b32 "
            "{%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
            : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]),
              "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
            : "r"(t));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r[i]);
    } else if constexpr (N == 4) {
        uint32_t r[4];
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
            : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
            : "r"(t));
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(r[i]);
    } else {
        static_assert(N == 2, "columns");
        uint32_t r[2];
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x2.b32 {%0,%1}, [%2];"
                     : "=r"(r[0]), "=r"(r[1])
                     : "r"(t));
        x[0] = __uint_as_float(r[0]);
        x[1] = __uint_as_float(r[1]);
    }
}

// V = 2 or 4 neighbouring bf16 values.
template <int V>
__device__ __forceinline__ void load_row(const __nv_bfloat16 *p, float *x) {
    uint32_t w[V / 2];
    if constexpr (V == 4) {
        const uint2 a = *(const uint2 *)p;
        w[0] = a.x;
        w[1] = a.y;
    } else {
        w[0] = *(const uint32_t *)p;
    }
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}

// Largest of the warp's values, in every lane.
__device__ __forceinline__ float redux_max(float x) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

// The pages of one tile, written by the producer.
struct TileMeta {
    float ks[kMaxPagesPerTile];   // key scale
    float vs[kMaxPagesPerTile];   // value scale over the tile's largest
    int pos[kMaxPagesPerTile];    // first position
    int rows[kMaxPagesPerTile];   // rows that count
    float vmax;
};

struct Bars {
    uint64_t k_full[6], k_empty[6], v_full[6], v_empty[6], m_full[6];
    uint64_t s_full[2], p_ready[2], o_full[2], q_full[2], q_empty[2], drain;
};

template <int D, int NV>
__global__ void __launch_bounds__(kTaThreads, 2)
    k_cache_attn_tc(const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV,
                    const __grid_constant__ CacheAttn A) {
    using C = Cfg<D, NV>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Bars bars;
    __shared__ TileMeta meta[C::VS];
    __shared__ Item items[2];
    __shared__ float factors[2][NV];  // of an item's columns' scores
    __shared__ int limits[2][NV];     // last positions that they see
    __shared__ uint32_t tbase;
    __shared__ int abort_flag;
    __shared__ __align__(16) float red[2][NV][4];
    __shared__ __align__(16) float fin[NV][4];
    __shared__ float half[D == 64 ? NV * 64 : 1];
    volatile int *abort = &abort_flag;
    const CacheView &c = A.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t sK = base, sV = sK + C::KS * C::kTile;
    const uint32_t sQ = sV + C::VS * C::kTile, sP = sQ + 2 * C::kQ;

    // set up while the kernel before ends
    if (warp == 5) tmem_alloc(&tbase, C::kTmem);
    if (tid == 0) {
        for (int s = 0; s < 6; ++s) {
            mbar_init(&bars.k_full[s], 1);
            mbar_init(&bars.k_empty[s], 1);
            mbar_init(&bars.v_full[s], 1);
            mbar_init(&bars.v_empty[s], 1);
            mbar_init(&bars.m_full[s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars.s_full[s], 1);
            mbar_init(&bars.p_ready[s], 128);
            mbar_init(&bars.o_full[s], 1);
            mbar_init(&bars.q_full[s], 2);   // the query warps
            mbar_init(&bars.q_empty[s], 5);  // products, four softmax warps
        }
        mbar_init(&bars.drain, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tbase;
    wait_for_stream();
    const Start first =
        divide<kTaThreads>(A, (int *)(smem_raw + C::kSmem));
    const int count = first.count;

    if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(
            kTaRegsOther));
        if (warp == 4) {
            // ------------------------------------------------ pages and scales
            const int pt = kCacheTile / c.ps;  // pages of a tile
            Walk walk(first);
            Item it;
            it.count = it.off = 0;
            bool ok = true;
            int kn = 0, vn = 0;  // loads issued
            int t = 0;           // tile within the item
            for (int i = 0; i < count; ++i, ++t) {
                if (t == it.off + it.count) {
                    it = walk.next(A);
                    t = it.off;
                }
                // lane l: the tile's l-th page
                const int e = t * pt + lane;
                int p = -1, id = -1, rows = 0;
                if (lane < pt && (long)e * c.ps < it.walk)
                    p = A.pages ? A.pages[((size_t)it.b * c.Hkv + it.h) *
                                              A.n_sel + e]
                                : e;
                if (p >= 0 && p < c.max_pages) {
                    rows = min(it.len - p * c.ps, c.ps);
                    if (rows > 0) id = page_id(c, it.b, p);
                }
                if (id < 0) rows = 0;
                const int ph = id * c.Hkv + it.h;  // fits: checked by the host
                const uint32_t live = __ballot_sync(0xffffffffu, id >= 0);
                const uint32_t bytes = __popc(live) * c.ps * D;
                const int ks = i % C::KS, vs = i % C::VS;
                if (i >= C::KS)
                    ok = __all_sync(0xffffffffu,
                                    mbar_wait_or_abort(&bars.k_empty[ks],
                                                       (i / C::KS - 1) & 1, abort,
                                                       c.status, 180));
                if (!ok) break;
                if (lane == 0) mbar_expect_tx(&bars.k_full[ks], bytes);
                __syncwarp();
                if (id >= 0)
                    tma_load_2d(sK + ks * C::kTile + lane * c.ps * D, &tmK, 0,
                                ph * c.ps, &bars.k_full[ks]);
                ++kn;
                float k_sc = 0.0f, v_sc = 0.0f;
                if (id >= 0) {
                    k_sc = c.ks[ph];
                    v_sc = c.vs[ph];
                }
                if (i >= C::VS)
                    ok = __all_sync(0xffffffffu,
                                    mbar_wait_or_abort(&bars.v_empty[vs],
                                                       (i / C::VS - 1) & 1, abort,
                                                       c.status, 181));
                if (!ok) break;
                if (lane == 0) mbar_expect_tx(&bars.v_full[vs], bytes);
                __syncwarp();
                if (id >= 0)
                    tma_load_2d(sV + vs * C::kTile + lane * c.ps * D, &tmV, 0,
                                D == 128 ? ph * c.ps : ph * c.ps / 2,
                                &bars.v_full[vs]);
                ++vn;
                const float vmax = warp_max(v_sc);
                if (lane < pt) {
                    TileMeta &m = meta[vs];
                    m.ks[lane] = k_sc;
                    m.vs[lane] = vmax > 0.0f ? v_sc / vmax : 0.0f;
                    m.pos[lane] = p * c.ps;
                    m.rows[lane] = rows;
                    if (lane == 0) m.vmax = vmax;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.m_full[vs]);
            }
            // whatever was asked for has arrived before the CTA ends
            for (int j = max(0, kn - C::KS); j < kn; ++j)
                mbar_wait(&bars.k_full[j % C::KS], (j / C::KS) & 1, c.status,
                          182);
            for (int j = max(0, vn - C::VS); j < vn; ++j)
                mbar_wait(&bars.v_full[j % C::VS], (j / C::VS) & 1, c.status,
                          183);
        } else if (warp == 5) {
            // -------------------------------------------------------- products
            const bool el = elect_one();
            auto wait = [&](uint64_t *bar, uint32_t par, int site) {
                return __all_sync(0xffffffffu,
                                  mbar_wait_or_abort(bar, par, abort, c.status,
                                                     site));
            };
            const uint32_t id_s = idesc_e4m3(128, C::N1, false, false);
            const uint32_t id_o = idesc_e4m3(128, C::NP, true, true);
            bool ok = true;
            auto values = [&](int j) {  // O of tile j
                const int vs = j % C::VS, b = j & 1;
                if (!wait(&bars.v_full[vs], (j / C::VS) & 1, 185)) return false;
                if (!wait(&bars.p_ready[b], (j >> 1) & 1, 186)) return false;
                tc_fence_after();
                if (el) {
                    const uint64_t dV = line_desc(sV + vs * C::kTile, 128);
                    const uint64_t dP = line_desc(sP + b * C::kP, C::W);
                    const uint32_t o = tm + 2 * C::N1 + b * C::NO;
                    if (D == 128) {
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            mma_e4m3(o, desc_at(dV, x * 4096),
                                     desc_at(dP, x * 32 * C::W), id_o, x > 0);
                    } else {
#pragma unroll
                        for (int par = 0; par < 2; ++par)
#pragma unroll
                            for (int x = 0; x < 2; ++x)
                                mma_e4m3(o + par * C::NP, desc_at(dV, x * 4096),
                                         desc_at(dP, (par * 64 + x * 32) * C::W),
                                         id_o, x > 0);
                    }
                    mma_commit(&bars.o_full[b]);
                    mma_commit(&bars.v_empty[vs]);
                }
                __syncwarp();
                return true;
            };
            int item = 0, left = 0;  // tiles of the item
            uint64_t dQ = 0;
            for (int i = 0; i < count && ok; ++i) {
                if (left == 0) {
                    ok = wait(&bars.q_full[item & 1], (item >> 1) & 1, 187);
                    if (!ok) break;
                    left = items[item & 1].count;
                    dQ = line_desc(sQ + (item & 1) * C::kQ, D);
                    ++item;
                }
                --left;
                const int ks = i % C::KS, b = i & 1;
                ok = wait(&bars.k_full[ks], (i / C::KS) & 1, 188);
                if (!ok) break;
                tc_fence_after();
                if (el) {
                    const uint64_t dK = line_desc(sK + ks * C::kTile, D);
#pragma unroll
                    for (int x = 0; x < D / 32; ++x)
                        mma_e4m3(tm + b * C::N1, desc_at(dK, x * 32),
                                 desc_at(dQ, x * 32), id_s, x > 0);
                    mma_commit(&bars.s_full[b]);
                    mma_commit(&bars.k_empty[ks]);
                    if (left == 0) mma_commit(&bars.q_empty[(item - 1) & 1]);
                }
                __syncwarp();
                if (i > 0) ok = values(i - 1);
            }
            if (ok && count > 0) values(count - 1);
            // every product is complete before the tensor memory is given back
            if (el) mma_commit(&bars.drain);
            mbar_wait(&bars.drain, 0, c.status, 189);
            __syncwarp();
        } else if (warp >= 6) {
            // --------------------------------------------------------- queries
            Walk walk(first);
            constexpr int V = D / 32;  // elements a lane
            for (int k = 0; walk.left > 0; ++k) {
                const Item it = walk.next(A);
                const int qs = k & 1;
                bool ok = true;
                // this warp's columns, a few at a time; the first are read before
                // the buffer is free
                constexpr int Z = (NV + 1) / 2, ZB = Z < 4 ? Z : 4;
#pragma unroll 1
                for (int z0 = 0; z0 < Z; z0 += ZB) {
                    float x[ZB][V];
                    int lim[ZB];
#pragma unroll
                    for (int z = 0; z < ZB; ++z) {
                        const int g = 2 * (z0 + z) + warp - 6;
                        lim[z] = g < it.cols
                                     ? last_seen(A, it.len, it.n, it.col0 + g)
                                     : -1;
#pragma unroll
                        for (int i = 0; i < V; ++i) x[z][i] = 0.0f;
                        if (lim[z] >= 0)
                            load_row<V>((const __nv_bfloat16 *)A.q +
                                            query_row(A, it.b, it.h, it.col0 + g) *
                                                D + lane * V,
                                        x[z]);
                    }
                    if (z0 == 0 && k >= 2)
                        ok = __all_sync(0xffffffffu,
                                        mbar_wait_or_abort(&bars.q_empty[qs],
                                                           ((k >> 1) - 1) & 1,
                                                           abort, c.status, 184));
                    if (!ok) break;
#pragma unroll
                    for (int z = 0; z < ZB; ++z) {
                        const int g = 2 * (z0 + z) + warp - 6;
                        if (g >= NV) break;
                        float amax = 0.0f;
#pragma unroll
                        for (int i = 0; i < V; ++i)
                            amax = fmaxf(amax, magnitude(x[z][i]));
                        const int e = least_exponent(warp_max(amax), 0x600000u, 8,
                                                     -100, kCacheExpHigh);
                        const float f = pow2(-e);
                        uint32_t w[2] = {0, 0};
#pragma unroll
                        for (int i = 0; i < V; i += 2) {
                            // an infinity has no split: it counts as NaN
                            const float y0 = isinf(x[z][i]) ? NAN : x[z][i] * f;
                            const float y1 =
                                isinf(x[z][i + 1]) ? NAN : x[z][i + 1] * f;
                            const uint32_t hi = e4m3x2(y0, y1);
                            const float2 u = from_e4m3x2(hi);
                            w[0] |= hi << (8 * i);
                            w[1] |= e4m3x2((y0 - u.x) * 16.0f,
                                           (y1 - u.y) * 16.0f)
                                    << (8 * i);
                        }
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const uint32_t at =
                                sQ + qs * C::kQ +
                                line_offset<D>(p * NV + g, (lane * V) >> 4) +
                                ((lane * V) & 15);
                            if (V == 4)
                                asm volatile("st.shared.u32 [%0], %1;" ::"r"(at),
                                             "r"(w[p])
                                             : "memory");
                            else
                                asm volatile("st.shared.u16 [%0], %1;" ::"r"(at),
                                             "h"((uint16_t)w[p])
                                             : "memory");
                        }
                        if (lane == 0) {
                            factors[qs][g] = pow2(e) * (c.scale * kLog2eF);
                            limits[qs][g] = lim[z];
                        }
                    }
                }
                if (!ok) break;
                if (warp == 6 && lane == 0) items[qs] = it;
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.q_full[qs]);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(
            kTaRegsSoft));
        // --------------------------------------------------------- softmax
        auto wait = [&](uint64_t *bar, uint32_t par, int site) {
            return __all_sync(0xffffffffu,
                              mbar_wait_or_abort(bar, par, abort, c.status,
                                                 site));
        };
        const int GT = c.G * c.T;
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        float acc[NV], l[NV], M[NV], al[NV], be[NV];
        Item it;
        int item = 0, t = 0, end = 0;
        bool ok = true;
        // acc of the current item takes tile j's O
        auto take = [&](int j) {
            const bool fine = wait(&bars.o_full[j & 1], (j >> 1) & 1, 190);
            tc_fence_after();
            float o[C::NP];
            uint32_t at = tm + lanes + 2 * C::N1 + (j & 1) * C::NO;
            if (D == 64 && warp >= 2) at += C::NP;
            tmem_read<C::NP>(at, o);
            tmem_wait_ld();
#pragma unroll
            for (int g = 0; g < NV; ++g)
                acc[g] = acc[g] * al[g] +
                         be[g] * (o[g] + 0.0625f * o[NV + g] +
                                  0.00390625f * o[2 * NV + g]);
            tc_fence_before();
            return fine;
        };
        for (int i = 0; i < count; ++i, ++t) {
            if (t == end) {
                const int qs = item & 1;
                ok = wait(&bars.q_full[qs], (item >> 1) & 1, 195) && ok;
                it = ok ? items[qs] : Item{};
                t = it.off;
                end = it.off + it.count;
                ++item;
#pragma unroll
                for (int g = 0; g < NV; ++g) {
                    acc[g] = l[g] = al[g] = be[g] = 0.0f;
                    M[g] = -INFINITY;
                }
            }
            const int vs = i % C::VS, b = i & 1;
            ok = wait(&bars.m_full[vs], (i / C::VS) & 1, 191) && ok;
            const int j = tid / c.ps, row = tid % c.ps;
            const TileMeta &m = meta[vs];
            const bool in = row < m.rows[j];
            const int pos = m.pos[j] + row;
            const float ks = m.ks[j], vrel = m.vs[j], vmax = m.vmax;
            ok = wait(&bars.s_full[b], (i >> 1) & 1, 192) && ok;
            tc_fence_after();
            float s[NV];
            {
                float x[2 * NV];
                tmem_read<2 * NV>(tm + lanes + b * C::N1, x);
                tmem_wait_ld();
                const bool all = pos <= it.len - it.n;
                const float *factor = factors[(item - 1) & 1];
                const int *limit = limits[(item - 1) & 1];
#pragma unroll
                for (int g = 0; g < NV; ++g) {
                    s[g] = (x[g] + 0.0625f * x[NV + g]) * (ks * factor[g]);
                    if (!in || (!all && pos > limit[g]))
                        s[g] = -INFINITY;
                }
            }
            if (t + 1 == end) {  // the queries may go
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.q_empty[(item - 1) & 1]);
            }
            if (A.scores) {
                const int w = t * kCacheTile + tid;
                if (w < it.walk) {
                    float *at = A.scores +
                                (((size_t)it.b * c.Hkv + it.h) * GT +
                                 it.col0) * A.slots + w;
#pragma unroll
                    for (int g = 0; g < NV; ++g)
                        if (g < it.cols) at[(size_t)g * A.slots] = s[g];
                }
            }
#pragma unroll
            for (int g = 0; g < NV; ++g) {
                const float x = redux_max(s[g]);
                if (lane == 0) red[b][g][warp] = x;
            }
            // also agrees on whether every wait of the four warps ended well
            ok = named_sync_and(1, 128, ok);
            if (!ok) break;
            // tile j's factors move on once its O is taken, which is after
            // this tile's weights: keep both
            float al2[NV], be2[NV];
            uint32_t hi[(NV + 1) / 2], mid[(NV + 1) / 2], lo[(NV + 1) / 2];
#pragma unroll
            for (int g = 0; g < NV; g += 2) {
                float y[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    y[k] = 0.0f;
                    if (g + k >= NV) continue;
                    const float4 w = *(const float4 *)red[b][g + k];
                    const float mt = fmaxf(fmaxf(w.x, w.y), fmaxf(w.z, w.w));
                    const float Mn = fmaxf(M[g + k], mt);
                    const float ref = mt == -INFINITY ? 0.0f : mt;
                    const float Mr = Mn == -INFINITY ? 0.0f : Mn;
                    const float p = ex2_approx(s[g + k] - ref);
                    const float a2 = ex2_approx(M[g + k] - Mr);
                    const float b2 = ex2_approx(mt - Mr);
                    M[g + k] = Mn;
                    l[g + k] = l[g + k] * a2 + b2 * p;
                    al2[g + k] = a2;
                    be2[g + k] = b2 * vmax * 0.00390625f;
                    y[k] = p * vrel * 256.0f;
                }
                const uint32_t h = e4m3x2(y[0], y[1]);
                const float2 u = from_e4m3x2(h);
                y[0] = (y[0] - u.x) * 16.0f;
                y[1] = (y[1] - u.y) * 16.0f;
                const uint32_t q = e4m3x2(y[0], y[1]);
                const float2 v = from_e4m3x2(q);
                hi[g / 2] = h;
                mid[g / 2] = q;
                lo[g / 2] = e4m3x2((y[0] - v.x) * 16.0f,
                                   (y[1] - v.y) * 16.0f);
            }
            {
                // the token's row of P: all hi, all mid, all lo
                const int pr = D == 128 ? tid : tid >> 1;
                const uint32_t at = sP + b * C::kP +
                                    (D == 128 ? 0u : (tid & 1) * 64u * C::W);
                uint32_t w[12];
#pragma unroll
                for (int k = 0; k < 12; ++k) w[k] = 0;
                if constexpr (NV == 1) {
                    w[0] = (hi[0] & 0xffu) | (mid[0] & 0xffu) << 8 |
                           (lo[0] & 0xffu) << 16;
                } else if constexpr (NV == 2) {
                    w[0] = hi[0] | mid[0] << 16;
                    w[1] = lo[0];
                } else {
#pragma unroll
                    for (int k = 0; k < NV / 4; ++k) {
                        w[k] = hi[2 * k] | hi[2 * k + 1] << 16;
                        w[NV / 4 + k] = mid[2 * k] | mid[2 * k + 1] << 16;
                        w[NV / 2 + k] = lo[2 * k] | lo[2 * k + 1] << 16;
                    }
                }
#pragma unroll
                for (int k = 0; k < (3 * NV + 15) / 16; ++k)
                    st_shared_v4(at + line_offset<C::W>(pr, k), w[4 * k],
                                 w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
            }
            if (!in) {
                // a row that does not count may hold anything, NaN too: its
                // weight is 0, its values have to be
                ok = mbar_wait_or_abort(&bars.v_full[vs], (i / C::VS) & 1,
                                        abort, c.status, 193) &&
                     ok;
                const int vr = D == 128 ? tid : tid >> 1;
                const int c0 = D == 128 ? 0 : (tid & 1) * 4;
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    st_shared_zero16(sV + vs * C::kTile +
                                     line_offset<128>(vr, c0 + k));
            }
            __syncwarp();
            fence_proxy_async_smem();
            tc_fence_before();
            mbar_arrive(&bars.p_ready[b]);
            if (t > it.off) ok = take(i - 1) && ok;
#pragma unroll
            for (int g = 0; g < NV; ++g) {
                al[g] = al2[g];
                be[g] = be2[g];
            }
            if (t + 1 < end) continue;

            // ------------------------------------------- the item's end
            ok = take(i) && ok;
#pragma unroll
            for (int g = 0; g < NV; ++g) {
                const float x = warp_sum(l[g]);
                if (lane == 0) fin[g][warp] = x;
                if (D == 64 && tid >= 64) half[g * 64 + tid - 64] = acc[g];
            }
            ok = named_sync_and(1, 128, ok);
            if (!ok) break;
            if (i + 1 == count && tid == 0) let_next_launch();
#pragma unroll
            for (int g = 0; g < NV; ++g) {
                if (g >= it.cols) break;
                const float4 w = *(const float4 *)fin[g];
                const float L = (w.x + w.y) + (w.z + w.w);
                const int col = it.col0 + g;
                float x = acc[g];
                if (D == 64 && tid < 64) x += half[g * 64 + tid];
                if (it.slot >= 0) {
                    float *at = piece(A, blockIdx.x, it.slot, g);
                    if (tid < D) at[tid] = x;
                    if (tid == 0) {
                        at[D] = M[g];
                        at[D + 1] = L;
                    }
                } else {
                    if (tid == 0)
                        store_lse(A, it.b, it.h, it.n, col, M[g], L);
                    if (tid < D && col % c.T < it.n)
                        store_o(A, query_row(A, it.b, it.h, col), tid,
                                L == 0.0f ? 0.0f : x / L);
                }
            }
            // fin and half are written again only behind the next tile's
            // barrier
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 5) tmem_dealloc(tm, C::kTmem);
}

template <int D, int NV>
cudaError_t launch_tc(const CacheAttn &A, cudaStream_t st) {
    using C = Cfg<D, NV>;
    const CacheView &c = A.c;
    const uint64_t rows = (uint64_t)c.num_pages * c.Hkv * c.ps;
    CUtensorMap tmK, tmV;
    cudaError_t e = make_tma_map_u8(&tmK, c.k, rows, D, c.ps);
    if (e == cudaSuccess)
        e = make_tma_map_u8(&tmV, c.v, D == 128 ? rows : rows / 2, 128,
                            D == 128 ? c.ps : c.ps / 2);
    if (e != cudaSuccess) return e;
    return launch_after(k_cache_attn_tc<D, NV>, dim3(A.ctas), kTaThreads,
                        C::kSmem + sizeof(int) * (c.B + 1), st, tmK, tmV, A);
}

template <int D>
cudaError_t launch_cols(const CacheAttn &A, cudaStream_t st) {
    switch (A.cols) {
        case 1: return launch_tc<D, 1>(A, st);
        case 2: return launch_tc<D, 2>(A, st);
        case 4: return launch_tc<D, 4>(A, st);
        case 8: return launch_tc<D, 8>(A, st);
        default: return launch_tc<D, 16>(A, st);
    }
}

}  // namespace

bool cache_attn_tc_supported(const CacheView &c) {
    return c.dtype == ELSAA_BF16 && (c.d == 64 || c.d == 128);
}

cudaError_t launch_cache_attn_tc(const CacheAttn &A, cudaStream_t st) {
    return A.c.d == 64 ? launch_cols<64>(A, st) : launch_cols<128>(A, st);
}

}  // namespace elsaa
