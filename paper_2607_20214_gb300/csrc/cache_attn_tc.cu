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
// softmax weight is rounded to fp16, whose 11 bits (2^-11 relative at most,
// and 2^-33 of the step's largest) three e4m3 numbers hold exactly, down to
// 2^-26 of the largest: a bf16 weight would have 8 bits. A step's weights are
// relative to the step's own maximum, so that a flat tail behind one large
// score keeps its bits; sums (of the weights before rounding) and O, in
// registers, are rescaled in fp32.
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
//
// Measured with the merge: 16 sequences, 8 heads of 128, 4 queries a head,
// 65536 tokens 324 to 328 us (6.6 TB/s, 0.97 to 0.98 of a copy); 2 x 16 heads
// of 16384 tokens 30 us, of which 24 at 5.6 TB/s, the rest its start (lengths,
// table, first tile: 5000 cycles) and the merge. With more columns a tile takes
// longer (8 sequences, 8 heads, 8192 tokens: 1 column 31 us, 8 33, 16 40, about
// 2000 cycles a tile) without a unit being full: with 16 columns 24 % of the
// issue slots, 18 % of the ALU, 42 % of DRAM, 6 % of the tensor pipe. Its warps
// wait, for loads and at barriers above all.
#include <limits.h>

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

constexpr int kSub = 2;  // tiles of a softmax step

template <int D, int NV>
struct Cfg {
    static constexpr int N1 = 2 * NV < 16 ? 16 : 2 * NV;  // columns of S
    static constexpr int NP = (3 * NV + 15) / 16 * 16;    // of one P product
    static constexpr int NO = D == 128 ? NP : 2 * NP;     // of O
    static constexpr int W = NP <= 32 ? 32 : 64;  // bytes of a token's P row
    // K is free again as soon as S is made, V only when O is
    static constexpr int KS = D == 64 ? 4 : 2;
    static constexpr int VS = D == 64 ? (NV < 16 ? 8 : 6) : (NV < 16 ? 4 : 3);
    // a tile's pages and scales are written before its V buffer is waited
    // for: by then tile - 1 - VS is read
    static constexpr int MS = VS + 1;
    static constexpr uint32_t kTile = kCacheTile * D;
    static constexpr uint32_t kQ = N1 * D;
    static constexpr uint32_t kP = kCacheTile * W;
    static constexpr uint32_t kSmem =
        1024 + (KS + VS) * kTile + 2 * kQ + kSub * kP;
    static constexpr uint32_t kCols = 2 * kSub * N1 + NO;
    static constexpr uint32_t kTmem = kCols <= 128 ? 128 : 256;
    static_assert(kCols <= 256, "two CTAs share tensor memory");
    static_assert(VS > kSub, "the next step's V has to fit");
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

// Largest of the warp's values, in every lane.
__device__ __forceinline__ float redux_max(float x) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

// Sums of NV columns over the warp: in lane i, column i / (32 / NV)'s. Every
// exchange halves the columns that a lane still holds.
template <int NV>
__device__ __forceinline__ float column_sums(const float *x) {
    float v[NV];
#pragma unroll
    for (int g = 0; g < NV; ++g) v[g] = x[g];
    const int lane = threadIdx.x & 31;
    int o = 16;
#pragma unroll
    for (int n = NV / 2; n >= 1; n /= 2, o /= 2) {
        const bool up = (lane & o) != 0;
#pragma unroll
        for (int g = 0; g < n; ++g) {
            const float mine = up ? v[g + n] : v[g];
            const float his = up ? v[g] : v[g + n];
            v[g] = mine + __shfl_xor_sync(0xffffffffu, his, o);
        }
    }
#pragma unroll
    for (; o >= 1; o /= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
    return v[0];
}

// fp16 pairs (low half first) and their e4m3 roundings.
__device__ __forceinline__ uint32_t e4m3x2_of(uint32_t h) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(h));
    return r;
}
__device__ __forceinline__ uint32_t f16x2_of(uint32_t e) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)e));
    return r;
}
// 16 (a - b), exact for a >= 0 and b its e4m3 rounding: a has 11 bits, b the
// first four of them.
__device__ __forceinline__ uint32_t rest16(uint32_t a, uint32_t b) {
    uint32_t x, r;
    constexpr uint32_t k16 = 0x4c004c00u, km16 = 0xcc00cc00u;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(x) : "r"(a), "r"(k16));
    asm("fma.rn.f16x2 %0, %1, %2, %3;"
        : "=r"(r)
        : "r"(b), "r"(km16), "r"(x));
    return r;
}

// 0x80 in every byte whose low 7 bits are all set: e4m3's NaN.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
    return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t at) {
    uint4 r;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
                 : "r"(at)
                 : "memory");
    return r;
}
// The NaN codes among 16 in shared memory become 0; their channels' `from`
// falls to pos.
static __device__ __noinline__ void drop_nan(uint32_t at, int *from,
                                             int pos) {
    const uint4 q = ld_shared_v4(at);
    uint32_t w[4] = {q.x, q.y, q.z, q.w};
    for (int i = 0; i < 4; ++i) {
        const uint32_t bad = nan_bytes(w[i]);
        for (int k = 0; k < 4; ++k)
            if (bad >> (8 * k) & 0x80u) {
                w[i] &= ~(0xffu << (8 * k));
                atomicMin(from + 4 * i + k, pos);
            }
    }
    st_shared_v4(at, w[0], w[1], w[2], w[3]);
}

// The pages of one tile, written by the producer.
struct TileMeta {
    float ks[kMaxPagesPerTile];   // key scale
    float vs[kMaxPagesPerTile];   // value scale
    int pos[kMaxPagesPerTile];    // first position
    int rows[kMaxPagesPerTile];   // rows that count
    float vmax;                   // largest value scale
};

struct Bars {
    uint64_t k_full[4], k_empty[4], v_full[8], v_empty[8], m_full[9];
    uint64_t s_full[2], p_ready, o_full, q_full[2], q_empty[2], drain;
};

template <int D, int NV>
__global__ void __launch_bounds__(kTaThreads, 2)
    k_cache_attn_tc(const __grid_constant__ CUtensorMap tmK,
                    const __grid_constant__ CUtensorMap tmV,
                    const __grid_constant__ CacheAttn A) {
    using C = Cfg<D, NV>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Bars bars;
    __shared__ TileMeta meta[C::MS];
    __shared__ Item items[2];
    __shared__ Seq near[kNearSeqs];
    __shared__ float factors[2][NV];  // of an item's columns' scores
    __shared__ int limits[2][NV];     // last positions that they see
    __shared__ uint32_t tbase;
    __shared__ int abort_flag;
    // per step parity: every warp's maxima, and for every warp a column's
    // numbers: minus its reference, score factor, factor of the sums so far,
    // factor of the step's
    __shared__ float red[2][4][NV];
    __shared__ __align__(16) float stat[2][4][4][NV];
    __shared__ float4 fin[2][NV];  // sums of the four warps' tokens
    // of an item, by channel: the first new token whose value is no number
    __shared__ int nan_from[D];
    volatile int *abort = &abort_flag;
    const CacheView &c = A.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t sK = base, sV = sK + C::KS * C::kTile;
    const uint32_t sQ = sV + C::VS * C::kTile, sP = sQ + 2 * C::kQ;

    // set up while the kernel before ends
    if (warp == 5) tmem_alloc(&tbase, C::kTmem);
    if (tid == 0) {
        for (int s = 0; s < C::KS; ++s) {
            mbar_init(&bars.k_full[s], 1);
            mbar_init(&bars.k_empty[s], 1);
        }
        for (int s = 0; s < C::VS; ++s) {
            mbar_init(&bars.v_full[s], 1);
            mbar_init(&bars.v_empty[s], 1);
        }
        for (int s = 0; s < C::MS; ++s) mbar_init(&bars.m_full[s], 1);
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars.s_full[s], 1);
            mbar_init(&bars.q_full[s], 2);   // the query warps
            mbar_init(&bars.q_empty[s], 5);  // products, four softmax warps
        }
        mbar_init(&bars.p_ready, 128);
        mbar_init(&bars.o_full, 1);
        mbar_init(&bars.drain, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tbase;
    wait_for_stream();
    let_next_launch();
    Seq own;
    const Start first = divide<kTaThreads>(A, near, own);
    const int count = first.count;

    if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(
            kTaRegsOther));
        auto wait = [&](uint64_t *bar, uint32_t par, int site) {
            return __all_sync(0xffffffffu,
                              mbar_wait_or_abort(bar, par, abort, c.status,
                                                 site));
        };
        if (warp == 4) {
            // -------------------------------------------- pages and scales
            // A batch is the next 32 pages of an item, a page a lane, which
            // loads it; the next batch's table entries and scales are asked
            // for as soon as this one's first tile is on its way.
            const int lp = __ffs(kCacheTile / c.ps) - 1;  // pages of a tile
            const int pt = 1 << lp, slot = lane & (pt - 1);
            struct Page {
                int id, pos, rows;
                float ks, vs;
            };
            auto fetch = [&](const Item &it, int tile) {
                Page g = {-1, 0, 0, 0.0f, 0.0f};
                const int e = (tile << lp) + lane;
                int p = -1;
                if ((long)e * c.ps < it.walk)
                    p = A.pages ? A.pages[((size_t)it.b * c.Hkv + it.h) *
                                              A.n_sel + e]
                                : e;
                if (p >= 0 && p < c.max_pages) {
                    g.pos = p * c.ps;
                    g.rows = min(it.len - g.pos, c.ps);
                    if (g.rows > 0) g.id = page_id(c, it.b, p);
                }
                if (g.id >= 0) {
                    const int ph = g.id * c.Hkv + it.h;  // fits: the host's
                    g.ks = c.ks[ph];                     // check
                    g.vs = c.vs[ph];
                } else {
                    g.rows = 0;
                }
                return g;
            };
            Walk walk(first, near, own);
            Item it = {}, nit = {};
            Page page = {}, next = {};
            int tile = 0, ntile = 0;
            bool ok = true;
            int kn = 0, vn = 0;  // loads issued
            if (count > 0) {
                it = walk.next(A);
                tile = it.off;
                page = fetch(it, tile);
            }
            for (int i = 0; i < count && ok;) {
                const int nt = min(32 >> lp, it.off + it.count - tile);
                // bytes to come of the lane's tile
                const uint32_t live =
                    __ballot_sync(0xffffffffu, page.id >= 0) >>
                    (lane & ~(pt - 1));
                const uint32_t bytes =
                    __popc(live & ((1u << pt) - 1)) * c.ps * D;
                const int row = (page.id * c.Hkv + it.h) * c.ps;
                const uint32_t to = slot * c.ps * D;
                // tile k of the batch into its buffers
                auto load_k = [&](int k, int ks) {
                    if (lane >> lp == k) {
                        if (slot == 0) mbar_expect_tx(&bars.k_full[ks], bytes);
                        if (page.id >= 0)
                            tma_load_2d(sK + ks * C::kTile + to, &tmK, 0, row,
                                        &bars.k_full[ks]);
                    }
                    ++kn;
                };
                // the first tiles' K need not wait for the scales (12 heads of
                // 700 tokens, d = 64: 8.8 -> 8.4 us; with V's as well long
                // sequences lost that again)
                if (i == 0)
                    for (int k = 0; k < min(nt, C::KS); ++k) load_k(k, k);
                // largest value scale of the lane's tile
                float vmax = page.vs;
                for (int o = 1; o < pt; o <<= 1)
                    vmax = fmaxf(vmax, __shfl_xor_sync(0xffffffffu, vmax, o));
                for (int k = 0; k < nt; ++k, ++i) {
                    const int ks = i % C::KS, vs = i % C::VS, ms = i % C::MS;
                    if (i >= kn) {
                        if (i >= C::KS)
                            ok = wait(&bars.k_empty[ks], (i / C::KS - 1) & 1,
                                      180);
                        if (!ok) break;
                        load_k(k, ks);
                    }
                    if (lane >> lp == k) {
                        TileMeta &m = meta[ms];
                        m.ks[slot] = page.ks;
                        m.vs[slot] = page.vs;
                        m.pos[slot] = page.pos;
                        m.rows[slot] = page.rows;
                        m.vmax = vmax;
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.m_full[ms]);
                    if (i >= C::VS)
                        ok = wait(&bars.v_empty[vs], (i / C::VS - 1) & 1, 181);
                    if (!ok) break;
                    if (lane >> lp == k) {
                        if (slot == 0) mbar_expect_tx(&bars.v_full[vs], bytes);
                        if (page.id >= 0)
                            tma_load_2d(sV + vs * C::kTile + to, &tmV, 0,
                                        D == 128 ? row : row / 2,
                                        &bars.v_full[vs]);
                    }
                    ++vn;
                    if (k == 0) {
                        nit = it;
                        ntile = tile + nt;
                        if (ntile == it.off + it.count && walk.left > 0) {
                            nit = walk.next(A);
                            ntile = nit.off;
                        }
                        if (i + nt < count) next = fetch(nit, ntile);
                    }
                }
                it = nit;
                tile = ntile;
                page = next;
            }
            __syncwarp();
            // whatever was asked for has arrived before the CTA ends
            for (int j = max(0, kn - C::KS); j < kn; ++j)
                mbar_wait(&bars.k_full[j % C::KS], (j / C::KS) & 1, c.status,
                          182);
            for (int j = max(0, vn - C::VS); j < vn; ++j)
                mbar_wait(&bars.v_full[j % C::VS], (j / C::VS) & 1, c.status,
                          183);
        } else if (warp == 5) {
            // ---------------------------------------------------- products
            const bool el = elect_one();
            const uint32_t id_s = idesc_e4m3(128, C::N1, false, false);
            const uint32_t id_o = idesc_e4m3(128, C::NP, true, true);
            const uint32_t o = tm + 2 * kSub * C::N1;
            // O of step j: `n` tiles from tile u on
            auto values = [&](int j, int u, int n) {
                for (int x = 0; x < n; ++x)
                    if (!wait(&bars.v_full[(u + x) % C::VS],
                              ((u + x) / C::VS) & 1, 185))
                        return false;
                if (!wait(&bars.p_ready, j & 1, 186)) return false;
                tc_fence_after();
                if (el) {
                    for (int x = 0; x < n; ++x) {
                        const int vs = (u + x) % C::VS;
                        const uint64_t dV = line_desc(sV + vs * C::kTile, 128);
                        const uint64_t dP = line_desc(sP + x * C::kP, C::W);
                        if (D == 128) {
#pragma unroll
                            for (int y = 0; y < 4; ++y)
                                mma_e4m3(o, desc_at(dV, y * 4096),
                                         desc_at(dP, y * 32 * C::W), id_o,
                                         x + y > 0);
                        } else {
#pragma unroll
                            for (int par = 0; par < 2; ++par)
#pragma unroll
                                for (int y = 0; y < 2; ++y)
                                    mma_e4m3(o + par * C::NP,
                                             desc_at(dV, y * 4096),
                                             desc_at(dP, (par * 64 + y * 32) *
                                                             C::W),
                                             id_o, x + y > 0);
                        }
                    }
                    mma_commit(&bars.o_full);
                    for (int x = 0; x < n; ++x)
                        mma_commit(&bars.v_empty[(u + x) % C::VS]);
                }
                __syncwarp();
                return true;
            };
            bool ok = true;
            int item = 0, left = 0;  // tiles of the item
            int u0 = 0, n0 = 0;      // tiles of the step before
            uint64_t dQ = 0;
            int i = 0;
            for (int u = 0; u < count; ++i) {
                if (left == 0) {
                    ok = wait(&bars.q_full[item & 1], (item >> 1) & 1, 187);
                    if (!ok) break;
                    left = items[item & 1].count;
                    dQ = line_desc(sQ + (item & 1) * C::kQ, D);
                    ++item;
                }
                const int n = min(left, kSub);
                left -= n;
                for (int x = 0; x < n && ok; ++x) {
                    const int ks = (u + x) % C::KS;
                    ok = wait(&bars.k_full[ks], ((u + x) / C::KS) & 1, 188);
                    if (!ok) break;
                    tc_fence_after();
                    if (el) {
                        const uint64_t dK = line_desc(sK + ks * C::kTile, D);
                        const uint32_t s = tm + ((i & 1) * kSub + x) * C::N1;
#pragma unroll
                        for (int y = 0; y < D / 32; ++y)
                            mma_e4m3(s, desc_at(dK, y * 32),
                                     desc_at(dQ, y * 32), id_s, y > 0);
                        mma_commit(&bars.k_empty[ks]);
                        if (x + 1 == n) {
                            mma_commit(&bars.s_full[i & 1]);
                            if (left == 0)
                                mma_commit(&bars.q_empty[(item - 1) & 1]);
                        }
                    }
                    __syncwarp();
                }
                if (ok && i > 0) ok = values(i - 1, u0, n0);
                if (!ok) break;
                u0 = u;
                n0 = n;
                u += n;
            }
            if (ok && count > 0) values(i - 1, u0, n0);
            // every product is complete before tensor memory is given back
            if (el) mma_commit(&bars.drain);
            mbar_wait(&bars.drain, 0, c.status, 189);
            __syncwarp();
        } else {
            // ----------------------------------------------------- queries
            // D / 16 lanes a column, 16 elements each: a line's 16-byte chunk
            constexpr int LPC = D / 16, CPW = 32 / LPC;
            const int ch = lane % LPC;
            Walk walk(first, near, own);
            bool ok = true;
            for (int k = 0; walk.left > 0; ++k) {
                const Item it = walk.next(A);
                const int qs = k & 1;
#pragma unroll 1
                for (int g0 = 0; g0 < NV; g0 += 2 * CPW) {
                    const int g = g0 + (warp - 6) * CPW + lane / LPC;
                    const int lim =
                        g < it.cols
                            ? last_seen(A, it.len, it.n, it.col0 + g)
                            : -1;
                    float x[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = 0.0f;
                    if (lim >= 0) {
                        const __nv_bfloat16 *src =
                            (const __nv_bfloat16 *)A.q +
                            query_row(A, it.b, it.h, it.col0 + g) * D +
                            ch * 16;
                        load8(src, x);
                        load8(src + 8, x + 8);
                    }
                    // the first columns are read before the buffer is free
                    if (g0 == 0 && k >= 2)
                        ok = wait(&bars.q_empty[qs], ((k >> 1) - 1) & 1, 184);
                    if (!ok) break;
                    float amax = 0.0f;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        amax = fmaxf(amax, magnitude(x[i]));
#pragma unroll
                    for (int o = 1; o < LPC; o <<= 1)
                        amax = fmaxf(amax,
                                     __shfl_xor_sync(0xffffffffu, amax, o));
                    const int e = least_exponent(amax, 0x600000u, 8, -100,
                                                 kCacheExpHigh);
                    const float f = pow2(-e);
                    uint32_t hi[4] = {0, 0, 0, 0}, lo[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        // an infinity has no split: it counts as NaN
                        const float y0 = isinf(x[i]) ? NAN : x[i] * f;
                        const float y1 = isinf(x[i + 1]) ? NAN : x[i + 1] * f;
                        const uint32_t h = e4m3x2(y0, y1);
                        const float2 z = from_e4m3x2(h);
                        hi[i / 4] |= h << (8 * (i & 3));
                        lo[i / 4] |= e4m3x2((y0 - z.x) * 16.0f,
                                            (y1 - z.y) * 16.0f)
                                     << (8 * (i & 3));
                    }
                    if (g < NV) {
                        const uint32_t q = sQ + qs * C::kQ;
                        st_shared_v4(q + line_offset<D>(g, ch), hi[0], hi[1],
                                     hi[2], hi[3]);
                        st_shared_v4(q + line_offset<D>(NV + g, ch), lo[0],
                                     lo[1], lo[2], lo[3]);
                        if (ch == 0) {
                            // A masked score is -inf in any unit, and
                            // -inf times 0 is no number: a factor below
                            // fp32's least, of a small scale, becomes that
                            // (2^-149 of a score of less than 2^128).
                            factors[qs][g] = fmaxf(
                                pow2(e) * (c.scale * kLog2eF), 1.4e-45f);
                            limits[qs][g] = lim;
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
        // A step is up to kSub tiles of an item: a thread has a token of each,
        // so that what a step costs whatever it holds (waits, the maximum
        // over the warps, O's way back) is paid once.
        auto wait = [&](uint64_t *bar, uint32_t par, int site) {
            return __all_sync(0xffffffffu,
                              mbar_wait_or_abort(bar, par, abort, c.status,
                                                 site));
        };
        const int GT = c.G * c.T;
        const int shift = __ffs(c.ps) - 1;
        const int slot = tid >> shift, row = tid & (c.ps - 1);
        const uint32_t lanes = (uint32_t)(warp * 32) << 16;
        constexpr int NH = (NV + 1) / 2;  // columns in pairs
        constexpr int NW = 4 * ((3 * NV + 15) / 16);  // words of a P row
        float2 acc[NH], l[NH];
        float M = -INFINITY;      // lane g: of column g, in the scores' unit
        Item it = {}, last = {};  // this step's, the unfinished one before
        float lastM = 0.0f, factor = 0.0f;
        int item = 0, t = 0, end = 0;
        bool ok = true, fine = count > 0;
        if (tid < D) nan_from[tid] = INT_MAX;
#pragma unroll
        for (int g = 0; g < NH; ++g) acc[g] = l[g] = make_float2(0.0f, 0.0f);
        // column pair g of a row of stat
        auto pair = [&](const float *p, int g) {
            return NV == 1 ? make_float2(p[0], 0.0f)
                           : *(const float2 *)(p + 2 * g);
        };
        // acc takes step j's O
        auto take = [&](int j) {
            const bool done = wait(&bars.o_full, j & 1, 190);
            tc_fence_after();
            float o[C::NP];
            uint32_t at = tm + lanes + 2 * kSub * C::N1;
            if (D == 64 && warp >= 2) at += C::NP;
            tmem_read<C::NP>(at, o);
            tmem_wait_ld();
            const float(*f)[NV] = stat[j & 1][warp];
            const float2 c1 = make_float2(0.0625f, 0.0625f);
            const float2 c2 = make_float2(0.00390625f, 0.00390625f);
#pragma unroll
            for (int g = 0; g < NH; ++g) {
                auto at = [&](int k) {
                    return make_float2(o[k * NV + 2 * g],
                                       NV == 1 ? 0.0f : o[k * NV + 2 * g + 1]);
                };
                const float2 x = fma2(c2, at(2), fma2(c1, at(1), at(0)));
                acc[g] = fma2(pair(f[3], g), x, mul2(acc[g], pair(f[2], g)));
            }
            tc_fence_before();
            return done;
        };
        // the sums of a finished item, where every warp finds them behind the
        // next barrier
        auto leave = [&](int k) {
            const float x = column_sums<NV>((const float *)l);
            if (lane % (32 / NV) == 0)
                ((float *)&fin[k & 1][lane / (32 / NV)])[warp] = x;
#pragma unroll
            for (int g = 0; g < NH; ++g) l[g] = make_float2(0.0f, 0.0f);
            last = it;
            lastM = M * factor;
            M = -INFINITY;
        };
        // Item k is complete in acc: it leaves through the P buffer, which no
        // product reads now, as whole rows.
        auto finish = [&](int k) {
            float *buf = (float *)(smem_raw + (sP - smem_u32(smem_raw)));
#pragma unroll
            for (int g = 0; g < NV; ++g)
                buf[g * 128 + tid] = g & 1 ? acc[g / 2].y : acc[g / 2].x;
#pragma unroll
            for (int g = 0; g < NH; ++g) acc[g] = make_float2(0.0f, 0.0f);
            if (tid < D && nan_from[tid] != INT_MAX) {
                for (int g = 0; g < last.cols; ++g)
                    if (nan_from[tid] <=
                        last_seen(A, last.len, last.n, last.col0 + g))
                        buf[g * 128 + tid] = NAN;
                nan_from[tid] = INT_MAX;
            }
            named_sync(1, 128);
            const size_t r0 = query_row(A, last.b, last.h, last.col0);
#pragma unroll 1
            for (int e = tid; e < last.cols * (D / 4); e += 128) {
                const int g = e / (D / 4), ch = e % (D / 4) * 4;
                float4 x = *(const float4 *)(buf + g * 128 + ch);
                if (D == 64) {
                    const float4 y = *(const float4 *)(buf + g * 128 + 64 + ch);
                    x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
                }
                if (last.slot >= 0) {
                    float *at = piece(A, blockIdx.x, last.slot, g) + ch;
                    *(float2 *)at = make_float2(x.x, x.y);
                    *(float2 *)(at + 2) = make_float2(x.z, x.w);
                } else if (token_of(A, last.col0 + g) < last.n) {
                    const float4 w = fin[k & 1][g];
                    const float L = (w.x + w.y) + (w.z + w.w);
                    const float f = L == 0.0f ? 0.0f : 1.0f / L;
                    *(uint2 *)((__nv_bfloat16 *)A.o + (r0 + g) * D + ch) =
                        make_uint2(pack_bf16x2(x.x * f, x.y * f),
                                   pack_bf16x2(x.z * f, x.w * f));
                }
            }
            if (tid < last.cols) {  // column `tid`
                const float4 w = fin[k & 1][tid];
                const float L = (w.x + w.y) + (w.z + w.w);
                if (last.slot >= 0) {
                    float *at = piece(A, blockIdx.x, last.slot, tid);
                    at[D] = lastM;
                    at[D + 1] = L;
                } else {
                    store_lse(A, last.b, last.h, last.n, last.col0 + tid,
                              lastM, L);
                }
            }
            named_sync(1, 128);
        };
        int i = 0;
        for (int u = 0; u < count; ++i) {
            const bool begins = t == end;
            if (begins) {
                if (i > 0) leave(item - 1);
                const int qs = item & 1;
                ok = wait(&bars.q_full[qs], (item >> 1) & 1, 195) && ok;
                it = ok ? items[qs] : Item{};
                factor = lane < NV ? factors[qs][lane] : 0.0f;
                t = it.off;
                end = it.off + it.count;
                ++item;
            }
            // a second tile that the item does not have counts as one without
            // rows
            const int n = min(end - t, kSub), b = i & 1;
            float vrel[kSub], ks[kSub], vmax = 0.0f;
            bool in[kSub];
            int pos[kSub];
#pragma unroll
            for (int x = 0; x < kSub; ++x) {
                in[x] = false;
                ks[x] = vrel[x] = 0.0f;
                pos[x] = 0;
                if (x < n) {
                    const int ms = (u + x) % C::MS;
                    ok = wait(&bars.m_full[ms], ((u + x) / C::MS) & 1, 191) &&
                         ok;
                    const TileMeta &m = meta[ms];
                    in[x] = row < m.rows[slot];
                    pos[x] = m.pos[slot] + row;
                    ks[x] = m.ks[slot];
                    vrel[x] = m.vs[slot];
                    vmax = fmaxf(vmax, m.vmax);
                }
            }
            const bool free = in[0] && in[1] &&
                              max(pos[0], pos[1]) <= it.len - it.n;
            ok = wait(&bars.s_full[b], (i >> 1) & 1, 192) && ok;
            tc_fence_after();
            float2 s[kSub][NH];
#pragma unroll
            for (int x = 0; x < kSub; ++x) {
                float y[2 * NV];
                tmem_read<2 * NV>(tm + lanes + (b * kSub + x) * C::N1, y);
                tmem_wait_ld();
                const float2 c1 = make_float2(0.0625f, 0.0625f);
                const float2 kk = make_float2(ks[x], ks[x]);
#pragma unroll
                for (int g = 0; g < NH; ++g) {
                    const float2 hi = make_float2(y[2 * g],
                                                  NV == 1 ? 0.0f
                                                          : y[2 * g + 1]);
                    const float2 lo = make_float2(y[NV + 2 * g],
                                                  NV == 1 ? 0.0f
                                                          : y[NV + 2 * g + 1]);
                    s[x][g] = mul2(fma2(c1, lo, hi), kk);
                }
            }
            tc_fence_before();
            if (!__all_sync(0xffffffffu, free)) {
                // rows that do not count, keys behind a query
                const int *limit = limits[(item - 1) & 1];
#pragma unroll
                for (int x = 0; x < kSub; ++x)
#pragma unroll
                    for (int g = 0; g < NV; ++g)
                        if (!in[x] || (pos[x] > it.len - it.n &&
                                       pos[x] > limit[g])) {
                            if (g & 1)
                                s[x][g / 2].y = -INFINITY;
                            else
                                s[x][g / 2].x = -INFINITY;
                        }
            }
            if (A.scores) {
#pragma unroll
                for (int x = 0; x < kSub; ++x) {
                    const int w = (t + x) * kCacheTile + tid;
                    if (x < n && w < it.walk) {
                        float *at = A.scores +
                                    (((size_t)it.b * c.Hkv + it.h) * GT +
                                     it.col0) * A.slots + w;
#pragma unroll
                        for (int g = 0; g < NV; ++g)
                            if (g < it.cols)
                                at[(size_t)g * A.slots] =
                                    (g & 1 ? s[x][g / 2].y : s[x][g / 2].x) *
                                    factors[(item - 1) & 1][g];
                    }
                }
            }
            if (t + n == end) {  // the queries may go
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.q_empty[(item - 1) & 1]);
            }
            // lane g keeps column g's maximum
            float top = -INFINITY;
#pragma unroll
            for (int g = 0; g < NV; ++g) {
                const float x =
                    redux_max(g & 1 ? fmaxf(s[0][g / 2].y, s[1][g / 2].y)
                                    : fmaxf(s[0][g / 2].x, s[1][g / 2].x));
                if (lane == g) top = x;
            }
            if (lane < NV) red[b][warp][lane] = top;
            // also agrees on whether every wait of the four warps ended well
            fine = named_sync_and(1, 128, ok);
            if (!fine) break;
            if (lane < NV) {
                const float mt = fmaxf(fmaxf(red[b][0][lane], red[b][1][lane]),
                                       fmaxf(red[b][2][lane], red[b][3][lane]));
                const float Mn = fmaxf(M, mt);
                const float Mr = Mn == -INFINITY ? 0.0f : Mn;
                float(*f)[NV] = stat[b][warp];
                f[0][lane] = mt == -INFINITY ? 0.0f : -mt * factor;
                f[1][lane] = factor;
                f[2][lane] = ex2_approx((M - Mr) * factor);
                f[3][lane] = ex2_approx((mt - Mr) * factor) * vmax *
                             0.00390625f;
                M = Mn;
            }
            __syncwarp();
            const float inv = vmax > 0.0f ? 256.0f / vmax : 0.0f;
            const float2 inv2 = make_float2(inv, inv);
            uint32_t w[kSub][NW];
#pragma unroll
            for (int x = 0; x < kSub; ++x) {
                vrel[x] *= inv;
#pragma unroll
                for (int k = 0; k < NW; ++k) w[x][k] = 0;
            }
#pragma unroll
            for (int g = 0; g < NH; ++g) {
                const float(*f)[NV] = stat[b][warp];
                const float2 nref = pair(f[0], g), fac = pair(f[1], g);
                float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
                for (int x = 0; x < kSub; ++x) {
                    float2 p = fma2(s[x][g], fac, nref);
                    p.x = ex2_approx(p.x);
                    if (NV > 1) p.y = ex2_approx(p.y);
                    sum = add2(sum, p);
                    p = mul2(p, make_float2(vrel[x], vrel[x]));
                    // the pieces of the weights, hi, mid, lo
                    uint32_t r = pack_f16x2(p.x, p.y);
#pragma unroll
                    for (int k = 0; k < 3; ++k) {
                        const uint32_t e = e4m3x2_of(r);
                        if (k < 2) r = rest16(r, f16x2_of(e));
                        if constexpr (NV == 1)
                            w[x][0] |= (e & 0xffu) << (8 * k);
                        else
                            w[x][(k * NV + 2 * g) / 4] |=
                                e << (8 * ((k * NV + 2 * g) & 3));
                    }
                }
                l[g] = fma2(pair(f[3], g), mul2(sum, inv2),
                            mul2(l[g], pair(f[2], g)));
            }
            // the O of the step before; its products have read P by then
            if (i > 0) ok = take(i - 1) && ok;
            if (begins && i > 0) finish(item - 2);
            const int pr = D == 128 ? tid : tid >> 1;
#pragma unroll
            for (int x = 0; x < kSub; ++x) {
                const uint32_t at = sP + x * C::kP +
                                    (D == 128 ? 0u : (tid & 1) * 64u * C::W);
#pragma unroll
                for (int k = 0; k < NW / 4; ++k)
                    st_shared_v4(at + line_offset<C::W>(pr, k), w[x][4 * k],
                                 w[x][4 * k + 1], w[x][4 * k + 2],
                                 w[x][4 * k + 3]);
                if (x < n && (!in[x] || pos[x] > it.len - it.n)) {
                    // A row that does not count may hold anything, NaN too:
                    // its weight is 0, its values have to be. A new token's
                    // weight is 0 for the queries before it: values that are
                    // no numbers become 0 and are kept for the others.
                    const int vs = (u + x) % C::VS;
                    const bool there = mbar_wait_or_abort(
                        &bars.v_full[vs], ((u + x) / C::VS) & 1, abort,
                        c.status, 193);
                    ok = there && ok;
                    const uint32_t line = sV + vs * C::kTile;
                    const int c0 = D == 128 ? 0 : (tid & 1) * 4;
                    if (!in[x]) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
                            st_shared_zero16(line +
                                             line_offset<128>(pr, c0 + k));
                    } else if (there) {
                        uint32_t bad = 0;
#pragma unroll 4
                        for (int k = 0; k < D / 16; ++k) {
                            const uint4 q = ld_shared_v4(
                                line + line_offset<128>(pr, c0 + k));
                            bad |= nan_bytes(q.x) | nan_bytes(q.y) |
                                   nan_bytes(q.z) | nan_bytes(q.w);
                        }
                        for (int k = 0; bad != 0 && k < D / 16; ++k)
                            drop_nan(line + line_offset<128>(pr, c0 + k),
                                     nan_from + 16 * k, pos[x]);
                    }
                }
            }
            __syncwarp();
            fence_proxy_async_smem();
            tc_fence_before();
            mbar_arrive(&bars.p_ready);
            t += n;
            u += n;
        }
        if (fine) {
            ok = take(i - 1) && ok;
            leave(item - 1);
            ok = named_sync_and(1, 128, ok);
            if (ok) finish(item - 1);
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
    return launch_cache<k_cache_attn_tc<D, NV>>(
        dim3(A.ctas), kTaThreads, C::kSmem, C::kSmem, 1, st, tmK, tmV, A);
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

// Whatever the size: the CUDA cores are faster in the smallest caches only
// (bf16, a head of 64 with 16 tokens: 4.8 us against 5.3), where setting up
// tensor memory and barriers shows; 8 heads of 40 tokens take 5.3 us here and
// 5.9 there, 2 sequences with 8 heads of 300 tokens 6.7 and 9.7, with 4 queries
// a head 7.0 and 14.7, 16 sequences of 4096 tokens 30 and 42.
bool cache_attn_tc_supported(const CacheView &c) {
    return c.dtype == ELSAA_BF16 && (c.d == 64 || c.d == 128);
}

cudaError_t launch_cache_attn_tc(const CacheAttn &A, cudaStream_t st) {
    return A.c.d == 64 ? launch_cols<64>(A, st) : launch_cols<128>(A, st);
}

}  // namespace elsaa
