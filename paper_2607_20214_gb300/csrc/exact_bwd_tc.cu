// The backward pass of exact attention on the tensor cores
// (include/elsaa_exact.h), bf16. With s = scale Q K^T, P = exp(s - lse),
// D_i = <dO_i, O_i>, dS = P (dO V^T - D):
//     dV = P^T dO,  dK = scale dS^T Q,  dQ = scale dS K.
// Two kernels compute P and dS again, each for sums of its own: k_exact_dq_tc
// holds 128 query rows and walks the keys, k_exact_dkv_tc holds 128 keys and
// walks the query rows of every head that reads them. That is seven products
// instead of five, but every sum stays in tensor memory, in one order: no fp32
// dQ in memory, no atomics, the same bits on every call. With fewer items than
// places for CTAs the walks are divided too, and k_exact_sum adds up, in order,
// what the parts leave.
//
// What bounds them. At D = 128 the products and the shared memory that feeds
// them: tensor pipe 73 % (dQ) and 67 % (dK, dV). B4 H12 N4096 causal: both 490 us,
// 1.06 PFLOP/s counting five products, 0.55 of the measured bf16 rate. For D <= 64
// the weights' warps, whose steps of a tile stand one behind the other: B4 H12
// N4096 d64 causal, dQ 137 us, dK and dV 205.
#include <type_traits>

#include "device_common.cuh"
#include "exact.h"
#include "tc_common.cuh"
#include "tc_race.cuh"

namespace elsaa {

namespace {

using namespace tc;

// What a CTA of either kernel is made of, by the head's size. It holds 128 rows
// and walks tiles of `rows` others; weights are made by threads of 32 columns,
// rows / 32 of them a held row; four more warps issue and load.
//   D = 128: tiles of 128, 16 warps for the weights, one CTA an SM (it needs
//            all of its tensor memory).
//   D <= 64: tiles of 64, 8 warps, two CTAs an SM. A tile's waits, loads,
//            exponentials and stores stand one behind the other; two CTAs fill
//            each other's gaps.
template <int D>
struct Eb {
    static constexpr int rows = D > 64 ? 128 : 64;
    static constexpr int parts = rows / 32;
    static constexpr int weights = 4 * parts;  // warps
    static constexpr int threads = 32 * (weights + 4);
    static constexpr int ctas = D > 64 ? 1 : 2;
    static constexpr int columns = D > 64 ? 512 : 256;  // of tensor memory
    static constexpr int out = D / parts;  // columns of sums a thread writes
    // registers: at launch, of the weights' threads, of the others
    static constexpr int regs = D > 64 ? 96 : 80;
    static constexpr int soft = D > 64 ? 104 : 88, other = 64;
    static_assert(32 * weights * soft + 128 * other <= threads * regs,
                  "register shares within the launch's total");
    static constexpr int panels = D > 64 ? 2 : 1;
    static constexpr uint32_t held = panels * 16384;       // bytes of 128 rows
    static constexpr uint32_t tile = panels * rows * 128;  // of a tile
};

// A test of a barrier takes about 54 clocks, a try_wait 90.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t par,
                                          volatile int *abort,
                                          DeviceStatus *st, int site) {
    if (__all_sync(0xffffffffu, mbar_test(bar, par))) return true;
    return __all_sync(0xffffffffu,
                      mbar_wait_or_abort(bar, par, abort, st, site));
}
// Two at once, tested side by side.
__device__ __forceinline__ bool warp_wait2(uint64_t *a, uint32_t pa,
                                           uint64_t *b, uint32_t pb,
                                           volatile int *abort,
                                           DeviceStatus *st, int site) {
    const bool ready = mbar_test(a, pa) & mbar_test(b, pb);
    if (__all_sync(0xffffffffu, ready)) return true;
    return __all_sync(0xffffffffu,
                      mbar_wait_or_abort(a, pa, abort, st, site) &&
                          mbar_wait_or_abort(b, pb, abort, st, site));
}

// 32 columns of tensor memory
__device__ __forceinline__ void load32(uint32_t t, float2 (&x)[16]) {
    uint32_t a[32];
    tmem_ld32(t, a);
    tmem_wait_ld();
#pragma unroll
    for (int i = 0; i < 16; ++i)
        x[i] = make_float2(__uint_as_float(a[2 * i]),
                           __uint_as_float(a[2 * i + 1]));
}
// as bf16 (rounded to nearest) in 16 columns, for the products: one lane of
// the warp then arrives on `bar`
__device__ __forceinline__ void store32(uint32_t t, const float2 (&x)[16],
                                        uint64_t *bar, int lane_id) {
    uint32_t y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) y[i] = pack_bf16x2(x[i].x, x[i].y);
    tmem_st16(t, y);
    tmem_wait_st();
    tc_fence_before();
    __syncwarp();
    if (lane_id == 0) mbar_arrive(bar);
}

// A product of K = D (both K-major) and one of K = rows (A from tensor
// memory: 16 columns of every 32, as threads of 32 columns write them; B
// MN-major), issued by one lane.
template <int D>
__device__ __forceinline__ void mma_scores(uint32_t dst, uint64_t a,
                                           uint64_t b) {
    const uint32_t id = idesc_bf16(128, Eb<D>::rows, false, false);
#pragma unroll
    for (int x = 0; x < D / 16; ++x) {
        const uint32_t o = (x >> 2) * 1024 + (x & 3) * 2;
        mma_ss(dst, a + o, b + o, id, x > 0);
    }
}
template <int D>
__device__ __forceinline__ void mma_sums(uint32_t dst, uint32_t a, uint64_t b,
                                         bool more) {
    const uint32_t id = idesc_bf16(128, D, false, true);
#pragma unroll
    for (int x = 0; x < Eb<D>::rows / 16; ++x)
        mma_ts(dst, a + (x >> 1) * 32 + (x & 1) * 8, b + 128 * x, id,
               x > 0 || more);
}

// The rows of a tile in shared memory from `part` on become zeros (all lanes).
template <int D>
__device__ __forceinline__ void zero_rows(uint32_t tile, int part,
                                          int lane_id) {
    using E = Eb<D>;
    for (int i = max(part, 0) * 8 + lane_id; i < E::rows * 8; i += 32)
        for (int p = 0; p < E::panels; ++p)
            st_shared_zero16(tile + p * E::rows * 128 + i * 16);
    fence_proxy_async_smem();
    __syncwarp();
}

// A thread's columns of sums in tensor memory, times f, to a row of bf16 (the
// whole warp).
template <int D>
__device__ __forceinline__ void store_sums(uint32_t t, float f, uint16_t *o,
                                           bool valid, int lane_id) {
    constexpr int n = Eb<D>::out;
    uint32_t x[n], y[n / 2];
    if constexpr (n == 32)
        tmem_ld32(t, x);
    else
        tmem_ld16(t, x);
    tmem_wait_ld();
#pragma unroll
    for (int e = 0; e < n / 2; ++e)
        y[e] = pack_bf16x2(__uint_as_float(x[2 * e]) * f,
                           __uint_as_float(x[2 * e + 1]) * f);
    store_rows<D, n / 8>(y, o, valid, lane_id);
}
template <int D>
__device__ __forceinline__ void store_zeros(uint16_t *o) {
#pragma unroll
    for (int c = 0; c < Eb<D>::out; c += 8)
        *reinterpret_cast<uint4 *>(o + c) = make_uint4(0, 0, 0, 0);
}

// The same columns as they are, to [D / 8][128 rows][8].
template <int D>
__device__ __forceinline__ void store_part(uint32_t t, float *o) {
    constexpr int n = Eb<D>::out;
#pragma unroll
    for (int c = 0; c < n; c += 16) {
        uint32_t x[16], y[8];
        tmem_ld16(t + c, x);
        tmem_wait_ld();
#pragma unroll
        for (int h = 0; h < 16; h += 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = x[h + e];
            st_global_v8(o + (c + h) * 128, y);
        }
    }
}

// D_i = <dO_i, O_i>, D / 8 lanes a row; clears the status, two counters and the
// flag behind them.
template <int D>
__global__ void __launch_bounds__(256)
    k_exact_delta(const __grid_constant__ ExactView a, int *counters) {
    wait_for_stream();
    constexpr int L = D / 8;
    if (blockIdx.x == 0 && threadIdx.x < 7)
        (threadIdx.x < 4 ? &a.status->code + threadIdx.x
                         : counters + threadIdx.x - 4)[0] = 0;
    const long row = ((long)blockIdx.x * 256 + threadIdx.x) / L;
    const int c = threadIdx.x % L * 8;
    if (row >= (long)a.B * a.H * a.Nq) return;
    const int b = (int)(row / ((long)a.H * a.Nq)), i = (int)(row % a.Nq);
    float t = 0.0f;
    if (i < ExactSeq(a, b).ql) {
        const uint4 x = *reinterpret_cast<const uint4 *>(
            (const uint16_t *)a.d_o + row * D + c);
        const uint4 y = *reinterpret_cast<const uint4 *>(
            (const uint16_t *)a.o + row * D + c);
        const uint32_t u[4] = {x.x, x.y, x.z, x.w};
        const uint32_t w[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            t = fmaf(__uint_as_float(u[e] << 16), __uint_as_float(w[e] << 16),
                     t);
            t = fmaf(__uint_as_float(u[e] & 0xffff0000u),
                     __uint_as_float(w[e] & 0xffff0000u), t);
        }
    }
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1)
        t += __shfl_xor_sync(0xffffffffu, t, o);
    if (c == 0) a.delta[row] = t;
}

// ------------------------------------------------------------------- dQ

// Key and value tiles held: K(j) serves S(j) and dQ(j), behind S(j + 2).
template <int D>
constexpr int kDqK = D > 64 ? 3 : 5;
template <int D>
constexpr int kDqV = D > 64 ? 2 : 4;

template <int D>
struct DqBars {
    uint64_t item_full[2], item_empty[2], q_full, q_empty;
    uint64_t k_full[kDqK<D>], k_empty[kDqK<D>];
    uint64_t v_full[kDqV<D>], v_empty[kDqV<D>];
    uint64_t s_full[2], dp_full, dp_read, ds_full[2], dq_full, dq_empty;
};
struct BwdItem {
    int item;  // -1: no more
    int b, kvh, r0;
    int ql, kl;
    int n;     // tiles to walk
    int first; // keys held: the first query row that sees one
    int t0;    // the first tile of the walk
    int part;  // where a divided walk's sums go, -1: the walk is whole
    int rest;  // 1: a part of nothing, whose item others write
};

// Walks of n tiles in at most `splits` parts of kEbLeast tiles and more. Part p
// of item i of the call leaves its sums in o[i splits + p][D / 8][128][8] (keys:
// dK, then dV).
constexpr int kEbLeast = 4;
struct EbSplit {
    int splits;
    float *o;
};
__device__ __forceinline__ int parts_of(const EbSplit &s, int n) {
    return min(s.splits, max(1, n / kEbLeast));
}
// Part p of a walk: sets t0, n, part and rest.
__device__ __forceinline__ void take_part(const EbSplit &s, int p, int index,
                                          BwdItem &w) {
    const int parts = parts_of(s, w.n);
    w.rest = p >= parts;
    const int end = w.rest ? 0 : (int)((long)w.n * (p + 1) / parts);
    w.t0 = w.rest ? 0 : (int)((long)w.n * p / parts);
    w.part = parts > 1 ? index * s.splits + p : -1;
    w.n = end - w.t0;
}

// A CTA holds Q and dO of 128 rows (of the heads that share a K/V head,
// counted through) and walks key tiles. The first warps make the weights; then
// one issues S and dQ, one dP, one takes the items and loads Q, dO and K, one V.
// Tensor memory: S of two tiles, dP, dQ; dS goes over the S it came from.
template <int D>
__global__ void __launch_bounds__(Eb<D>::threads, Eb<D>::ctas)
    k_exact_dq_tc(const __grid_constant__ CUtensorMap tmQ,
                  const __grid_constant__ CUtensorMap tmG,
                  const __grid_constant__ CUtensorMap tmK,
                  const __grid_constant__ CUtensorMap tmV,
                  const __grid_constant__ ExactView a,
                  const __grid_constant__ ExactOrder order,
                  const __grid_constant__ EbSplit split, int items,
                  int *__restrict__ next_item, int *far_rows) {
    wait_for_stream();
    extern __shared__ unsigned char smem_raw[];
    __shared__ DqBars<D> bars;
    constexpr int kK = kDqK<D>, kV = kDqV<D>;
    __shared__ uint32_t tbase;
    __shared__ int abort_flag;
    __shared__ BwdItem item_s[2];
    volatile int *abort = &abort_flag;
    using E = Eb<D>;
    constexpr uint32_t kTile = E::tile;
    // tensor memory columns
    constexpr uint32_t kS = 0, kP = 2 * E::rows, kO = 3 * E::rows;
    const int tid = threadIdx.x, warp = tid >> 5, lane_id = tid & 31;
    const uint32_t sQ = align1k(smem_u32(smem_raw)), sG = sQ + E::held;
    const uint32_t sK = sG + E::held, sV = sK + kK * kTile;
    DeviceStatus *status = a.status;

    if (warp == E::weights) tmem_alloc(&tbase, E::columns);
    if (tid == 0) {
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars.item_full[s], 1);
            mbar_init(&bars.item_empty[s], E::weights + 3);
            mbar_init(&bars.s_full[s], 1);
            mbar_init(&bars.ds_full[s], E::weights);
        }
        for (int s = 0; s < kK; ++s) {
            mbar_init(&bars.k_full[s], 1);
            mbar_init(&bars.k_empty[s], 1);
        }
        for (int s = 0; s < kV; ++s) {
            mbar_init(&bars.v_full[s], 1);
            mbar_init(&bars.v_empty[s], 1);
        }
        mbar_init(&bars.q_full, 1);
        mbar_init(&bars.q_empty, 2);  // S and dP
        mbar_init(&bars.dp_full, 1);
        mbar_init(&bars.dp_read, E::weights);
        mbar_init(&bars.dq_full, 1);
        mbar_init(&bars.dq_empty, E::weights);
        abort_flag = 0;
        fence_mbar_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tbase;

    if (warp >= E::weights) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(
            E::other));
        if (warp == E::weights + 2 && lane_id == 0) {
            // ---------------------------------------------- items and loads
            int c = 0, qs = 0;  // key tiles and items loaded so far
            bool ok = true;
            const int heads = a.B * a.Hkv, rows = order.rows;
            auto tile = [&](uint64_t *full, uint32_t dst,
                            const CUtensorMap *map, int row, int rows_) {
                for (int p = 0; p < E::panels; ++p)
                    tma_load_2d(dst + p * rows_ * 128, map, 64 * p, row, full);
            };
            for (int it = 0; ok; ++it) {
                const long item =
                    it == 0 ? blockIdx.x
                            : (long)gridDim.x + atomicAdd(next_item, 1);
                if (it >= 2 && !mbar_wait_or_abort(&bars.item_empty[it & 1],
                                                   ((it >> 1) - 1) & 1, abort,
                                                   status, 420))
                    break;
                BwdItem w = {-1};
                if (item < items) {
                    // the last rows of every query head, which see most, first
                    const int h = (int)(item % heads);
                    w.item = (int)item;
                    const int x = order.tile((int)(item / heads) /
                                             split.splits);
                    w.r0 = x * 128;
                    w.b = h / a.Hkv;
                    w.kvh = h - w.b * a.Hkv;
                    const ExactSeq seq(a, w.b);
                    w.ql = seq.ql;
                    w.kl = seq.kl;
                    w.n = (exact_most(seq, w.r0, min(w.r0 + 128, rows),
                                      order.pitch) + E::rows - 1) / E::rows;
                    take_part(split, (int)(item / heads) % split.splits,
                              h * order.groups * order.per + x, w);
                }
                item_s[it & 1] = w;
                mbar_arrive(&bars.item_full[it & 1]);
                if (w.item < 0) break;
                if (w.n == 0) continue;
                if (qs >= 1 && !mbar_wait_or_abort(&bars.q_empty, (qs - 1) & 1,
                                                   abort, status, 421))
                    break;
                ++qs;
                const int q0 = (w.b * a.H + w.kvh * a.G) * a.Nq +
                               order.row(w.r0, a.Nq);
                const int k0 =
                    (w.b * a.Hkv + w.kvh) * a.Nk + E::rows * w.t0;
                mbar_expect_tx(&bars.q_full, 2 * E::held);
                tile(&bars.q_full, sQ, &tmQ, q0, 128);
                tile(&bars.q_full, sG, &tmG, q0, 128);
                for (int kt = 0; kt < w.n; ++kt, ++c) {
                    const int ks = c % kK;
                    if (c >= kK &&
                        !(ok = mbar_wait_or_abort(&bars.k_empty[ks],
                                                  (c / kK - 1) & 1, abort,
                                                  status, 422)))
                        break;
                    mbar_expect_tx(&bars.k_full[ks], kTile);
                    tile(&bars.k_full[ks], sK + ks * kTile, &tmK,
                         k0 + E::rows * kt, E::rows);
                }
            }
        } else if (warp == E::weights + 3 && lane_id == 0) {
            // ------------------------------------------ loads of the values
            int c = 0;
            bool ok = true;
            for (int it = 0; ok; ++it) {
                if (!mbar_wait_or_abort(&bars.item_full[it & 1], (it >> 1) & 1,
                                        abort, status, 423))
                    break;
                const BwdItem w = item_s[it & 1];
                mbar_arrive(&bars.item_empty[it & 1]);
                if (w.item < 0) break;
                const int k0 =
                    (w.b * a.Hkv + w.kvh) * a.Nk + E::rows * w.t0;
                for (int kt = 0; kt < w.n; ++kt, ++c) {
                    const int vs = c % kV;
                    if (c >= kV &&
                        !(ok = mbar_wait_or_abort(&bars.v_empty[vs],
                                                  (c / kV - 1) & 1, abort,
                                                  status, 435)))
                        break;
                    mbar_expect_tx(&bars.v_full[vs], kTile);
                    for (int p = 0; p < E::panels; ++p)
                        tma_load_2d(sV + vs * kTile + p * E::rows * 128, &tmV, 64 * p,
                                    k0 + E::rows * kt, &bars.v_full[vs]);
                }
            }
        } else if (warp < E::weights + 2) {
            // ---------------------------------------------------- MMA issue
            // One warp for S and dQ, one for dP: a wait costs a warp about 150
            // clocks even when there is nothing to wait for, and few products
            // are queued behind those that run. S(j + 2) goes over dS(j)
            // behind dQ(j), which reads it: products of one thread run in the
            // order of their issue.
            const bool el = elect_one();
            auto wait = [&](uint64_t *bar, uint32_t par, int site) {
                return warp_wait(bar, par, abort, status, site);
            };
            const bool first = warp == E::weights;
            const uint64_t dQ = smem_desc(sQ, 16, 1024);
            const uint64_t dG = smem_desc(sG, 16, 1024);
            const uint64_t dK = smem_desc(sK, 16, 1024);
            const uint64_t dKm = smem_desc(sK, 16384, 1024);
            const uint64_t dV = smem_desc(sV, 16, 1024);
            int c = 0, qs = 0;  // tiles of earlier items, items
            bool ok = true;
            for (int it = 0; ok; ++it) {
                if (!wait(&bars.item_full[it & 1], (it >> 1) & 1, 424)) break;
                const int item = item_s[it & 1].item, n = item_s[it & 1].n;
                // keys of the sequence from the walk's first tile on
                const int kl =
                    item_s[it & 1].kl - E::rows * item_s[it & 1].t0;
                __syncwarp();
                if (el) mbar_arrive(&bars.item_empty[it & 1]);
                if (item < 0) break;
                if (n == 0) continue;
                if (!wait(&bars.q_full, qs & 1, 425)) break;
                if (!first) {
                    for (int j = 0; j < n; ++j) {
                        const int x = c + j, vs = x % kV;
                        ok = wait(&bars.v_full[vs], x / kV & 1, 427) &&
                             (x == 0 ||
                              wait(&bars.dp_read, (x - 1) & 1, 428));
                        if (!ok) break;
                        tc_fence_after();
                        if (el) {
                            mma_scores<D>(tm + kP, dG, desc_at(dV, vs * kTile));
                            mma_commit(&bars.dp_full);
                            mma_commit(&bars.v_empty[vs]);
                            if (j == n - 1) mma_commit(&bars.q_empty);
                        }
                    }
                    c += n;
                    ++qs;
                    continue;
                }
                auto scores = [&](int j) {
                    const int x = c + j, ks = x % kK;
                    if (!wait(&bars.k_full[ks], x / kK & 1, 426))
                        return false;
                    // keys that the sequence does not have count with dS = 0
                    // in dQ and must be numbers
                    if (kl - E::rows * j < E::rows)
                        zero_rows<D>(sK + ks * kTile, kl - E::rows * j,
                                     lane_id);
                    tc_fence_after();
                    if (el) {
                        mma_scores<D>(tm + kS + E::rows * (x & 1), dQ,
                                      desc_at(dK, ks * kTile));
                        mma_commit(&bars.s_full[x & 1]);
                        if (j == n - 1) mma_commit(&bars.q_empty);
                    }
                    return true;
                };
                ok = scores(0) && (n < 2 || scores(1));
                if (ok && qs > 0)
                    ok = wait(&bars.dq_empty, (qs - 1) & 1, 429);
                for (int j = 0; j < n && ok; ++j) {
                    const int x = c + j, ks = x % kK;
                    ok = wait(&bars.ds_full[x & 1], x / 2 & 1, 430);
                    if (!ok) break;
                    tc_fence_after();
                    if (el) {
                        mma_sums<D>(tm + kO, tm + kS + E::rows * (x & 1),
                                    desc_at(dKm, ks * kTile), j > 0);
                        mma_commit(&bars.k_empty[ks]);
                        if (j == n - 1) mma_commit(&bars.dq_full);
                    }
                    if (j + 2 < n) ok = scores(j + 2);
                }
                c += n;
                ++qs;
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------- weights
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(E::soft));
        const int part = warp >> 2, row = (warp & 3) * 32 + lane_id;
        const uint32_t lane = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t0 = tm + lane + 32 * part;
        const float sl2 = a.scale * kLog2e;
        const float2 sl22 = make_float2(sl2, sl2);
        int c = 0, qs = 0;
        bool ok = true;
        for (int it = 0; ok; ++it) {
            if (!warp_wait(&bars.item_full[it & 1], (it >> 1) & 1, abort,
                           status, 431))
                break;
            const BwdItem w = item_s[it & 1];
            __syncwarp();
            if (lane_id == 0) mbar_arrive(&bars.item_empty[it & 1]);
            if (w.item < 0) break;
            const int r = w.r0 + row, i = r % order.pitch;
            const bool valid = r < order.rows && i < w.ql;
            const size_t at = (size_t)(w.b * a.H + w.kvh * a.G) * a.Nq +
                              order.row(r, a.Nq);
            uint16_t *o = (uint16_t *)a.dq + at * D + E::out * part;
            if (w.n == 0) {
                if (valid && !w.rest) store_zeros<D>(o);
                continue;
            }
            int seen = 0;
            float nl = 0.0f, nd = 0.0f;
            if (valid) {
                seen = a.causal ? max(0, min(w.kl, i + 1 + w.kl - w.ql))
                                : w.kl;
                nl = -exact_lse(a.lse + at) * kLog2e;
                nd = -a.delta[at];
            }
            const float2 nl2 = make_float2(nl, nl), nd2 = make_float2(nd, nd);
            // Two loops, here and for dK and dV: the backward pass of B4 H12
            // N4096 d64 causal takes 344 us, with a branch in one loop 346,
            // without either 338.
            auto walk = [&](auto far) {
                const float edge = exact_edge(nl);
                for (int j = 0; j < w.n; ++j, ++c) {
                    if (!(ok = warp_wait(&bars.s_full[c & 1], c / 2 & 1, abort,
                                         status, 432)))
                        break;
                    tc_fence_after();
                    const uint32_t tS = t0 + kS + E::rows * (c & 1);
                    float2 p[16], g[16];
                    load32(tS, p);
#pragma unroll
                    for (int q = 0; q < 16; ++q) {
                        p[q] = fma2(p[q], sl22, nl2);
                        if (decltype(far)::value)
                            p[q] = make_float2(exact_exponent(p[q].x, edge),
                                               exact_exponent(p[q].y, edge));
                        p[q] = make_float2(ex2_approx(p[q].x), ex2_approx(p[q].y));
                    }
                    if (!(ok = warp_wait(&bars.dp_full, c & 1, abort, status,
                                         433)))
                        break;
                    tc_fence_after();
                    load32(t0 + kP, g);
                    tc_fence_before();
                    __syncwarp();
                    if (lane_id == 0) mbar_arrive(&bars.dp_read);
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        g[q] = mul2(p[q], add2(g[q], nd2));
                    const int lim = seen - E::rows * (w.t0 + j) - 32 * part;
                    if (__any_sync(0xffffffffu, lim < 32)) {
#pragma unroll
                        for (int q = 0; q < 16; ++q) {
                            if (2 * q >= lim) g[q].x = 0.0f;
                            if (2 * q + 1 >= lim) g[q].y = 0.0f;
                        }
                    }
                    store32(tS, g, &bars.ds_full[c & 1], lane_id);
                }
            };
            if (__any_sync(0xffffffffu, exact_edge(nl) < INFINITY)) {
                if (lane_id == 0) *far_rows = 1;
                walk(std::true_type{});
            } else {
                walk(std::false_type{});
            }
            if (!ok) break;
            if (!(ok = warp_wait(&bars.dq_full, qs & 1, abort, status, 434)))
                break;
            ++qs;
            tc_fence_after();
            const uint32_t to = tm + lane + kO + E::out * part;
            if (w.part >= 0)
                store_part<D>(to, split.o + (size_t)w.part * 128 * D +
                                      E::out * part * 128 + row * 8);
            else
                store_sums<D>(to, a.scale, o, valid, lane_id);
            tc_fence_before();
            __syncwarp();
            if (lane_id == 0) mbar_arrive(&bars.dq_empty);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == E::weights) tmem_dealloc(tm, E::columns);
}

// --------------------------------------------------------------- dK and dV

template <int D>
struct Dkv {
    static constexpr int kQ = D > 64 ? 3 : 4, kG = D > 64 ? 2 : 4;  // tiles held
    // tensor memory columns
    static constexpr uint32_t cS = 0, cP = Eb<D>::rows, cV = 2 * Eb<D>::rows,
                              cK = cV + D;
};
template <int D>
struct DkvBars {
    uint64_t item_full[2], item_empty[2], kv_full, kv_empty;
    uint64_t q_full[Dkv<D>::kQ], q_empty[Dkv<D>::kQ];
    uint64_t g_full[Dkv<D>::kG], g_empty[Dkv<D>::kG];
    uint64_t l_empty[2], s_full[2], p_full[2];
    uint64_t dp_full, ds_full, sum_full, sum_empty;
};

// What lies behind the tiles in shared memory (there are 3 KB).
template <int D>
struct DkvShared {
    // -lse (base 2) and -D of the rows
    float row_l[2][Eb<D>::rows], row_d[2][Eb<D>::rows];
    DkvBars<D> bars;
    BwdItem item[2];
    uint32_t tbase;
    int abort_flag;
};

// A CTA holds K and V of 128 rows and walks tiles of query rows of every head
// that reads them; scores and weights stand transposed, a key a lane. The first
// warps make the weights; then one issues the products, one (behind one that
// has nothing to do) takes the items and loads K, V and Q, and one loads dO and
// fetches the rows' lse and D. Tensor memory: S^T, dP^T, dV, dK; P^T and dS^T go
// over the S^T and dP^T that they came from.
template <int D>
__global__ void __launch_bounds__(Eb<D>::threads, Eb<D>::ctas)
    k_exact_dkv_tc(const __grid_constant__ CUtensorMap tmQ,
                   const __grid_constant__ CUtensorMap tmG,
                   const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV,
                   const __grid_constant__ ExactView a,
                   const __grid_constant__ EbSplit split, int items,
                   int *__restrict__ next_item,
                   const volatile int *far_rows) {
    wait_for_stream();
    using X = Dkv<D>;
    extern __shared__ unsigned char smem_raw[];
    using E = Eb<D>;
    constexpr uint32_t kTile = E::tile;
    constexpr uint32_t kTiles = 2 * E::held + (X::kQ + X::kG) * kTile;
    // there is no room for a whole KB of padding: dynamic shared memory begins
    // on one, as the kernel has no other
    const uint32_t pad = align1k(smem_u32(smem_raw)) - smem_u32(smem_raw);
    if (pad > 0) {
        report(a.status, kDevLayout, 459, (int)pad, 0);
        return;
    }
    DkvShared<D> &sh = *reinterpret_cast<DkvShared<D> *>(smem_raw + kTiles);
    auto &bars = sh.bars;
    auto &item_s = sh.item;
    auto &row_l = sh.row_l, &row_d = sh.row_d;
    volatile int *abort = &sh.abort_flag;
    const int tid = threadIdx.x, warp = tid >> 5, lane_id = tid & 31;
    const uint32_t sK = smem_u32(smem_raw), sV = sK + E::held;
    const uint32_t sQ = sV + E::held, sG = sQ + X::kQ * kTile;
    DeviceStatus *status = a.status;

    if (warp == E::weights) tmem_alloc(&sh.tbase, E::columns);
    if (tid == 0) {
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars.item_full[s], 1);
            mbar_init(&bars.item_empty[s], E::weights + 2);
            mbar_init(&bars.l_empty[s], E::weights);
            mbar_init(&bars.s_full[s], 2);  // the product, lse and D
            mbar_init(&bars.p_full[s], E::weights);
        }
        for (int s = 0; s < X::kG; ++s) {
            mbar_init(&bars.g_full[s], 1);
            mbar_init(&bars.g_empty[s], 1);
        }
        for (int s = 0; s < X::kQ; ++s) {
            mbar_init(&bars.q_full[s], 1);
            mbar_init(&bars.q_empty[s], 1);
        }
        mbar_init(&bars.kv_full, 1);
        mbar_init(&bars.kv_empty, 1);
        mbar_init(&bars.dp_full, 1);
        mbar_init(&bars.ds_full, E::weights);
        mbar_init(&bars.sum_full, 1);
        mbar_init(&bars.sum_empty, E::weights);
        sh.abort_flag = 0;
        fence_mbar_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = sh.tbase;
    // tiles of a query head's rows, walked head by head
    auto tiles_of = [](const BwdItem &w) {
        return (w.ql - w.first + E::rows - 1) / E::rows;
    };

    if (warp >= E::weights) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(
            E::other));
        if (warp == E::weights + 2 && lane_id == 0) {
            // ---------------------------------------------- items and loads
            int c = 0, ks = 0;  // query tiles and items loaded so far
            bool ok = true;
            const int heads = a.B * a.Hkv;
            auto tile = [&](uint64_t *full, uint32_t dst,
                            const CUtensorMap *map, int row, int rows_) {
                for (int p = 0; p < E::panels; ++p)
                    tma_load_2d(dst + p * rows_ * 128, map, 64 * p, row, full);
            };
            for (int it = 0; ok; ++it) {
                const long item =
                    it == 0 ? blockIdx.x
                            : (long)gridDim.x + atomicAdd(next_item, 1);
                if (it >= 2 && !mbar_wait_or_abort(&bars.item_empty[it & 1],
                                                   ((it >> 1) - 1) & 1, abort,
                                                   status, 440))
                    break;
                BwdItem w = {-1};
                if (item < items) {
                    // the first keys, which are seen most, first
                    const int h = (int)(item % heads);
                    w.item = (int)item;
                    const int x = (int)(item / heads) / split.splits;
                    w.r0 = x * 128;
                    w.b = h / a.Hkv;
                    w.kvh = h - w.b * a.Hkv;
                    const ExactSeq seq(a, w.b);
                    w.ql = seq.ql;
                    w.kl = seq.kl;
                    w.first = seq.first_row(w.r0);
                    w.n = a.G * tiles_of(w);
                    take_part(split, (int)(item / heads) % split.splits,
                              h * ((a.Nk + 127) / 128) + x, w);
                }
                item_s[it & 1] = w;
                mbar_arrive(&bars.item_full[it & 1]);
                if (w.item < 0) break;
                if (w.n == 0) continue;
                if (ks >= 1 && !mbar_wait_or_abort(&bars.kv_empty,
                                                   (ks - 1) & 1, abort,
                                                   status, 441))
                    break;
                ++ks;
                const int k0 = (w.b * a.Hkv + w.kvh) * a.Nk + w.r0;
                mbar_expect_tx(&bars.kv_full, 2 * E::held);
                tile(&bars.kv_full, sK, &tmK, k0, 128);
                tile(&bars.kv_full, sV, &tmV, k0, 128);
                const int per = tiles_of(w);
                int head = (w.b * a.H + w.kvh * a.G + w.t0 / per) * a.Nq;
                int i = w.first + w.t0 % per * E::rows;
                for (int t = 0; t < w.n; ++t, ++c) {
                    const int qs = c % X::kQ;
                    if (c >= X::kQ &&
                        !(ok = mbar_wait_or_abort(&bars.q_empty[qs],
                                                  (c / X::kQ - 1) & 1, abort,
                                                  status, 442)))
                        break;
                    mbar_expect_tx(&bars.q_full[qs], kTile);
                    tile(&bars.q_full[qs], sQ + qs * kTile, &tmQ, head + i,
                         E::rows);
                    i += E::rows;
                    if (i >= w.ql) {
                        i = w.first;
                        head += a.Nq;
                    }
                }
            }
        } else if (warp == E::weights) {
            // ---------------------------------------------------- MMA issue
            // In the order dV(t), S(t + 1), dK(t), dP(t + 1): P(t + 1) is
            // made during dK(t) and dP(t + 1), dS(t) during dV(t) and
            // S(t + 1). Few products are queued behind those that run, so
            // that the tensor cores stand still during waits, even such that
            // find their barrier complete: two products a wait. (A warp for
            // each pair let the pairs' products run mixed, each of them later:
            // 216 us instead of 201 at D = 128.) Products of one thread run in
            // the order of their issue, which S over P and dP over dS rely on.
            const bool el = elect_one();
            auto wait = [&](uint64_t *bar, uint32_t par, int site) {
                return warp_wait(bar, par, abort, status, site);
            };
            auto wait2 = [&](uint64_t *x, uint32_t px, uint64_t *y,
                             uint32_t py, int site) {
                return warp_wait2(x, px, y, py, abort, status, site);
            };
            const uint64_t dK = smem_desc(sK, 16, 1024);
            const uint64_t dV = smem_desc(sV, 16, 1024);
            const uint64_t dQ = smem_desc(sQ, 16, 1024);
            const uint64_t dQm = smem_desc(sQ, 16384, 1024);
            const uint64_t dG = smem_desc(sG, 16, 1024);
            const uint64_t dGm = smem_desc(sG, 16384, 1024);
            int c = 0, ks = 0;
            bool ok = true;
            for (int it = 0; ok; ++it) {
                if (!wait(&bars.item_full[it & 1], (it >> 1) & 1, 444)) break;
                const int item = item_s[it & 1].item, n = item_s[it & 1].n;
                // Rows that the sequence does not have count with weights of
                // 0 and must be numbers: rows of the next Q or dO tile that
                // it has.
                const int all = item_s[it & 1].ql - item_s[it & 1].first;
                const int t0 = item_s[it & 1].t0;
                __syncwarp();
                if (el) mbar_arrive(&bars.item_empty[it & 1]);
                if (item < 0) break;
                if (n == 0) continue;
                int left_q =
                    all - t0 % ((all + E::rows - 1) / E::rows) * E::rows;
                int left_g = left_q;
                // the tile of S(t) or dP(t) is there
                auto scores = [&](int t) {
                    const int x = c + t, qs = x % X::kQ;
                    if (left_q < E::rows)
                        zero_rows<D>(sQ + qs * kTile, left_q, lane_id);
                    left_q = left_q > E::rows ? left_q - E::rows : all;
                    tc_fence_after();
                    if (el) {
                        mma_scores<D>(tm + X::cS, dK,
                                      desc_at(dQ, qs * kTile));
                        mma_commit(&bars.s_full[x & 1]);
                    }
                };
                auto products = [&](int t) {
                    const int x = c + t, gs = x % X::kG;
                    if (left_g < E::rows)
                        zero_rows<D>(sG + gs * kTile, left_g, lane_id);
                    left_g = left_g > E::rows ? left_g - E::rows : all;
                    tc_fence_after();
                    if (el) {
                        mma_scores<D>(tm + X::cP, dV, desc_at(dG, gs * kTile));
                        mma_commit(&bars.dp_full);
                        if (t == n - 1) mma_commit(&bars.kv_empty);
                    }
                };
                auto q_at = [&](int t) { return &bars.q_full[(c + t) % X::kQ]; };
                auto g_at = [&](int t) { return &bars.g_full[(c + t) % X::kG]; };
                ok = wait2(&bars.kv_full, ks & 1, q_at(0), c / X::kQ & 1, 445);
                if (!ok) break;
                scores(0);
                if (!(ok = wait(g_at(0), c / X::kG & 1, 447))) break;
                products(0);
                if (ks > 0 &&
                    !(ok = wait(&bars.sum_empty, (ks - 1) & 1, 448)))
                    break;
                for (int t = 0; t < n && ok; ++t) {
                    const int x = c + t, qs = x % X::kQ, gs = x % X::kG;
                    const int u = t + 1;
                    uint64_t *p = &bars.p_full[x & 1];
                    ok = u < n ? wait2(p, x / 2 & 1, q_at(u),
                                       (c + u) / X::kQ & 1, 449)
                               : wait(p, x / 2 & 1, 460);
                    if (!ok) break;
                    tc_fence_after();
                    if (el) {
                        mma_sums<D>(tm + X::cV, tm + X::cS,
                                    desc_at(dGm, gs * kTile), t > 0);
                        mma_commit(&bars.g_empty[gs]);
                    }
                    if (u < n) scores(u);
                    ok = t + 1 < n
                             ? wait2(&bars.ds_full, x & 1, g_at(t + 1),
                                     (x + 1) / X::kG & 1, 450)
                             : wait(&bars.ds_full, x & 1, 461);
                    if (!ok) break;
                    tc_fence_after();
                    if (el) {
                        mma_sums<D>(tm + X::cK, tm + X::cP,
                                    desc_at(dQm, qs * kTile), t > 0);
                        mma_commit(&bars.q_empty[qs]);
                        if (t == n - 1) mma_commit(&bars.sum_full);
                    }
                    if (t + 1 < n) products(t + 1);
                }
                c += n;
                ++ks;
            }
        } else if (warp == E::weights + 3) {
            // --------------------------------- loads of dO, of lse and D
            int c = 0;
            bool ok = true;
            for (int it = 0; ok; ++it) {
                if (!warp_wait(&bars.item_full[it & 1], (it >> 1) & 1, abort,
                               status, 451))
                    break;
                const BwdItem w = item_s[it & 1];
                __syncwarp();
                if (lane_id == 0) mbar_arrive(&bars.item_empty[it & 1]);
                if (w.item < 0) break;
                if (w.n == 0) continue;
                const int per = tiles_of(w);
                int head = (w.b * a.H + w.kvh * a.G + w.t0 / per) * a.Nq;
                int i0 = w.first + w.t0 % per * E::rows;
                for (int t = 0; t < w.n; ++t, ++c) {
                    const int gs = c % X::kG;
                    const size_t at = (size_t)head + i0;
                    float l[E::parts], d[E::parts];
#pragma unroll
                    for (int q = 0; q < E::parts; ++q) {
                        const int i = lane_id + 32 * q;
                        l[q] = d[q] = 0.0f;
                        if (i0 + i < w.ql) {
                            l[q] = exact_lse(a.lse + at + i);
                            d[q] = a.delta[at + i];
                        }
                    }
                    if (c >= X::kG &&
                        !(ok = warp_wait(&bars.g_empty[gs],
                                         (c / X::kG - 1) & 1, abort, status,
                                         443)))
                        break;
                    if (lane_id == 0) {
                        mbar_expect_tx(&bars.g_full[gs], kTile);
                        for (int p = 0; p < E::panels; ++p)
                            tma_load_2d(sG + gs * kTile + p * E::rows * 128, &tmG,
                                        64 * p, head + i0, &bars.g_full[gs]);
                    }
                    if (c >= 2 && !(ok = warp_wait(&bars.l_empty[c & 1],
                                                   (c / 2 - 1) & 1, abort,
                                                   status, 452)))
                        break;
#pragma unroll
                    for (int q = 0; q < E::parts; ++q) {
                        row_l[c & 1][lane_id + 32 * q] = -l[q] * kLog2e;
                        row_d[c & 1][lane_id + 32 * q] = -d[q];
                    }
                    __syncwarp();
                    if (lane_id == 0) mbar_arrive(&bars.s_full[c & 1]);
                    i0 += E::rows;
                    if (i0 >= w.ql) {
                        i0 = w.first;
                        head += a.Nq;
                    }
                }
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------- weights
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(E::soft));
        const int part = warp >> 2, row = (warp & 3) * 32 + lane_id;
        const uint32_t lane = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t0 = tm + lane + 32 * part;
        const float sl2 = a.scale * kLog2e;
        const float2 sl22 = make_float2(sl2, sl2);
        const bool far_call = *far_rows != 0;
        int c = 0, ks = 0;
        bool ok = true;
        for (int it = 0; ok; ++it) {
            if (!warp_wait(&bars.item_full[it & 1], (it >> 1) & 1, abort,
                           status, 453))
                break;
            const BwdItem w = item_s[it & 1];
            __syncwarp();
            if (lane_id == 0) mbar_arrive(&bars.item_empty[it & 1]);
            if (w.item < 0) break;
            const int j = w.r0 + row;
            const bool valid = j < w.kl;
            const size_t at = ((size_t)(w.b * a.Hkv + w.kvh) * a.Nk + j) * D +
                              E::out * part;
            uint16_t *ok_ = (uint16_t *)a.dk + at, *ov = (uint16_t *)a.dv + at;
            if (w.n == 0) {
                if (valid && !w.rest) {
                    store_zeros<D>(ok_);
                    store_zeros<D>(ov);
                }
                continue;
            }
            // the first query row that sees the key, none: ql
            const int first = !valid ? w.ql
                              : a.causal ? min(w.ql, max(0, j + w.ql - w.kl))
                                         : 0;
            const int lo0 = first - w.first - 32 * part;
            const int hi0 = w.ql - w.first - 32 * part;
            const int skip = w.t0 % tiles_of(w) * E::rows;
            // columns of this part that see the key
            int lo = lo0 - skip, hi = hi0 - skip;
            auto walk = [&](auto far) {
                for (int t = 0; t < w.n; ++t, ++c) {
                    const bool edge = __any_sync(0xffffffffu, lo > 0 || hi < 32);
                    if (!(ok = warp_wait(&bars.s_full[c & 1], c / 2 & 1, abort,
                                         status, 455)))
                        break;
                    tc_fence_after();
                    const uint32_t tS = t0 + X::cS;
                    const float4 *nl = reinterpret_cast<const float4 *>(
                        &row_l[c & 1][32 * part]);
                    const float4 *nd = reinterpret_cast<const float4 *>(
                        &row_d[c & 1][32 * part]);
                    float2 p[16], g[16];
                    load32(tS, p);
#pragma unroll
                    for (int q = 0; q < 16; q += 2) {
                        const float4 l = nl[q / 2];
                        p[q] = fma2(p[q], sl22, make_float2(l.x, l.y));
                        p[q + 1] = fma2(p[q + 1], sl22, make_float2(l.z, l.w));
                        if (decltype(far)::value) {
                            p[q] = make_float2(
                                exact_exponent(p[q].x, exact_edge(l.x)),
                                exact_exponent(p[q].y, exact_edge(l.y)));
                            p[q + 1] = make_float2(
                                exact_exponent(p[q + 1].x, exact_edge(l.z)),
                                exact_exponent(p[q + 1].y, exact_edge(l.w)));
                        }
                    }
#pragma unroll
                    for (int q = 0; q < 16; ++q)
                        p[q] = make_float2(ex2_approx(p[q].x), ex2_approx(p[q].y));
                    if (edge) {
#pragma unroll
                        for (int q = 0; q < 16; ++q) {
                            if (2 * q < lo || 2 * q >= hi) p[q].x = 0.0f;
                            if (2 * q + 1 < lo || 2 * q + 1 >= hi) p[q].y = 0.0f;
                        }
                    }
                    store32(tS, p, &bars.p_full[c & 1], lane_id);
                    if (!(ok = warp_wait(&bars.dp_full, c & 1, abort, status,
                                         456)))
                        break;
                    tc_fence_after();
                    load32(t0 + X::cP, g);
#pragma unroll
                    for (int q = 0; q < 16; q += 2) {
                        const float4 d = nd[q / 2];
                        g[q] = mul2(p[q], add2(g[q], make_float2(d.x, d.y)));
                        g[q + 1] =
                            mul2(p[q + 1], add2(g[q + 1], make_float2(d.z, d.w)));
                    }
                    if (edge) {
#pragma unroll
                        for (int q = 0; q < 16; ++q) {
                            if (2 * q < lo || 2 * q >= hi) g[q].x = 0.0f;
                            if (2 * q + 1 < lo || 2 * q + 1 >= hi) g[q].y = 0.0f;
                        }
                    }
                    store32(t0 + X::cP, g, &bars.ds_full, lane_id);
                    if (lane_id == 0) mbar_arrive(&bars.l_empty[c & 1]);
                    lo -= E::rows;
                    hi -= E::rows;
                    if (hi + 32 * part <= 0) {  // the next head
                        lo = lo0;
                        hi = hi0;
                    }
                }
            };
            if (far_call)
                walk(std::true_type{});
            else
                walk(std::false_type{});
            if (!ok) break;
            if (!(ok = warp_wait(&bars.sum_full, ks & 1, abort, status, 457)))
                break;
            ++ks;
            tc_fence_after();
            const uint32_t t = tm + lane + E::out * part;
            if (w.part >= 0) {
                float *o = split.o + (size_t)w.part * 256 * D +
                           E::out * part * 128 + row * 8;
                store_part<D>(t + X::cK, o);
                store_part<D>(t + X::cV, o + 128 * D);
            } else {
                store_sums<D>(t + X::cV, 1.0f, ov, valid, lane_id);
                store_sums<D>(t + X::cK, a.scale, ok_, valid, lane_id);
            }
            tc_fence_before();
            __syncwarp();
            if (lane_id == 0) mbar_arrive(&bars.sum_empty);
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == E::weights) tmem_dealloc(tm, E::columns);
}

// The sums of walks that were divided: rows of dQ, then of dK and dV, D / 8
// lanes a row.
template <int D>
__global__ void __launch_bounds__(256)
    k_exact_sum(const __grid_constant__ ExactView a,
                const __grid_constant__ ExactOrder order,
                const __grid_constant__ EbSplit sq,
                const __grid_constant__ EbSplit sk) {
    wait_for_stream();
    using E = Eb<D>;
    int c;
    long row = piece_of<D>((long)blockIdx.x * 256 + threadIdx.x, &c);
    const long nq = sq.splits > 1 ? (long)a.B * a.H * a.Nq : 0;
    const bool keys = row >= nq;
    const float *from;
    size_t step;
    int parts;
    uint16_t *to;
    if (!keys) {
        const int group = a.G * a.Nq, head = (int)(row / group);
        const int x = (int)(row % group), i = x % a.Nq;
        const ExactSeq seq(a, head / a.Hkv);
        if (i >= seq.ql) return;
        const int r = x / a.Nq * order.pitch + i, r0 = r / 128 * 128;
        const int n = (exact_most(seq, r0, min(r0 + 128, order.rows),
                                  order.pitch) + E::rows - 1) / E::rows;
        parts = parts_of(sq, n);
        const size_t index = (size_t)head * order.groups * order.per + r / 128;
        from = sq.o + index * sq.splits * 128 * D + c * 128 + (r - r0) * 8;
        step = 128 * D;
        to = (uint16_t *)a.dq + row * D + c;
    } else {
        row -= nq;
        if (sk.splits == 1 || row >= (long)a.B * a.Hkv * a.Nk) return;
        const int head = (int)(row / a.Nk), j = (int)(row % a.Nk);
        const ExactSeq seq(a, head / a.Hkv);
        if (j >= seq.kl) return;
        const int r0 = j / 128 * 128;
        const int n =
            a.G * ((seq.ql - seq.first_row(r0) + E::rows - 1) / E::rows);
        parts = parts_of(sk, n);
        const size_t index = (size_t)head * ((a.Nk + 127) / 128) + j / 128;
        from = sk.o + index * sk.splits * 256 * D + c * 128 + (j - r0) * 8;
        step = 256 * D;
        to = (uint16_t *)a.dk + row * D + c;
    }
    if (parts == 1) return;
    for (int which = 0; which < (keys ? 2 : 1); ++which) {
        float x[8] = {};
        for (int p = 0; p < parts; ++p) {
            const float4 *y = reinterpret_cast<const float4 *>(
                from + p * step + which * 128 * D);
            const float4 u = y[0], v = y[1];
            const float e[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] += e[i];
        }
        const float f = which ? 1.0f : a.scale;
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            y[i] = pack_bf16x2(x[2 * i] * f, x[2 * i + 1] * f);
        if (which) to = (uint16_t *)a.dv + row * D + c;
        *reinterpret_cast<uint4 *>(to) = make_uint4(y[0], y[1], y[2], y[3]);
    }
}

struct Maps {
    CUtensorMap q, g, k, v;
};
// q_rows, k_rows: of the tiles of Q and dO, of K and V
cudaError_t make_maps(const ExactView &a, int q_rows, int k_rows, Maps *m) {
    const uint64_t nq = (uint64_t)a.B * a.H * a.Nq;
    const uint64_t nk = (uint64_t)a.B * a.Hkv * a.Nk;
    cudaError_t e = make_tma_map_bf16(&m->q, a.q, nq, a.d, q_rows);
    if (e == cudaSuccess) e = make_tma_map_bf16(&m->g, a.d_o, nq, a.d, q_rows);
    if (e == cudaSuccess) e = make_tma_map_bf16(&m->k, a.k, nk, a.d, k_rows);
    if (e == cudaSuccess) e = make_tma_map_bf16(&m->v, a.v, nk, a.d, k_rows);
    return e;
}
int sm_count() {
    int dev = 0, sms = 152;
    if (cudaGetDevice(&dev) == cudaSuccess)
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    return sms;
}
template <typename F>
cudaError_t by_width(int d, F f) {
    return d == 128  ? f(std::integral_constant<int, 128>{})
           : d == 64 ? f(std::integral_constant<int, 64>{})
                     : f(std::integral_constant<int, 32>{});
}

}  // namespace

cudaError_t launch_exact_delta(const ExactView &a, int *counters,
                               cudaStream_t st) {
    const long threads = (long)a.B * a.H * a.Nq * (a.d / 8);
    return by_width(a.d, [&](auto dim) {
        return launch_after(k_exact_delta<decltype(dim)::value>,
                            dim3((unsigned)((threads + 255) / 256)), 256, 0,
                            st, a, counters);
    });
}

namespace {

// Parts of a walk of at most n tiles: one and a half for each place for a CTA (a
// GB300 has 152 SMs) when the items fill less than half of them; two of long
// walks when there are fewer items than places, since with causal = 1 the
// longest walk is twice the average. Otherwise none, as what parts leave is
// written and read again. B1 H8 H_kv1 N2048 d64 (16 items of dK, dV): the
// backward pass takes 60 us, undivided 238; B64 H8 H_kv2 N256 d64 (256 items,
// walks of 16 tiles) 52 undivided, 69 in three parts. (By the sizes alone: the
// workspace does not depend on the device.)
int divide_walks(long items, long n, int d) {
    const long places = 152 * (d > 64 ? 1 : 2);
    long parts = 1;
    if (items < places / 2)
        parts = (places * 3 / 2 + items - 1) / items;
    else if (items < places && n >= 32)
        parts = 2;
    if (parts > n / kEbLeast) parts = n / kEbLeast;
    return parts < 1 ? 1 : (int)parts;
}
// of the walks over keys (dQ) and over query rows (dK, dV)
int query_parts(const ExactView &a, const ExactOrder &order) {
    const int rows = a.d > 64 ? 128 : 64;
    return divide_walks(order.items(a), ((long)a.Nk + rows - 1) / rows, a.d);
}
long key_items(const ExactView &a) {
    return (long)((a.Nk + 127) / 128) * a.B * a.Hkv;
}
int key_parts(const ExactView &a) {
    const int rows = a.d > 64 ? 128 : 64;
    return divide_walks(key_items(a), a.G * (((long)a.Nq + rows - 1) / rows),
                        a.d);
}
// Floats that the parts of dK, dV and of dQ leave.
size_t key_floats(const ExactView &a) {
    const int parts = key_parts(a);
    return parts > 1 ? (size_t)key_items(a) * parts * 256 * a.d : 0;
}
size_t query_floats(const ExactView &a, bool padded) {
    const ExactOrder order(a, 128, padded);
    const int parts = query_parts(a, order);
    return parts > 1 ? (size_t)order.items(a) * parts * 128 * a.d : 0;
}
EbSplit key_split(const ExactView &a, float *part) {
    return EbSplit{key_parts(a), part};
}
EbSplit query_split(const ExactView &a, float *part) {
    return EbSplit{query_parts(a, ExactOrder(a, 128)), part + key_floats(a)};
}

}  // namespace

size_t exact_part_bytes(const ExactView &a) {
    // with and without q_len, which the workspace's size does not know of
    const size_t x = query_floats(a, false), y = query_floats(a, true);
    return sizeof(float) * (key_floats(a) + (x > y ? x : y));
}

cudaError_t launch_exact_dq_tc(const ExactView &a, int *next_item, int *far,
                               float *part, cudaStream_t st) {
    const ExactOrder order(a, 128);
    const EbSplit split = query_split(a, part);
    const long items = order.items(a) * split.splits;
    return by_width(a.d, [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        using E = Eb<D>;
        const long most = (long)sm_count() * E::ctas;
        Maps m;
        const cudaError_t e = make_maps(a, 128, E::rows, &m);
        if (e != cudaSuccess) return e;
        const size_t smem =
            1024 + 2 * E::held + (size_t)(kDqK<D> + kDqV<D>) * E::tile;
        return launch_after(
            k_exact_dq_tc<D>, dim3((unsigned)(items < most ? items : most)),
            E::threads, smem, st, m.q, m.g, m.k, m.v, a, order, split,
            (int)items, next_item, far);
    });
}

cudaError_t launch_exact_dkv_tc(const ExactView &a, int *next_item,
                                const int *far, float *part,
                                cudaStream_t st) {
    const EbSplit split = key_split(a, part);
    const long items = key_items(a) * split.splits;
    return by_width(a.d, [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        using E = Eb<D>;
        const long most = (long)sm_count() * E::ctas;
        Maps m;
        const cudaError_t e = make_maps(a, E::rows, 128, &m);
        if (e != cudaSuccess) return e;
        constexpr size_t smem =
            2 * E::held + (size_t)(Dkv<D>::kQ + Dkv<D>::kG) * E::tile +
            sizeof(DkvShared<D>);
        static_assert(smem <= 232448, "shared memory of a CTA");
        return launch_after(
            k_exact_dkv_tc<D>, dim3((unsigned)(items < most ? items : most)),
            E::threads, smem, st, m.q, m.g, m.k, m.v, a, split, (int)items,
            next_item, (const volatile int *)far);
    });
}

cudaError_t launch_exact_sum(const ExactView &a, float *part,
                             cudaStream_t st) {
    const EbSplit sq = query_split(a, part), sk = key_split(a, part);
    long rows = sq.splits > 1 ? (long)a.B * a.H * a.Nq : 0;
    if (sk.splits > 1) rows += (long)a.B * a.Hkv * a.Nk;
    if (rows == 0) return cudaSuccess;
    const long threads = (rows + 7) / 8 * a.d;  // 8 rows a warp
    return by_width(a.d, [&](auto dim) {
        return launch_after(k_exact_sum<decltype(dim)::value>,
                            dim3((unsigned)((threads + 255) / 256)), 256, 0,
                            st, a, ExactOrder(a, 128), sq, sk);
    });
}

}  // namespace elsaa
