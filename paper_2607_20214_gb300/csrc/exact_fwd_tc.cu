// Exact attention on the tensor cores (include/elsaa_exact.h), bf16: one pass
// over the keys with the running maximum and sum of the softmax.
//
// The query rows of the heads that share a K/V head are counted through (row r
// is row r mod N of head r / N), so that a tile of short sequences is filled by
// several heads. An item is 256 such rows, two slots of 128, over the keys that
// they see; the slots share every key and value tile. Roles:
//   warps 0-3, 4-7  softmax of slot 0 / 1: one thread per query row holds all
//                   128 scores of a key tile in registers, so neither the row
//                   maximum nor the sum needs another thread
//   warp 8          issues the products: S = Q K^T, O += P V (P from TMEM); for
//                   D <= 64 those of slot 0, and warp 9 those of slot 1
//   warp 10         takes the items, TMA loads of Q and K; warp 11 loads V
// With few items every CTA gets an equal share of all key tiles instead, in
// order, and k_exact_merge joins what the CTAs of a divided item leave.
// TMEM: S_s at 128 s, O_s at 256 + 128 s, P_s behind O_s for D <= 64, over S_s
// at D = 128. O stays in tensor memory; a softmax warp rescales it when the
// maximum of one of its rows has grown much.
//
// What bounds it: at D = 128 the products, 2048 of a tile's 2900 clocks (256 rows,
// 128 keys), and the steps of a slot between them, of which the softmax takes
// 1260: B1 H16 H_kv4 N16384 causal 0.71 ms, 1.56 PFLOP/s, 0.81 of the measured bf16
// rate. For D <= 64 the waits between a slot's steps, no pipe is full: B4 H12 N4096
// d64 without a mask 200 us, 1.03 PFLOP/s.
#include <algorithm>
#include <type_traits>

#include "device_common.cuh"
#include "exact.h"
#include "tc_common.cuh"
#include "tc_race.cuh"

namespace elsaa {

namespace {

using namespace tc;

// 384 x 168 registers at launch = 256 x 200 (softmax) + 128 x 104
constexpr int kEfThreads = 384;
constexpr int kEfRegsSoft = 200, kEfRegsOther = 104;
static_assert(256 * kEfRegsSoft + 128 * kEfRegsOther <= kEfThreads * 168,
              "register shares within the launch's total");
// O is rescaled when the maximum of one of a warp's rows has grown by more than
// this (base 2) since it last was: weights are up to 2^8, which costs neither
// them nor their sum any precision, but for the largest, which bf16 then rounds
// too. Rescaling for every new maximum: 753 us instead of 710 (B1 H16 H_kv4
// N16384 d128 causal), since among 32 rows there is one in nearly every tile.
constexpr float kGrown = 8.0f;
// Scores go ahead of the last tile's P V product, as soon as the softmax has
// read the scores before them, where they do not lie over P; each slot's
// products then have a warp of their own. B4 H12 N4096 d64 causal: 125 us
// without, 114 with. (At D = 128 two warps let the slots' products run mixed,
// each of them later: B1 H16 H_kv4 N16384 735 us instead of 703.)
template <int D>
constexpr bool kEfAhead = D <= 64;
// Key and value tiles held.
template <int D>
constexpr int kEfK = D > 64 ? 3 : 4;
template <int D>
constexpr int kEfV = D > 64 ? 2 : 4;
// a score (base 2) of this or less counts as -inf
constexpr float kLowest = -1e38f;
// The reference of a row's weights is a rounded product, score * sl2, and
// fma(score, sl2, -reference) does not round it: the largest weight comes out
// as 2^d, d up to half a unit in the reference's last place. Up to 2^24 that is
// 2^0.5, which the sum of the weights takes out again; behind 2^31 the weights
// would overflow, or none be left. A warp that meets a reference behind 2^24
// goes on in a second loop, where such rows have the reference's score
// subtracted from the others before the product. The vote that it takes costs
// 1 % (B1 H16 H_kv4 N16384 d128 causal 699 -> 707 us; single rows of 16384 keys
// 101 -> 106); the subtraction in the same loop, behind a branch, 2 (715), and
// padded chunks of 500 rows 61 instead of 57.
constexpr float kFar = 16777216.0f;

template <int D>
struct EfBars {
    uint64_t item_full[2], item_empty[2], q_full[2], q_empty[2];
    uint64_t k_full[kEfK<D>], k_empty[kEfK<D>];
    uint64_t v_full[kEfV<D>], v_empty[kEfV<D>];
    uint64_t s_full[2], s_read[2], p_half[2], p_full[2];
    uint64_t o_done[2], o_empty[2];
};

// How long a slot's softmax waits for its next item: as long as the other slot
// may take for its own, which can have 2^23 tiles more (2^30 keys; a tile takes
// 1.2 to 1.8 us). The CTA's other waits are of kWaitLimitNs, and end this one.
constexpr unsigned long long kEfItemNs = 30 * kWaitLimitNs;

// What the roles know of an item.
struct EfItem {
    int item;   // -1: no more
    int b, kvh, r0;
    int ql, kl;
    int kt0;    // the first key tile
    int n[2];   // key tiles of each slot, from kt0 on
    int part;   // where a divided item's sums go, -1: the item is whole
};

// Shares. The items of a K/V head in their order, of all heads of a sequence,
// of all sequences make one row of units: kEfHead for an item (what it costs
// beside its tiles) and one for each of its key tiles (of 256 rows). CTA c of C
// takes units [W c / C, W (c + 1) / C) of the W. Of an item that is divided,
// every CTA leaves 256 rows of sums of e^(z - m) v in o[part][D / 8][row][8] and
// (m, sum of e^(z - m)) in ml[part][row], z and m base 2: part 2 c + 1 of the
// CTA that begins it, part 2 c of the others. rec[c] tells k_exact_merge of
// the item that CTA c begins.
constexpr int kEfHead = 2;
constexpr int kEfLeast = 6;     // units of a share at least, on average
constexpr int kEfCtas = 152;    // one for each SM of a GB300
constexpr int kEfMaxB = 256;
struct EfRecord {
    int b, kvh, r0, last;  // last: the CTA that ends it, -1: none
};
struct EfShares {
    int on, tiles;  // tiles: items of a K/V head
    float *o;
    float2 *ml;
    EfRecord *rec;
};

// Units of item t of sequence `seq`, none if it has no row.
__device__ __forceinline__ int ef_weight(const ExactSeq &seq,
                                         const ExactOrder &batch, int t) {
    const ExactOrder order = batch.of(seq.ql);
    if (t >= order.groups * order.per) return 0;
    const int r0 = order.tile(t) * 256, r1 = min(r0 + 256, order.rows);
    if (r0 >= r1 || seq.ql == 0) return 0;
    if (r0 / order.pitch == (r1 - 1) / order.pitch &&
        r0 % order.pitch >= seq.ql)
        return 0;
    return kEfHead + (exact_most(seq, r0, r1, order.pitch) + 127) / 128;
}

template <int D>
__global__ void __launch_bounds__(kEfThreads, 1)
    k_exact_fwd_tc(const __grid_constant__ CUtensorMap tmQ,
                   const __grid_constant__ CUtensorMap tmK,
                   const __grid_constant__ CUtensorMap tmV,
                   const __grid_constant__ ExactView a,
                   const __grid_constant__ EfShares shares,
                   const __grid_constant__ ExactOrder order, int items,
                   int *__restrict__ next_item) {
    wait_for_stream();
    extern __shared__ unsigned char smem_raw[];
    __shared__ EfBars<D> bars;
    __shared__ uint32_t tbase;
    __shared__ int abort_flag;
    __shared__ EfItem item_s[2];
    volatile int *abort = &abort_flag;
    // a row is D <= 64 elements of one 128-byte line, or two lines
    constexpr int kPanels = D > 64 ? 2 : 1;
    constexpr uint32_t kTileB = kPanels * 16384;
    const int tid = threadIdx.x, warp = tid >> 5, lane_id = tid & 31;
    const uint32_t sQ = align1k(smem_u32(smem_raw));
    constexpr int kK = kEfK<D>, kV = kEfV<D>;
    constexpr bool kAhead = kEfAhead<D>;
    const uint32_t sK = sQ + 2 * kTileB, sV = sK + kK * kTileB;
    DeviceStatus *status = a.status;

    // units of all heads of the sequences up to b
    __shared__ int upto[kEfMaxB];
    if (!next_item && blockIdx.x == 0 && tid < 4)
        (&status->code)[tid] = 0;  // a wait runs out much later
    if (shares.on) {
        for (int b = tid; b < a.B; b += kEfThreads) upto[b] = 0;
        __syncthreads();
        for (int i = tid; i < a.B * shares.tiles; i += kEfThreads) {
            const int b = i / shares.tiles;
            const int w =
                ef_weight(ExactSeq(a, b), order, i - b * shares.tiles);
            if (w) atomicAdd(&upto[b], w * a.Hkv);
        }
        __syncthreads();
        if (warp == 0) {
            int sum = 0;
            for (int b = lane_id; b - lane_id < a.B; b += 32) {
                int x = b < a.B ? upto[b] : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, x, o);
                    if (lane_id >= o) x += y;
                }
                x += sum;
                if (b < a.B) upto[b] = x;
                sum = __shfl_sync(0xffffffffu, x, 31);
            }
        }
    }
    if (warp == 8) tmem_alloc(&tbase, 512);
    if (tid == 0) {
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars.item_full[s], 1);
            // warps 0-8 and 11, and 9 where it issues products
            mbar_init(&bars.item_empty[s], 10 + kAhead);
            mbar_init(&bars.q_full[s], 1);
            mbar_init(&bars.q_empty[s], 1);
            mbar_init(&bars.s_full[s], 1);
            mbar_init(&bars.s_read[s], 4);
            mbar_init(&bars.p_half[s], 4);
            mbar_init(&bars.p_full[s], 4);
            mbar_init(&bars.o_done[s], 1);
            mbar_init(&bars.o_empty[s], 4);
        }
        for (int s = 0; s < kK; ++s) {
            mbar_init(&bars.k_full[s], 1);
            mbar_init(&bars.k_empty[s], 1 + kAhead);
        }
        for (int s = 0; s < kV; ++s) {
            mbar_init(&bars.v_full[s], 1);
            mbar_init(&bars.v_empty[s], 1 + kAhead);
        }
        abort_flag = 0;
        fence_mbar_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tm = tbase;

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(
            kEfRegsOther));
        // a tile of K or V
        auto load = [&](uint64_t *full, uint64_t *empty, int c, int stages,
                        uint32_t dst, const CUtensorMap *map, int row,
                        int site) {
            const int st = c % stages;
            if (c >= stages &&
                !mbar_wait_or_abort(&empty[st], (c / stages - 1) & 1, abort,
                                    status, site))
                return false;
            mbar_expect_tx(&full[st], kTileB);
            for (int p = 0; p < kPanels; ++p)
                tma_load_2d(dst + st * kTileB + p * 16384, map, 64 * p, row,
                            &full[st]);
            return true;
        };
        // of warp 10: where its share begins and how long it is
        int sb = 0, skvh = 0, st = 0, at = 0, rest = 0;
        long W = 0;
        int C = 1;
        if (shares.on && warp == 10) {
            W = upto[a.B - 1];
            C = (int)min((long)gridDim.x, max(1L, W / kEfLeast));
            if (blockIdx.x < C) {
                int u = (int)(W * blockIdx.x / C);
                rest = (int)(W * (blockIdx.x + 1) / C) - u;
                while (sb < a.B - 1 && upto[sb] <= u) ++sb;
                if (sb > 0) u -= upto[sb - 1];
                const int head =
                    max(1, (upto[sb] - (sb > 0 ? upto[sb - 1] : 0)) / a.Hkv);
                skvh = u / head;
                u -= skvh * head;
                const ExactSeq seq(a, sb);
                for (;; st += 32) {
                    int x = st + lane_id < shares.tiles
                                ? ef_weight(seq, order, st + lane_id)
                                : 0;
                    const int own = x;
#pragma unroll
                    for (int o = 1; o < 32; o <<= 1) {
                        const int y = __shfl_up_sync(0xffffffffu, x, o);
                        if (lane_id >= o) x += y;
                    }
                    const uint32_t past =
                        __ballot_sync(0xffffffffu, x > u);
                    if (past || st + 32 >= shares.tiles) {
                        const int k = past ? __ffs(past) - 1 : 31;
                        at = u - __shfl_sync(0xffffffffu, x - own, k);
                        st += k;
                        break;
                    }
                    u -= __shfl_sync(0xffffffffu, x, 31);
                }
            }
        }
        if (warp == 10 && lane_id == 0) {
            // ------------------------------------ items, loads of Q and K
            int c = 0;   // key tiles loaded so far
            int qs[2] = {0, 0};  // items whose queries were loaded
            bool ok = true;
            const int heads = a.B * a.Hkv;
            EfRecord rec = {0, 0, 0, -1};
            long unit = W * blockIdx.x / C;
            // the next item, of key tiles [kt0, kt1)
            auto fill = [&](EfItem &w, int b, int kvh, int t, int kt0,
                            int kt1) {
                w.item = 0;
                w.b = b;
                w.kvh = kvh;
                w.kt0 = kt0;
                w.part = -1;
                const ExactSeq seq(a, b);
                w.ql = seq.ql;
                w.kl = seq.kl;
                const ExactOrder own = order.of(seq.ql);
                w.r0 = (t < own.groups * own.per ? own.tile(t)
                                                 : own.groups * own.per) * 256;
                for (int s = 0; s < 2; ++s) {
                    const int r = w.r0 + 128 * s;
                    const int n = (exact_most(seq, r, min(r + 128, own.rows),
                                              own.pitch) + 127) / 128;
                    w.n[s] = max(0, min(n, kt1) - kt0);
                }
            };
            auto next_share = [&](EfItem &w) {
                while (rest > 0) {
                    const int t = st, b = sb, kvh = skvh, a0 = at;
                    const int all = ef_weight(ExactSeq(a, b), order, t);
                    const int a1 = min(all, a0 + rest);
                    const long begin = unit - a0;  // of the item
                    rest -= a1 - a0;
                    unit += a1 - a0;
                    at = 0;
                    if (++st == shares.tiles) {
                        st = 0;
                        if (++skvh == a.Hkv) {
                            skvh = 0;
                            // the next sequence that has rows (the last
                            // one's end is that of the last share)
                            while (sb < a.B - 1) {
                                ++sb;
                                if (upto[sb] != upto[sb - 1]) break;
                            }
                        }
                    }
                    if (all == 0) continue;
                    const int kt0 = max(a0 - kEfHead, 0);
                    const int kt1 = max(a1 - kEfHead, 0);
                    // nothing of it but its head, unless it has no more
                    if (kt0 == kt1 && (all > kEfHead || a0 > 0)) continue;
                    fill(w, b, kvh, t, kt0, kt1);
                    if (all > kEfHead) {
                        const int first =
                            (int)range_owner(begin + kEfHead, W, C);
                        const int last =
                            (int)range_owner(begin + all - 1, W, C);
                        if (first != last) {
                            w.part = 2 * (int)blockIdx.x;
                            if (first == (int)blockIdx.x) {
                                ++w.part;
                                rec = {b, kvh, w.r0, last};
                            }
                        }
                    }
                    return true;
                }
                return false;
            };
            // An item is drawn when the last one's key tiles are on their way:
            // earlier, and the longest items' CTAs draw others that they come
            // to late (B1 H16 H_kv4 N4096 d128 causal: 83 us instead of 58).
            bool begun = false;
            auto next = [&]() {
                EfItem w = {-1};
                if (shares.on) {
                    if (!next_share(w)) w.item = -1;
                    return w;
                }
                const long item = !begun      ? blockIdx.x
                                  : next_item ? (long)gridDim.x +
                                                    atomicAdd(next_item, 1)
                                              : items;
                begun = true;
                if (item < items) {
                    // the last rows of every query head, which see most,
                    // first
                    const int h = (int)item % heads, t = (int)item / heads;
                    fill(w, h / a.Hkv, h % a.Hkv, t, 0, 1 << 30);
                }
                return w;
            };
            for (int it = 0; ok; ++it) {
                const EfItem w = next();
                if (it >= 2 && !mbar_wait_or_abort(&bars.item_empty[it & 1],
                                                   ((it >> 1) - 1) & 1, abort,
                                                   status, 400))
                    break;
                item_s[it & 1] = w;
                mbar_arrive(&bars.item_full[it & 1]);
                if (w.item < 0) break;
                const int nk = max(w.n[0], w.n[1]);
                const int q0 = (w.b * a.H + w.kvh * a.G) * a.Nq;
                const int k0 =
                    (w.b * a.Hkv + w.kvh) * a.Nk + 128 * w.kt0;
                const ExactOrder own = order.of(w.ql);
                int kt = 0;
                for (int s = 0; s < 2 && ok; ++s) {
                    if (w.n[s] == 0) continue;
                    ok = qs[s] == 0 ||
                         mbar_wait_or_abort(&bars.q_empty[s], (qs[s] - 1) & 1,
                                            abort, status, 401);
                    if (!ok) break;
                    ++qs[s];
                    mbar_expect_tx(&bars.q_full[s], kTileB);
                    for (int p = 0; p < kPanels; ++p)
                        tma_load_2d(sQ + s * kTileB + p * 16384, &tmQ, 64 * p,
                                    q0 + own.row(w.r0 + 128 * s, a.Nq),
                                    &bars.q_full[s]);
                    if (kt == 0) {
                        ok = load(bars.k_full, bars.k_empty, c, kK, sK, &tmK,
                                  k0, 402);
                        ++kt;
                        ++c;
                    }
                }
                for (; kt < nk && ok; ++kt, ++c)
                    ok = load(bars.k_full, bars.k_empty, c, kK, sK, &tmK,
                              k0 + 128 * kt, 402);
            }
            if (shares.on) shares.rec[blockIdx.x] = rec;
        } else if (warp == 11 && lane_id == 0) {
            // ------------------------------------------------ loads of V
            int c = 0;
            bool ok = true;
            for (int it = 0; ok; ++it) {
                if (!mbar_wait_or_abort(&bars.item_full[it & 1], (it >> 1) & 1,
                                        abort, status, 403))
                    break;
                const EfItem w = item_s[it & 1];
                mbar_arrive(&bars.item_empty[it & 1]);
                if (w.item < 0) break;
                const int nk = max(w.n[0], w.n[1]);
                const int k0 =
                    (w.b * a.Hkv + w.kvh) * a.Nk + 128 * w.kt0;
                for (int kt = 0; kt < nk && ok; ++kt, ++c)
                    ok = load(bars.v_full, bars.v_empty, c, kV, sV, &tmV,
                              k0 + 128 * kt, 411);
            }
        } else if (kAhead && warp < 10) {
            // --------------------------------------- MMA issue of one slot
            const int s = warp - 8;
            const bool el = elect_one();
            auto wait = [&](uint64_t *bar, uint32_t par, int site) -> bool {
                if (__all_sync(0xffffffffu, mbar_test(bar, par))) return true;
                return __all_sync(0xffffffffu,
                                  mbar_wait_or_abort(bar, par, abort, status,
                                                     site));
            };
            const uint32_t id_s = idesc_bf16(128, 128, false, false);
            const uint32_t id_o = idesc_bf16(128, D, false, true);
            const uint64_t dQ = smem_desc(sQ + s * kTileB, 16, 1024);
            const uint64_t dK = smem_desc(sK, 16, 1024);
            const uint64_t dV = smem_desc(sV, 16384, 1024);
            const uint32_t tS = tm + 128 * s, tO = tS + 256, tP = tO + 64;
            int c = 0;          // key tiles before
            int g = 0, go = 0;  // tiles and items that this slot had
            bool ok = true;
            for (int it = 0; ok; ++it) {
                if (!wait(&bars.item_full[it & 1], (it >> 1) & 1, 380)) break;
                const EfItem &w = item_s[it & 1];
                const int item = w.item, n = w.n[s];
                const int nk = max(w.n[0], w.n[1]);
                const int part = w.kl - 128 * (w.kt0 + nk - 1);
                __syncwarp();
                if (el) mbar_arrive(&bars.item_empty[it & 1]);
                if (item < 0) break;
                if (nk == 0) continue;
                auto scores = [&](int kt) {
                    const int st = (c + kt) % kK;
                    if (!wait(&bars.k_full[st], (c + kt) / kK & 1, 382))
                        return false;
                    tc_fence_after();
                    const uint64_t k = desc_at(dK, st * kTileB);
                    if (el) {
#pragma unroll
                        for (int x = 0; x < D / 16; ++x)
                            mma_ss(tS, dQ + 2 * x, k + 2 * x, id_s, x > 0);
                        mma_commit(&bars.s_full[s]);
                        mma_commit(&bars.k_empty[st]);
                        if (kt + 1 == n) mma_commit(&bars.q_empty[s]);
                    }
                    return true;
                };
                if (n > 0) {
                    ok = wait(&bars.q_full[s], go & 1, 381) && scores(0) &&
                         (go == 0 ||
                          wait(&bars.o_empty[s], (go - 1) & 1, 383));
                    ++go;
                }
                for (int kt = 0; kt < n && ok; ++kt, ++g) {
                    const int st = (c + kt) % kV;
                    if (kt + 1 < n)
                        ok = wait(&bars.s_read[s], g & 1, 384) &&
                             scores(kt + 1);
                    ok = ok && wait(&bars.v_full[st], (c + kt) / kV & 1, 385);
                    if (!ok) break;
                    if (kt == nk - 1 && part < 128) {
                        // (both slots write the same zeros)
                        const uint32_t x = sV + st * kTileB;
                        for (int i = part * 8 + lane_id; i < 1024; i += 32)
                            st_shared_zero16(x + i * 16);
                        fence_proxy_async_smem();
                        __syncwarp();
                    }
                    const uint64_t v = desc_at(dV, st * kTileB);
                    ok = wait(&bars.p_half[s], g & 1, 386);
                    if (!ok) break;
                    tc_fence_after();
                    if (el) {
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            mma_ts(tO, tP + 8 * x, v + 128 * x, id_o,
                                   x > 0 || kt > 0);
                    }
                    ok = wait(&bars.p_full[s], g & 1, 387);
                    if (!ok) break;
                    tc_fence_after();
                    if (el) {
#pragma unroll
                        for (int x = 4; x < 8; ++x)
                            mma_ts(tO, tP + 8 * x, v + 128 * x, id_o, 1u);
                        mma_commit(&bars.o_done[s]);
                        mma_commit(&bars.v_empty[st]);
                    }
                }
                // tiles that only the other slot has
                for (int kt = n; kt < nk && ok; ++kt) {
                    const int ks = (c + kt) % kK, vs = (c + kt) % kV;
                    ok = wait(&bars.k_full[ks], (c + kt) / kK & 1, 388);
                    if (!ok) break;
                    if (el) mbar_arrive(&bars.k_empty[ks]);
                    ok = wait(&bars.v_full[vs], (c + kt) / kV & 1, 389);
                    if (!ok) break;
                    if (el) mbar_arrive(&bars.v_empty[vs]);
                }
                c += nk;
            }
        } else if (!kAhead && warp == 8) {
            // ---------------------------------------------------- MMA issue
            // Whenever half of a slot's P is ready: that half of its P V
            // product; then the other half, and right behind it the scores of
            // its next key tile; the softmax sees these only when both are
            // complete (a commit covers all that was issued before it). The
            // scores go over P, which relies on products of one thread
            // running in the order of their issue.
            // The whole warp runs the loop, so that its state and the
            // operands' descriptors are warp-uniform; one lane issues.
            const bool el = elect_one();
            auto test = [&](uint64_t *bar, uint32_t par) -> bool {
                return __all_sync(0xffffffffu, mbar_test(bar, par));
            };
            auto wait = [&](uint64_t *bar, uint32_t par, int site) -> bool {
                return __all_sync(0xffffffffu,
                                  mbar_wait_or_abort(bar, par, abort, status,
                                                     site));
            };
            const uint32_t id_s = idesc_bf16(128, 128, false, false);
            const uint32_t id_o = idesc_bf16(128, D, false, true);
            const uint64_t dQ = smem_desc(sQ, 16, 1024);
            const uint64_t dK = smem_desc(sK, 16, 1024);
            const uint64_t dV = smem_desc(sV, 16384, 1024);
            constexpr uint32_t kTile = kTileB >> 4;  // in descriptor units
            int c0 = 0;                // key tiles of earlier items
            int gp0 = 0, gp1 = 0;      // P V products issued per slot
            int go0 = 0, go1 = 0;      // items finished per slot
            bool ok = true;
            for (int it = 0; ok; ++it) {
                ok = wait(&bars.item_full[it & 1], (it >> 1) & 1, 404);
                if (!ok) break;
                const EfItem w = item_s[it & 1];
                __syncwarp();
                if (el) mbar_arrive(&bars.item_empty[it & 1]);
                if (w.item < 0) break;
                const int n0 = w.n[0], n1 = w.n[1], nk = max(n0, n1);
                if (nk == 0) continue;
                int us0 = 0, us1 = 0, up0 = 0, up1 = 0;
                // keys of the last tile that the sequence has: values of
                // others count with weights of 0 and must be numbers
                int part = w.kl - 128 * (w.kt0 + nk - 1);
                bool half0 = false, half1 = false;  // P V begun
                // the scores of slot s's next key tile
                auto scores = [&](auto slot, int &us, int n, int us_o,
                                  int n_o) {
                    constexpr int s = decltype(slot)::value;
                    const int st = (c0 + us) % kK;
                    if (!wait(&bars.k_full[st], (c0 + us) / kK & 1,
                              406))
                        return false;
                    tc_fence_after();
                    const uint64_t q = dQ + s * kTile, k = dK + st * kTile;
                    if (el) {
#pragma unroll
                        for (int x = 0; x < D / 16; ++x) {
                            const uint32_t o = (x >> 2) * 1024 + (x & 3) * 2;
                            mma_ss(tm + 128u * s, q + o, k + o, id_s, x > 0);
                        }
                        mma_commit(&bars.s_full[s]);
                        // both slots have used the tile
                        if (us >= n_o || us_o > us)
                            mma_commit(&bars.k_empty[st]);
                        if (us + 1 == n) mma_commit(&bars.q_empty[s]);
                    }
                    ++us;
                    return true;
                };
                auto step = [&](auto slot, int &us, int &up, bool &half,
                                int &gp, int go, int n, int us_o, int up_o,
                                int n_o) {
                    constexpr int s = decltype(slot)::value;
                    constexpr uint32_t cO = 128u * s + 256u;
                    constexpr uint32_t cP = 128u * s;
                    const int st = (c0 + up) % kV;
                    if (up == us) return false;
                    const uint64_t v = dV + st * kTile;
                    if (!half) {
                        // the tests side by side, then one vote
                        const bool ready =
                            mbar_test(&bars.p_half[s], gp & 1) &
                            mbar_test(&bars.v_full[st], (c0 + up) / kV & 1) &
                            (up > 0 || go == 0 ||
                             mbar_test(&bars.o_empty[s], (go - 1) & 1));
                        if (!__all_sync(0xffffffffu, ready)) return false;
                        if (up == nk - 1 && part < 128) {
                            const uint32_t x = sV + st * kTileB;
                            for (int i = part * 8 + lane_id; i < 1024;
                                 i += 32)
                                for (int p = 0; p < kPanels; ++p)
                                    st_shared_zero16(x + p * 16384 + i * 16);
                            part = 128;  // once for both slots
                            fence_proxy_async_smem();
                            __syncwarp();
                        }
                        tc_fence_after();
                        const uint32_t more = up > 0;
                        if (el) {
#pragma unroll
                            for (int x = 0; x < 4; ++x)
                                mma_ts(tm + cO, tm + cP + 8 * x, v + 128 * x,
                                       id_o, x > 0 ? 1u : more);
                        }
                        half = true;
                        if (!test(&bars.p_full[s], gp & 1)) return true;
                    } else if (!test(&bars.p_full[s], gp & 1)) {
                        return false;
                    }
                    half = false;
                    tc_fence_after();
                    if (el) {
#pragma unroll
                        for (int x = 4; x < 8; ++x)
                            mma_ts(tm + cO, tm + cP + 8 * x, v + 128 * x, id_o,
                                   1u);
                        mma_commit(&bars.o_done[s]);
                        if (up >= n_o || up_o > up)
                            mma_commit(&bars.v_empty[st]);
                    }
                    ++up;
                    ++gp;
                    if (us < n) ok = scores(slot, us, n, us_o, n_o);
                    return true;
                };
                using S0 = std::integral_constant<int, 0>;
                using S1 = std::integral_constant<int, 1>;
                if (n0 > 0)
                    ok = wait(&bars.q_full[0], go0 & 1, 405) &&
                         scores(S0{}, us0, n0, us1, n1);
                if (ok && n1 > 0)
                    ok = wait(&bars.q_full[1], go1 & 1, 418) &&
                         scores(S1{}, us1, n1, us0, n0);
                unsigned long long t_last = 0;
                uint32_t idle = 0;
                while (ok && (up0 < n0 || up1 < n1)) {
                    const bool x = step(S0{}, us0, up0, half0, gp0, go0, n0,
                                        us1, up1, n1);
                    const bool y = ok && step(S1{}, us1, up1, half1, gp1, go1,
                                              n1, us0, up0, n0);
                    if (x || y) {
                        idle = 0;
                    } else if ((++idle & 255u) == 0) {
                        if (idle == 256u) t_last = global_ns();
                        const bool late = global_ns() - t_last > kWaitLimitNs;
                        if (late) {
                            *abort = 1;
                            record_timeout(status, 407);
                        }
                        ok = !__any_sync(0xffffffffu, late || *abort);
                    }
                }
                c0 += nk;
                go0 += n0 > 0;
                go1 += n1 > 0;
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------- softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kEfRegsSoft));
        const int s = warp >> 2, row = (warp & 3) * 32 + lane_id;
        const uint32_t lane = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tm + lane + 128u * s, tO = tS + 256u;
        const uint32_t tP = D <= 64 ? tO + 64 : tS;
        const float sl2 = a.scale * kLog2e;
        const float2 sl22 = make_float2(sl2, sl2);
        auto wwait = [=](uint64_t *bar, uint32_t par, int site) {
            return __all_sync(0xffffffffu,
                              mbar_wait_or_abort(bar, par, abort, status,
                                                 site));
        };
        // what the warp did in tensor memory comes before the products that
        // wait for the barrier
        auto warp_done = [=](uint64_t *bar) {
            tc_fence_before();
            __syncwarp();
            if (lane_id == 0) mbar_arrive(bar);
        };
        int g = 0;  // key tiles of this slot so far
        bool ok = true;
        for (int it = 0; ok; ++it) {
            ok = __all_sync(0xffffffffu,
                            mbar_wait_or_abort_for(
                                kEfItemNs, &bars.item_full[it & 1],
                                (it >> 1) & 1, abort, status, 408));
            if (!ok) break;
            const EfItem &w_s = item_s[it & 1];
            const int item = w_s.item, n = w_s.n[s], part = w_s.part;
            const int kt0 = w_s.kt0, wb = w_s.b, kvh = w_s.kvh;
            const int ql = w_s.ql, kl = w_s.kl, slot0 = w_s.r0 + 128 * s;
            __syncwarp();
            if (lane_id == 0) mbar_arrive(&bars.item_empty[it & 1]);
            if (item < 0) break;
            const ExactOrder own = order.of(ql);
            const int r = slot0 + row, i = r % own.pitch;
            const bool valid = r < own.rows && i < ql;
            int seen = 0;
            if (valid)
                seen = a.causal ? max(0, min(kl, i + 1 + kl - ql))
                                : kl;
            // the reference; behind kFar the score that it comes from, else 0
            float mref = kLowest, from = 0.0f, lsum = 0.0f;
            auto refer = [&](float top, float z) {
                mref = fmaxf(z, kLowest);
                from = fabsf(z) > kFar && z > kLowest ? top : 0.0f;
            };
            int kt = 0;
            // key tiles from kt on; without kFarRows up to the one with such a
            // row's reference, which is read again
            auto walk = [&](auto far_rows) {
                constexpr bool kFarRows = decltype(far_rows)::value;
                for (; kt < n; ++kt, ++g) {
                    ok = wwait(&bars.s_full[s], g & 1, 409);
                    if (!ok) break;
                    tc_fence_after();
                    float v[128];
                    {
                        uint32_t x[32], b[32], c[32], e[32];
                        tmem_ld32(tS, x);
                        tmem_ld32(tS + 32, b);
                        tmem_ld32(tS + 64, c);
                        tmem_ld32(tS + 96, e);
                        tmem_wait_ld();
#pragma unroll
                        for (int q = 0; q < 32; ++q) {
                            v[q] = __uint_as_float(x[q]);
                            v[32 + q] = __uint_as_float(b[q]);
                            v[64 + q] = __uint_as_float(c[q]);
                            v[96 + q] = __uint_as_float(e[q]);
                        }
                    }
                    if (kAhead && kFarRows) warp_done(&bars.s_read[s]);
                    const int lim = seen - 128 * (kt0 + kt);
                    if (__any_sync(0xffffffffu, lim < 128)) {
#pragma unroll
                        for (int q = 0; q < 128; ++q)
                            if (q >= lim) v[q] = -INFINITY;
                    }
                    float mx[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
                    for (int q = 4; q < 124; q += 8)
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            mx[x] = max3(mx[x], v[q + 2 * x], v[q + 2 * x + 1]);
                    mx[0] = max3(mx[0], v[124], v[125]);
                    mx[1] = max3(mx[1], v[126], v[127]);
                    const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]);
                    // (rounded by itself, also where it is subtracted)
                    const float z = __fmul_rn(top, sl2);
                    bool need = kt == 0 ? z > -INFINITY : z >= mref + kGrown;
                    if (!kFarRows) {
                        if (__any_sync(0xffffffffu, need && fabsf(z) > kFar))
                            return;
                        if (kAhead) warp_done(&bars.s_read[s]);
                    }
                    if (kt == 0) {
                        if (kFarRows)
                            refer(top, z);
                        else
                            mref = fmaxf(z, kLowest);
                    } else {
                        // P and O are free: the last tile's P V product is
                        // complete (at D = 128 these scores were issued
                        // behind it and it is complete when they are)
                        if (kAhead) {
                            ok = wwait(&bars.o_done[s], (g - 1) & 1, 417);
                            if (!ok) break;
                            tc_fence_after();
                        }
                        float less = mref - z;
                        if (kFarRows && from != 0.0f) {
                            need = top > from;
                            less = (from - top) * sl2;
                        }
                        if (__any_sync(0xffffffffu, need)) {
                            const float f = need ? ex2_approx(less) : 1.0f;
                            const float2 f2 = make_float2(f, f);
#pragma unroll 1
                            for (int c = 0; c < D; c += 32) {
                                uint32_t o[32];
                                tmem_ld32(tO + c, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int q = 0; q < 32; q += 2) {
                                    const float2 y = mul2(
                                        make_float2(__uint_as_float(o[q]),
                                                    __uint_as_float(o[q + 1])),
                                        f2);
                                    o[q] = __float_as_uint(y.x);
                                    o[q + 1] = __float_as_uint(y.y);
                                }
                                tmem_st32(tO + c, o);
                            }
                            lsum *= f;
                            if (need) {
                                if (kFarRows)
                                    refer(top, z);
                                else
                                    mref = z;
                            }
                        }
                    }
                    float nref = -mref;
                    if (kFarRows) {
                        nref = from != 0.0f     ? 0.0f
                               : mref > kLowest ? -mref
                                                : -INFINITY;
#pragma unroll
                        for (int q = 0; q < 128; ++q) v[q] -= from;
                    }
                    const float2 nm = make_float2(nref, nref);
                    float2 ls[2] = {make_float2(0.0f, 0.0f),
                                    make_float2(0.0f, 0.0f)};
#pragma unroll
                    for (int c = 0; c < 128; c += 32) {
                        uint32_t pw[16];
#pragma unroll
                        for (int q = 0; q < 32; q += 2) {
                            const float2 x = fma2(
                                make_float2(v[c + q], v[c + q + 1]), sl22, nm);
                            const float2 p =
                                make_float2(ex2_approx(x.x), ex2_approx(x.y));
                            ls[(q >> 1) & 1] = add2(ls[(q >> 1) & 1], p);
                            pw[q >> 1] = pack_bf16x2(p.x, p.y);
                        }
                        tmem_st16(tP + c / 2, pw);
                        if (c == 32) {
                            tmem_wait_st();
                            warp_done(&bars.p_half[s]);
                        }
                    }
                    lsum += (ls[0].x + ls[1].x) + (ls[0].y + ls[1].y);
                    tmem_wait_st();
                    warp_done(&bars.p_full[s]);
                }
            };
            walk(std::false_type{});
            if (ok && kt < n) walk(std::true_type{});
            if (!ok) break;
            const size_t at =
                (size_t)(wb * a.H + kvh * a.G) * a.Nq + own.row(r, a.Nq);
            uint16_t *o = (uint16_t *)a.out + at * D;
            if (n > 0) {
                ok = wwait(&bars.o_done[s], (g - 1) & 1, 410);
                if (!ok) break;
                tc_fence_after();
            }
            if (part >= 0) {
                const int at_row = 128 * s + row;
                float *y = shares.o + (size_t)part * 256 * D + at_row * 8;
                for (int c = 0; c < D && n > 0; c += 32) {
                    uint32_t x[32];
                    tmem_ld32(tO + c, x);
                    tmem_wait_ld();
                    if (c + 32 == D) warp_done(&bars.o_empty[s]);
                    if (!valid) continue;
#pragma unroll
                    for (int q = 0; q < 32; q += 8) {
                        uint32_t e[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) e[i] = x[q + i];
                        st_global_v8(y + (c + q) * 256, e);
                    }
                }
                if (valid)
                    shares.ml[(size_t)part * 256 + at_row] =
                        make_float2(mref, lsum);
                continue;
            }
            // a row that sees nothing, or only scores of -inf: zeros
            const float inv = lsum == 0.0f ? 0.0f : 1.0f / lsum;
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                uint32_t x[32];
                if (n > 0) {
                    tmem_ld32(tO + c, x);
                    tmem_wait_ld();
                    if (c + 32 == D) {
                        warp_done(&bars.o_empty[s]);
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 32; ++q) x[q] = 0;
                }
                uint32_t y[16];
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    y[e] = pack_bf16x2(__uint_as_float(x[2 * e]) * inv,
                                       __uint_as_float(x[2 * e + 1]) * inv);
                store_rows<D, 4>(y, o + c, valid, lane_id);
            }
            if (valid && a.lse)
                a.lse[at] = lsum == 0.0f ? -INFINITY
                                         : (mref + log2f(lsum)) * kLn2;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 8) tmem_dealloc(tm, 512);
}

// Joins the parts of divided items: blockIdx.y is the CTA that begins one,
// D / 8 lanes a row.
template <int D>
__global__ void __launch_bounds__(256)
    k_exact_merge(const __grid_constant__ ExactView a,
                  const __grid_constant__ EfShares shares,
                  const __grid_constant__ ExactOrder order) {
    wait_for_stream();
    const int first = blockIdx.y;
    const EfRecord rec = shares.rec[first];
    if (rec.last < 0) return;
    int c;
    const int row = (int)piece_of<D>(blockIdx.x * 256 + threadIdx.x, &c);
    const int r = rec.r0 + row;
    const int ql = ExactSeq(a, rec.b).ql;
    const ExactOrder own = order.of(ql);
    if (r >= own.rows || r % own.pitch >= ql) return;
    auto at = [&](int cta) { return (size_t)(2 * cta + (cta == first)); };
    float m = kLowest;
    for (int p = first; p <= rec.last; ++p)
        m = fmaxf(m, shares.ml[at(p) * 256 + row].x);
    float l = 0.0f, o[8] = {};
    for (int p = first; p <= rec.last; ++p) {
        const float2 ml = shares.ml[at(p) * 256 + row];
        if (ml.y == 0.0f) continue;  // its sums may not have been written
        const float f = ex2_approx(ml.x - m);
        l = fmaf(ml.y, f, l);
        const float4 *x =
            reinterpret_cast<const float4 *>(shares.o + at(p) * 256 * D +
                                             c * 256 + row * 8);
        const float4 u = x[0], v = x[1];
        const float e[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = fmaf(e[i], f, o[i]);
    }
    const size_t to = (size_t)(rec.b * a.H + rec.kvh * a.G) * a.Nq +
                      own.row(r, a.Nq);
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        y[i] = pack_bf16x2(o[2 * i] * inv, o[2 * i + 1] * inv);
    *reinterpret_cast<uint4 *>((uint16_t *)a.out + to * D + c) =
        make_uint4(y[0], y[1], y[2], y[3]);
    if (a.lse && c == 0)
        a.lse[to] = l == 0.0f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// Shares may be used with fewer than four items for each SM, and not for short
// keys, where dividing costs more. (By the sizes alone, whether q_len is given
// or not: with it there are as many items or more.)
bool may_share(const ExactView &a, bool padded) {
    const long tiles = ((long)a.Nk + 127) / 128;
    return ExactOrder(a, 256, padded).items(a) < 4 * kEfCtas && tiles >= 8 &&
           tiles <= 1 << 20 && a.B <= kEfMaxB;
}

// Shares instead of whole items, the longest first. A share's parts cost a CTA
// about 7 tiles' time and k_exact_merge; whole items cost what the last CTA takes
// beyond an equal share: at least (j + 1) times the item of rank j C among the C
// CTAs'. In padded batches that is known to the device alone: shares. Causal
// B1 H16 H_kv4 N4096 d128 (32 tiles, equal shares 29): whole items 59 us, shares
// 70; B1 H4 N8192 (64 tiles, shares 28): 107 and 66; B2 H8 H_kv1 N3000, not
// causal (two items of 24 tiles one behind the other, shares 30): 87 and 73.
bool use_shares(const ExactView &a) {
    if (!may_share(a, a.q_len != nullptr)) return false;
    if (a.q_len || a.k_len) return true;
    const ExactOrder order(a, 256);
    int n[4 * kEfCtas], items = 0;
    long sum = 0;
    for (long r0 = 0; r0 < order.rows && items < 4 * kEfCtas; r0 += 256) {
        const long r1 = r0 + 256 < order.rows ? r0 + 256 : order.rows;
        // the last row of a head, if there is one, else the tile's last
        const long last =
            r0 / a.Nq != (r1 - 1) / a.Nq ? a.Nq - 1 : (r1 - 1) % a.Nq;
        long seen = a.causal ? last + 1 + a.Nk - a.Nq : a.Nk;
        if (seen > a.Nk) seen = a.Nk;
        n[items] = seen > 0 ? (int)((seen + 127) / 128) : 0;
        sum += n[items++];
    }
    std::sort(n, n + items, [](int x, int y) { return x > y; });
    const long heads = (long)a.B * a.Hkv;
    long most = 0;
    for (long j = 0; j * kEfCtas < items * heads; ++j) {
        const long t = (j + 1) * n[j * kEfCtas / heads];
        if (t > most) most = t;
    }
    return most - sum * heads / kEfCtas > 7;
}

}  // namespace

size_t exact_share_bytes(const ExactView &a) {
    if (!may_share(a, false)) return 0;
    return sizeof(EfRecord) * kEfCtas +
           (size_t)2 * kEfCtas * 256 * sizeof(float) * (a.d + 2);
}

cudaError_t launch_exact_fwd_tc(const ExactView &a, int *next_item,
                                float *part, cudaStream_t st) {
    const ExactOrder order(a, 256);
    const long items = order.items(a);
    EfShares shares = {};
    shares.on = use_shares(a);
    shares.tiles = order.groups * order.per;
    const size_t rows = (size_t)2 * kEfCtas * 256;
    shares.o = part;
    shares.ml = (float2 *)(part + rows * a.d);
    shares.rec = (EfRecord *)(shares.ml + rows);
    int dev = 0, sms = 152;
    if (cudaGetDevice(&dev) == cudaSuccess)
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    const int ctas = shares.on ? (sms < kEfCtas ? sms : kEfCtas)
                               : (int)(items < sms ? items : sms);
    // more items than CTAs: they are taken from a counter
    const bool counted = !shares.on && items > sms;
    CUtensorMap tmQ, tmK, tmV;
    const uint64_t nq = (uint64_t)a.B * a.H * a.Nq;
    const uint64_t nk = (uint64_t)a.B * a.Hkv * a.Nk;
    cudaError_t e = make_tma_map_bf16(&tmQ, a.q, nq, a.d, 128);
    if (e == cudaSuccess) e = make_tma_map_bf16(&tmK, a.k, nk, a.d, 128);
    if (e == cudaSuccess) e = make_tma_map_bf16(&tmV, a.v, nk, a.d, 128);
    if (e == cudaSuccess && counted)
        e = launch_clear(a.status, next_item, 1, st);
    if (e != cudaSuccess) return e;
    auto launch = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        const size_t smem =
            1024 + (size_t)(2 + kEfK<D> + kEfV<D>) * (D > 64 ? 2 : 1) * 16384;
        cudaError_t r = launch_after(
            k_exact_fwd_tc<D>, dim3((unsigned)ctas), kEfThreads, smem, st,
            tmQ, tmK, tmV, a, shares, order, (int)items,
            counted ? next_item : nullptr);
        if (r == cudaSuccess && shares.on)
            r = launch_after(k_exact_merge<D>,
                             dim3(256 * (D / 8) / 256, (unsigned)ctas), 256, 0,
                             st, a, shares, order);
        return r;
    };
    return a.d == 128  ? launch(std::integral_constant<int, 128>{})
           : a.d == 64 ? launch(std::integral_constant<int, 64>{})
                       : launch(std::integral_constant<int, 32>{});
}

}  // namespace elsaa
