// Exact attention (include/elsaa_exact.h): what a call is about, and how the
// kernels see it.
#pragma once

#include "../../include/elsaa_exact.h"
#include "cache.h"

namespace elsaa {

struct ExactView {
    int B, H, Hkv, G, Nq, Nk, d, dtype, causal;
    float scale;
    const void *q, *k, *v, *o, *d_o;
    const int32_t *q_len, *k_len;
    float *lse;    // forward: written, or NULL; backward: read
    float *delta;  // [B, H, Nq] scratch of the backward pass
    void *out, *dq, *dk, *dv;
    DeviceStatus *status;
};

// How the rows of the query heads that share a K/V head are laid on tiles of
// `tile` rows, and the order in which the tiles are taken: the last one of
// every head (with causal = 1 it sees most) before the one before it, as far as
// heads and tiles coincide. Row r is row r mod pitch of head r / pitch. Heads
// follow one another without a gap (pitch = N_q), so that several short ones
// fill a tile; but a padded batch of longer rows begins every head with 128 rows
// of its own, or tiles would hold the padding between two heads. Some of the
// tiles given are past the last row.
struct ExactOrder {
    int pitch, rows, groups, per, heads, size;
    bool padded;
    ExactOrder(const ExactView &a, int tile)
        : ExactOrder(a, tile, a.q_len != nullptr) {}
    ExactOrder(const ExactView &a, int tile, bool lengths)
        : heads(a.G), size(tile), padded(lengths && a.Nq > 128) {
        lay(padded ? (a.Nq + 127) / 128 * 128 : a.Nq);
    }
#ifdef __CUDACC__
    __host__ __device__
#endif
    void lay(int p) {
        pitch = p;
        rows = heads * p;
        const int tiles = (rows + size - 1) / size;
        groups = tiles < heads ? 1 : heads;
        per = (tiles + groups - 1) / groups;
    }
    long items(const ExactView &a) const {
        return (long)groups * per * a.B * a.Hkv;
    }
#ifdef __CUDACC__
    __device__ __forceinline__ int tile(int t) const {
        return t % groups * per + per - 1 - t / groups;
    }
    // Of a sequence of ql rows in a padded batch of short ones, heads as far
    // apart as these rows need: then no 128 rows are without one, and tile()
    // holds for the first groups * per of the tiles that the batch's own order
    // gives. B8 H16 H_kv4 N_k 4096 d128 causal, us, heads as the batch has them
    // and fitted, by the rows of a sequence:
    //   N_q    20 rows   20 to 300   1 to N_q    0.85 N_q to N_q
    //    500   31   27   47    42    49    49       67    67
    //    900   31   27   47    42    78    80      106    99
    //   1100   41   35   55    42   104   103      124   126
    //   2048   41   35   56    42   153   154      237   239
    //   4096   53   37   68    50   311   306      440   431
    // B32, and B8 with 12 heads of 64, gain and lose likewise; half of the
    // sequences short and half long loses up to 6 % (N_q 2048, d64: 89 and 94).
    // So the rule gives away what long batches of short sequences alone would
    // gain.
    __device__ __forceinline__ ExactOrder of(int ql) const {
        ExactOrder x = *this;
        if (padded && pitch <= 1024) x.lay(max(ql + 127, 128) / 128 * 128);
        return x;
    }
    // where row r lies in memory, from the first head on
    __device__ __forceinline__ int row(int r, int N) const {
        return r / pitch * N + r % pitch;
    }
#endif
};

#ifdef __CUDACC__
// Sequence b's lengths, and how many keys query row i sees: the first seen(i).
struct ExactSeq {
    int ql, kl, causal;
    __device__ __forceinline__ ExactSeq(const ExactView &a, int b)
        : ql(a.Nq), kl(a.Nk), causal(a.causal) {
        if (a.q_len) ql = min(max(a.q_len[b], 0), a.Nq);
        if (a.k_len) kl = min(max(a.k_len[b], 0), a.Nk);
    }
    __device__ __forceinline__ int seen(int i) const {
        if (i >= ql) return 0;
        return causal ? max(0, min(kl, i + 1 + kl - ql)) : kl;
    }
    // the first query row that sees key row j (ql: none)
    __device__ __forceinline__ int first_row(int j) const {
        if (j >= kl) return ql;
        return causal ? min(ql, max(0, j + ql - kl)) : 0;
    }
};

// A row without a weight above 0 has lse = -inf: as +inf it makes
// exp(s - lse) = 0 also where scores of finite q and k overflow to -inf.
__device__ __forceinline__ float exact_lse(const float *lse) {
    const float x = *lse;
    return x == -INFINITY ? INFINITY : x;
}

// The backward pass makes weights again as 2^x, x = fma(s, sl2, -lse2), from an
// lse that was rounded on its way: the forward pass's product, lse itself and
// lse2, with log2 e and ln 2 as fp32. x is off by up to 2^-22.3 |lse2|, which
// below kFarLse is a factor of 1.01 of the weight. Behind it the largest one, 1
// or a little less, could come out as any power of two, or infinite: there x
// counts as 0 from -2^-21 |lse2| on. exact_edge: where that begins, +inf for
// rows that need none of it.
constexpr float kFarLse = 65536.0f;
__device__ __forceinline__ float exact_edge(float lse2) {
    const float z = fabsf(lse2);
    return z > kFarLse && z < INFINITY ? -0x1p-21f * z : INFINITY;
}
// (a NaN stays one)
__device__ __forceinline__ float exact_exponent(float x, float edge) {
    return x > edge ? 0.0f : x;
}

// Rows of the query heads that share a K/V head, counted through: row r is row
// r mod N of head r / N of the group. `most` is the largest seen() among rows
// [r0, r1).
__device__ __forceinline__ int exact_most(const ExactSeq &s, int r0, int r1,
                                          int N) {
    if (r0 >= r1 || s.ql == 0) return 0;
    const int i0 = r0 % N, i1 = (r1 - 1) % N;
    const int heads = (r1 - 1) / N - r0 / N;
    // the last row of a head is among them
    if (heads > 1 || (heads == 1 && i0 < s.ql)) return s.seen(s.ql - 1);
    return heads == 1 || i0 < s.ql ? s.seen(min(i1, s.ql - 1)) : 0;
}

// Row and first of eight channels of thread t, of D / 8 threads a row: a warp
// has 8 rows and 4 pieces of 8 channels of each, so that its reads of sums laid
// out [D / 8][rows][8] cover 256 bytes and its writes of a bf16 row 64.
template <int D>
__device__ __forceinline__ long piece_of(long t, int *c) {
    const int lane = (int)(t & 31);
    const long warp = t >> 5;
    *c = (int)(warp % (D / 32)) * 32 + (lane & 3) * 8;
    return warp / (D / 32) * 8 + (lane >> 2);
}

// Writes CH 16-byte pieces (2 or 4) of every lane's row, rows D elements apart:
// y is the lane's own row from `row` on. Lanes first exchange pieces in groups
// of CH, so that a store covers 16 CH bytes of 32 / CH rows; with a row a lane
// each store met 32 lines, and the memory unit took them one after the other.
template <int D, int CH>
__device__ __forceinline__ void store_rows(uint32_t (&y)[4 * CH],
                                           uint16_t *row, bool valid,
                                           int lane) {
    const uint32_t rows = __ballot_sync(0xffffffffu, valid);
#pragma unroll
    for (int bit = 1; bit < CH; bit <<= 1) {
        const bool up = lane & bit;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
            if (k & bit) continue;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                uint32_t &a = y[4 * k + w], &b = y[4 * (k | bit) + w];
                const uint32_t r =
                    __shfl_xor_sync(0xffffffffu, up ? a : b, bit);
                if (up)
                    a = r;
                else
                    b = r;
            }
        }
    }
    // piece p of row (group + i) now is piece i of lane p of the group
    const int p = lane & (CH - 1), first = lane - p;
    uint16_t *to = row - p * D + 8 * p;
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (rows >> (first + i) & 1)
            *reinterpret_cast<uint4 *>(to + i * D) = make_uint4(
                y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
}
#endif

// bf16 on the tensor cores; next_item: an int of scratch; part:
// exact_share_bytes(a) of it, 256-byte aligned
size_t exact_share_bytes(const ExactView &a);
cudaError_t launch_exact_fwd_tc(const ExactView &a, int *next_item,
                                float *part, cudaStream_t st);
// Its backward pass: D_i first (which also clears the status, two work counters
// and `far`), then dQ (which sets `far` where a row's lse is behind kFarLse),
// and dK with dV, and the sums of walks that were divided. part:
// exact_part_bytes(a) of scratch, 256-byte aligned.
size_t exact_part_bytes(const ExactView &a);
cudaError_t launch_exact_delta(const ExactView &a, int *counters,
                               cudaStream_t st);
cudaError_t launch_exact_dq_tc(const ExactView &a, int *next_item, int *far,
                               float *part, cudaStream_t st);
cudaError_t launch_exact_dkv_tc(const ExactView &a, int *next_item,
                                const int *far, float *part, cudaStream_t st);
cudaError_t launch_exact_sum(const ExactView &a, float *part,
                             cudaStream_t st);
// CUDA cores (fp32, and bf16 with impl = SIMT)
// part: exact_chunk_bytes(a) of scratch
size_t exact_chunk_bytes(const ExactView &a);
cudaError_t launch_exact_fwd_simt(const ExactView &a, float *part,
                                  cudaStream_t st);
// part: exact_add_bytes(a) of scratch
size_t exact_add_bytes(const ExactView &a);
cudaError_t launch_exact_bwd_simt(const ExactView &a, bool keys, float *part,
                                  cudaStream_t st);

}  // namespace elsaa
