// Internal declarations of the cache operators (include/elsaa_cache.h): the
// view of a cache that kernels take by value, the division of attention work
// over CTAs, and the launchers.
#pragma once

#include "../../include/elsaa_cache.h"
#include "cache_division.h"
#include "internal.h"

namespace elsaa {

// Exponents of a page's scale, and of an 8-bit query in the page scores.
constexpr int kCacheExpLow = -64, kCacheExpHigh = 120;
constexpr int kQueryExpLow = -60;
// Tokens per tile of the attention kernels: a whole number of pages.
constexpr int kCacheTile = 128;
// Sequences of a call: every CTA of the attention kernels reads all lengths.
constexpr int kCacheMaxB = 4096;
// Tokens that a table row may hold: positions are ints, and the kernels' loops
// and tiles step beyond the last one, by 8192 at most.
constexpr long kCacheMaxSlots = (1L << 31) - (1L << 16);
// In-band status codes and sites of the cache kernels.
constexpr int kDevCachePage = 5;    // a page outside the pool was skipped
constexpr int kDevCacheLength = 6;  // a length outside the table was clipped

struct CacheView {
    int B, H, Hkv, G, d, ps, num_pages, max_pages, T;
    int dtype;
    float scale;
    uint8_t *k, *v;
    float *ks, *vs;
    int8_t *bounds;
    const int32_t *table, *lengths, *new_len;
    DeviceStatus *status;
};

// An item of the attention kernels that began in a CTA and went on in others.
struct alignas(16) CacheSplit {
    int b, hc;   // sequence; K/V head * groups + column group
    int pieces;  // CTAs; 0: none such
    int n;       // the sequence's new tokens
};

// One attention call. Columns of an item: the G T queries of a K/V head, in
// groups of `cols` (the last group may be smaller); column g T + t.
struct CacheAttn {
    CacheView c;
    const void *q;
    void *o;
    float *lse;              // or NULL
    const int32_t *pages;    // [B, Hkv, n_sel], or NULL
    int n_sel;
    const float *weight_in;
    float *weight_out;       // or NULL: no weights
    int cols, groups;        // columns per group, groups of a head
    int ctas;                // CTAs that share the tiles
    bool whole;              // no item is shared: an item a CTA
    unsigned per_t;          // col / T is col * per_t >> 16
    // workspace
    CacheSplit *split;       // [ctas]
    float *part;             // [ctas][2][cols][d + 2]: O, max, sum of pieces
    float *lse2;             // [B, Hkv, G T] log2 sums
    float *scores;           // [B, Hkv, G T, slots] log2 scores (weights)
    long slots;              // rows of a head's scores
};

// CTAs of the attention kernels on this chip's 152 SMs, and the columns that
// one walks at a time.
constexpr int kCacheSimtCtas = 152 * 3;
constexpr int kCacheTcCtas = 152 * 2;
// The tensor-core kernel's CTAs take whole items, and nothing is merged, where
// an item (of the table, or of the pages listed) has kCacheWhole tiles at most,
// every one finds a CTA, and a CTA gets at most kCacheMore tiles more than it
// would get of items that are shared. Sharing gives every CTA two beginnings
// and ends, and the merge is a launch: 8 sequences with 32 heads of 1024 tokens
// 15.8 us shared, 12.0 whole; 8 with 8 heads, 4 x 5 queries each, 512 tokens
// 19.0 and 11.2. Shared and whole, in a graph, by tiles more:
//                                    2     3     4     5     6     7     8
// 12 heads of 64, a sequence  shared 7.0   8.0   8.1   8.2   7.9   8.4   8.2
//                             whole  5.8   6.8   7.3   8.2   8.4   9.2   9.5
// 8 heads of 4 queries, 4 s.  shared 7.5   9.0   8.3   9.6   10.4  10.6  11.6
//                             whole  6.2   7.2   7.5   8.4   8.9   9.8   10.2
// One by one from Python a launch less counts too (12 heads, 6 tiles: 8.8 to
// 9.2 and 8.8; 7: 9.0 and 9.6): at 6 the rule gives away half a microsecond of
// the GPU's time with few items for the host's, and wins with many. Behind more
// than kCacheWholeSeqs sequences (a warp's lanes) the division counts tiles.
constexpr int kCacheWhole = 16, kCacheMore = 6;
constexpr int kCacheWholeSeqs = 32;
inline int cache_simt_cols(int gt) { return gt >= 3 ? 4 : gt; }
// A step of 16 columns costs as much as nearly two of 8, whether they are used
// or not, so 17 to 24 are three groups of 8 as long as the third reading of K
// and V finds them in L2 (129 MB; `bytes`: what the table can hold): with 20,
// 8 sequences of 8 heads and 2000 tokens on average 23.5 -> 20.1 us, one of
// 8192 tokens 22.0 -> 17.8; 32 of 8192 tokens (537 MB) 212 and 247.
constexpr long kCacheRereads = 96L << 20;
inline int cache_tc_cols(int gt, long bytes) {
    if (gt > 16 && gt <= 24 && bytes <= kCacheRereads) return 8;
    int n = 1;
    while (n < gt && n < 16) n *= 2;
    return n;
}

bool cache_attn_tc_supported(const CacheView &c);
cudaError_t launch_cache_attn_simt(const CacheAttn &A, cudaStream_t st);
cudaError_t launch_cache_attn_tc(const CacheAttn &A, cudaStream_t st);
cudaError_t launch_cache_merge(const CacheAttn &A, bool tensor_cores,
                               cudaStream_t st);
cudaError_t launch_cache_weights(const CacheAttn &A, cudaStream_t st);

cudaError_t launch_cache_append(const CacheView &c, const void *k,
                                const void *v, cudaStream_t st);
cudaError_t launch_cache_select(const CacheView &c, const void *q, int n_sel,
                                int first, int last, int32_t *pages,
                                float *scores, cudaStream_t st);
// rows: [B, Hkv, keep] pool rows of the kept tokens (page * page_size + row;
// -1: their page is outside the pool), kept: their positions, or NULL;
// count: [B] tokens kept.
struct CacheKept {
    int32_t *rows, *kept;
    int *count;
    float *weight_out;
    int dst_pages;
};
cudaError_t launch_cache_keep(const CacheView &c, const float *weight,
                              int keep, int recent, const CacheKept &out,
                              cudaStream_t st);
cudaError_t launch_cache_compact(const CacheView &c, int keep,
                                 const int32_t *rows, const int *count,
                                 const int32_t *dst_table, int dst_pages,
                                 int32_t *lengths_out, cudaStream_t st);

// Runs a launch under its name in the per-kernel timing of
// elsaa_profile_start (abi.cu).
cudaError_t timed_launch(const char *name, cudaStream_t st,
                         cudaError_t (*fn)(void *), void *arg);

}  // namespace elsaa
