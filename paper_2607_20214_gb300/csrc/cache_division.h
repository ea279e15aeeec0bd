// How the attention kernels' CTAs share the units of all items (what an item
// and a unit are: cache_common.cuh). In 32 bits, for whatever the host's checks
// accept: fewer than 2^31 units in all. Apart from the kernels, and without
// CUDA, so that tests/test_cache_division.py can run it on the host against
// wider numbers.
#pragma once

#ifdef __CUDACC__
#define ELSAA_DEV __device__ __forceinline__
#else
#define ELSAA_DEV inline
#endif

namespace elsaa {

// CTAs per shared item at most, on average over the items: the merge's cost
// grows with them (128 and 304 were slower).
constexpr int kCacheMaxPieces = 64;

namespace cache {

// Units of an item beside its tiles.
constexpr int kItemCost = 3;

// The units of CTA k of n, total / n or one more, without a product that needs
// 64 bits. `sum` units and `items` items for each of the HC heads and groups.
struct Cut {
    unsigned total, n, q, rest;
    ELSAA_DEV Cut(unsigned sum, unsigned items, unsigned HC, unsigned ctas,
                  bool whole) {
        const unsigned live = items * HC;
        total = sum * HC;
        // no more CTAs than tiles
        const unsigned tiles = whole ? live : total - live * kItemCost;
        n = ctas < tiles ? ctas : tiles;
        // live * kCacheMaxPieces < n, whose product may not fit
        if (live < (n + kCacheMaxPieces - 1) / kCacheMaxPieces)
            n = live * kCacheMaxPieces;
        q = n ? total / n : 0;
        rest = total - q * n;
    }
    // the first unit of CTA k; of the last and one: total
    ELSAA_DEV unsigned at(unsigned k) const { return q * k + rest * k / n; }
    // the CTA that has unit u
    ELSAA_DEV unsigned owner(unsigned u) const {
        unsigned k = (unsigned)((float)u * ((float)n / (float)total));
        if (k > n - 1) k = n - 1;
        while (k > 0 && at(k) > u) --k;
        while (at(k + 1) <= u) ++k;
        return k;
    }
};

}  // namespace cache
}  // namespace elsaa
