// The division of the cache attention's units over CTAs (cache_division.h) at
// the limits that the host's checks accept, against 128-bit arithmetic.
// Arguments: lines of `sum items HC ctas whole` on standard input.
#include <cstdio>

#include "cache_division.h"

using elsaa::kCacheMaxPieces;
using elsaa::cache::Cut;
using elsaa::cache::kItemCost;
typedef unsigned __int128 wide;

int main() {
    unsigned long sum, items, HC, ctas, whole, lines = 0;
    while (scanf("%lu %lu %lu %lu %lu", &sum, &items, &HC, &ctas, &whole) ==
           5) {
        ++lines;
        const Cut c((unsigned)sum, (unsigned)items, (unsigned)HC,
                    (unsigned)ctas, whole != 0);
        const wide total = (wide)sum * HC, live = (wide)items * HC;
        wide n = whole ? live : total - live * kItemCost;
        if (ctas < n) n = ctas;
        if (live * kCacheMaxPieces < n) n = live * kCacheMaxPieces;
        bool ok = c.total == total && c.n == n;
        for (unsigned k = 0; ok && k <= c.n && c.n > 0; ++k) {
            const wide q = total / n, rest = total % n;
            ok = c.at(k) == q * k + rest * k / n;
            if (k == c.n) break;
            const unsigned a = c.at(k), z = c.at(k + 1);
            ok = ok && z > a && c.owner(a) == k && c.owner(z - 1) == k &&
                 c.owner(a + (z - a) / 2) == k;
        }
        if (!ok) {
            printf("sum %lu items %lu HC %lu ctas %lu whole %lu: n %u\n", sum,
                   items, HC, ctas, whole, c.n);
            return 1;
        }
    }
    printf("%lu ok\n", lines);
    return 0;
}
