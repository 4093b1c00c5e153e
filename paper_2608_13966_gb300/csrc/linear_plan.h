// How many CTAs share a tile of a matrix product (host).
#pragma once

#include <algorithm>
#include <cstdint>

#include "quasar.h"

namespace quasar {

// CTAs that share a tile's reduction: as many as leave each two blocks, while
// all clusters run at once.  A CTA's copies bound it, so a split shortens the
// call until the SMs are full (2 against 3 CTAs a tile: 128 x 11008 x 4096
// 23.9 and 19.9 us with one input set over and over, 5012 x 160 x 12544 55 and
// 42), but clusters left over start when the rest is done (5012 x 128 x 12544:
// 40 clusters of 6 CTAs 29.8 us, of 7, more than fit, 45.8, of 4 33.2).
//
// How many clusters fit does not follow from the SM count, as one lies within
// a part of the device.  max_clusters(size, &n) asks the device, whose answer
// counts one CTA an SM; the kernel runs two, so a cluster of s takes the place
// of half one, or of one of half the size.  A size of which it holds none
// (UNSUPPORTED) is not taken; one CTA a tile always is.
template <typename MaxClusters>
quasar_status tile_split(int64_t tiles, int k_blocks, int n_sm, MaxClusters max_clusters, int* split)
{
    *split = 1;
    for (int s = std::min(8, k_blocks / 2); s > 1; --s) {
        if (tiles * s > 2 * (int64_t)n_sm) continue;
        int whole = 0, half = n_sm;
        quasar_status st = max_clusters(s, &whole);
        if (st == QUASAR_ERR_UNSUPPORTED) continue;
        if (st == QUASAR_OK && s > 2) st = max_clusters((s + 1) / 2, &half);
        if (st != QUASAR_OK) return st;
        if (tiles > std::max(2 * whole, half)) continue;
        // no more CTAs than the longest share needs
        while ((k_blocks + s - 2) / (s - 1) == (k_blocks + s - 1) / s) --s;
        *split = s;
        break;
    }
    return QUASAR_OK;
}

}  // namespace quasar
