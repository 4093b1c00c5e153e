// Instantiations of the one-tile-per-cluster matrix products.
#include "linear.cuh"

namespace quasar {

// The kernel of 128-row tiles with bn columns; nullptr if there is none.
const void* product_tile_kernel(int bn, bool a_mn, bool b_mn, bool promote)
{
#define QUASAR_TILE(n, am, bm)                                                              \
    if (bn == n && a_mn == am && b_mn == bm)                                                \
        return promote ? reinterpret_cast<const void*>(&k_product_tile<n, am, bm, true>)    \
                       : reinterpret_cast<const void*>(&k_product_tile<n, am, bm, false>);
    QUASAR_TILE(16, false, false)
    QUASAR_TILE(32, false, false)
    QUASAR_TILE(64, false, false)
    QUASAR_TILE(128, false, false)
    QUASAR_TILE(16, true, false)
    QUASAR_TILE(32, true, false)
    QUASAR_TILE(64, true, false)
    QUASAR_TILE(128, true, false)
    QUASAR_TILE(64, true, true)
    QUASAR_TILE(128, true, true)
#undef QUASAR_TILE
    return nullptr;
}

}  // namespace quasar
