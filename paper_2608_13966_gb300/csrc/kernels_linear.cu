// Instantiations of the paired matrix products, the product of one token,
// the column sums and the activation gradient.
#include "linear_one.cuh"
#include "linear_grad.cuh"

namespace quasar {

// The kernel of paired 256 x 256 tiles; nullptr if there is none.
const void* product_pair_kernel(bool a_mn, bool b_mn, bool promote)
{
#define QUASAR_PAIR(am, bm, pr) \
    if (a_mn == am && b_mn == bm && promote == pr) return reinterpret_cast<const void*>(&k_product_pair<am, bm, pr>);
    QUASAR_PAIR(false, false, false)
    QUASAR_PAIR(false, false, true)
    QUASAR_PAIR(true, false, false)
    QUASAR_PAIR(true, false, true)
    QUASAR_PAIR(true, true, false)
    QUASAR_PAIR(true, true, true)
#undef QUASAR_PAIR
    return nullptr;
}

int product_pair_threads() { return kPairThreads; }

size_t product_pair_smem() { return 1024 + kPairStages * kPairStageBytes + (2 * kPairStages + 8) * 8 + 16; }

const void* linear_one_kernel() { return reinterpret_cast<const void*>(&k_linear_one); }
// The kernel of up to 8 tokens' outer products; `padded`: the tokens it is
// built for.
const void* outer_kernel(int64_t tokens, bool f32, int* padded)
{
#define QUASAR_OUTER(n)                                                       \
    if (tokens <= n) {                                                        \
        *padded = n;                                                          \
        return f32 ? reinterpret_cast<const void*>(&k_outer<n, true>)         \
                   : reinterpret_cast<const void*>(&k_outer<n, false>);       \
    }
    QUASAR_OUTER(1)
    QUASAR_OUTER(2)
    QUASAR_OUTER(4)
    QUASAR_OUTER(8)
#undef QUASAR_OUTER
    return nullptr;
}

const void* column_sum_kernel() { return reinterpret_cast<const void*>(&k_column_sum); }
const void* activation_grad_kernel() { return reinterpret_cast<const void*>(&k_activation_grad); }

}  // namespace quasar
