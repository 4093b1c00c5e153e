// Instantiations of the attention's backward kernels.
#include "attention_grad.cuh"

namespace quasar {

const void* attention_stats_kernel(int d)
{
    return d <= 64 ? reinterpret_cast<const void*>(&k_attention_stats<8>)
                   : reinterpret_cast<const void*>(&k_attention_stats<16>);
}

const void* attention_grad_kernel(int d, bool keys)
{
    if (d <= 64)
        return keys ? reinterpret_cast<const void*>(&k_attention_grad<1, true>)
                    : reinterpret_cast<const void*>(&k_attention_grad<1, false>);
    return keys ? reinterpret_cast<const void*>(&k_attention_grad<2, true>)
                : reinterpret_cast<const void*>(&k_attention_grad<2, false>);
}

int attention_grad_threads() { return kGradThreads; }

size_t attention_grad_smem(int d)
{
    const size_t block = (size_t)(d <= 64 ? 1 : 2) * 128;
    return 1024 + 2 * kAttnRows * block + kGradSlots * (2 * kGradCols * block + kGradCols * 8) +
           (1 + 3 * kGradSlots + 4 + 2) * 8 + 8 + sizeof(AttnItem) + 8;
}

}  // namespace quasar
