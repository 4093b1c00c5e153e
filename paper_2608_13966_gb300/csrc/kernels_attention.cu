// Instantiations of the attention kernels.
#include "attention.cuh"

namespace quasar {

const void* attention_kernel(int d, bool far)
{
    if (d <= 64)
        return far ? reinterpret_cast<const void*>(&k_attention<1, true>)
                   : reinterpret_cast<const void*>(&k_attention<1, false>);
    return far ? reinterpret_cast<const void*>(&k_attention<2, true>)
               : reinterpret_cast<const void*>(&k_attention<2, false>);
}

int attention_threads() { return kAttnThreads; }

size_t attention_smem(int d)
{
    const size_t tile = (size_t)(d <= 64 ? 1 : 2) * kAttnBlock, slots = d <= 64 ? kAttnSlots<1> : kAttnSlots<2>;
    return 1024 + (2 + 2 * slots) * tile + (2 * slots + 26) * 8 + 10 * 128 * 8 + kAttnRowWarps * 1024 +
           2 * sizeof(AttnWork);
}

}  // namespace quasar
