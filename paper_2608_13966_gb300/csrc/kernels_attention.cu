// Instantiations of the attention kernels.
#include "attention.cuh"

namespace quasar {

const void* attention_kernel(int d)
{
    return d <= 64 ? reinterpret_cast<const void*>(&k_attention<1>) : reinterpret_cast<const void*>(&k_attention<2>);
}

int attention_threads() { return kAttnThreads; }

size_t attention_smem(int d)
{
    const size_t tile = (size_t)(d <= 64 ? 1 : 2) * kAttnBlock, slots = d <= 64 ? kAttnSlots<1> : kAttnSlots<2>;
    return 1024 + (2 + 2 * slots) * tile + (2 * slots + 26) * 8 + 10 * 128 * 8 + kAttnRowWarps * 1024 +
           2 * sizeof(AttnWork);
}

}  // namespace quasar
