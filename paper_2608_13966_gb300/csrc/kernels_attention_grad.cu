// Instantiations of the attention's backward kernels.
#include "attention_grad.cuh"

namespace quasar {

const void* attention_stats_kernel(int d)
{
    return d <= 64 ? reinterpret_cast<const void*>(&k_attention_stats<8>)
                   : reinterpret_cast<const void*>(&k_attention_stats<16>);
}

template <int DB, bool KEYS>
static const void* grad_kernel(bool far)
{
    return far ? reinterpret_cast<const void*>(&k_attention_grad<DB, KEYS, true>)
               : reinterpret_cast<const void*>(&k_attention_grad<DB, KEYS, false>);
}

const void* attention_grad_kernel(int d, bool keys, bool far)
{
    if (d <= 64) return keys ? grad_kernel<1, true>(far) : grad_kernel<1, false>(far);
    return keys ? grad_kernel<2, true>(far) : grad_kernel<2, false>(far);
}

int attention_grad_threads() { return kGradThreads; }

// (the memory starts at a multiple of 1024; where there is room, without relying on it)
size_t attention_grad_smem(int d)
{
    return d <= 64 ? 1024 + attention_grad_bytes(1) : attention_grad_bytes(2);
}

}  // namespace quasar
