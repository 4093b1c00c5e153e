// Instantiations of the kernels over rows of logits.
#include "top_logits.cuh"

namespace quasar {

const void* distill_kernel(bool f32, bool backward)
{
    if (f32)
        return backward ? reinterpret_cast<const void*>(&k_distill_top<float, true>)
                        : reinterpret_cast<const void*>(&k_distill_top<float, false>);
    return backward ? reinterpret_cast<const void*>(&k_distill_top<__nv_bfloat16, true>)
                    : reinterpret_cast<const void*>(&k_distill_top<__nv_bfloat16, false>);
}

const void* top_logits_kernel(bool f32)
{
    return f32 ? reinterpret_cast<const void*>(&k_top_logits<float>)
               : reinterpret_cast<const void*>(&k_top_logits<__nv_bfloat16>);
}

}  // namespace quasar
