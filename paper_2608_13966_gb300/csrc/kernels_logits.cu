// Instantiations of the kernels over rows of logits.
#include "distill.cuh"
#include "top_logits.cuh"

namespace quasar {

namespace {

template <typename T>
const void* distill(int threads, bool backward)
{
    if (threads == kFewThreads)
        return backward ? reinterpret_cast<const void*>(&k_distill_top<T, kFewThreads, true>)
                        : reinterpret_cast<const void*>(&k_distill_top<T, kFewThreads, false>);
    return backward ? reinterpret_cast<const void*>(&k_distill_top<T, kBackThreads, true>)
                    : reinterpret_cast<const void*>(&k_distill_top<T, kRowThreads, false>);
}

}  // namespace

const void* distill_kernel(bool f32, int threads, bool backward)
{
    return f32 ? distill<float>(threads, backward) : distill<__nv_bfloat16>(threads, backward);
}

const void* top_logits_kernel(bool f32, int threads)
{
    if (f32)
        return threads == kFewThreads ? reinterpret_cast<const void*>(&k_top_logits<float, kFewThreads>)
                                      : reinterpret_cast<const void*>(&k_top_logits<float, kRowThreads>);
    return threads == kFewThreads ? reinterpret_cast<const void*>(&k_top_logits<__nv_bfloat16, kFewThreads>)
                                  : reinterpret_cast<const void*>(&k_top_logits<__nv_bfloat16, kRowThreads>);
}

size_t top_logits_smem(int threads, int ctas, int k)
{
    return (size_t)kTopVectors * 20 + (size_t)kTopKeys * 8 + (ctas > 1 ? (size_t)ctas * k * 8 : 0) + 8 + kRowCtas * 8 +
           64 * 4 + 6 * 4 + ((size_t)threads + kTopVectors) * 2;
}

size_t distill_smem(int vecs, int threads)
{
    const size_t words = (size_t)(vecs + kHand * threads - 1) / (kHand * threads) * threads;
    return words * 4 + 3 * kMaxTop * 4 + 64 * 4 + 4 * 4 + kRowCtas * 8 + 8 + 8;
}

}  // namespace quasar
