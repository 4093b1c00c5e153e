// Instantiations of the embedding's kernels.
#include "embedding.cuh"

namespace quasar {

#define QUASAR_EMBED(name, kernel)                                                                            \
    const void* name(bool vectors, bool wide)                                                                 \
    {                                                                                                         \
        if (vectors)                                                                                          \
            return wide ? reinterpret_cast<const void*>(&kernel<true, true>)                                  \
                        : reinterpret_cast<const void*>(&kernel<true, false>);                                \
        return wide ? reinterpret_cast<const void*>(&kernel<false, true>)                                     \
                    : reinterpret_cast<const void*>(&kernel<false, false>);                                   \
    }
QUASAR_EMBED(embedding_kernel, k_embedding)
QUASAR_EMBED(embedding_chunks_kernel, k_embedding_chunks)
QUASAR_EMBED(embedding_grad_kernel, k_embedding_grad)
#undef QUASAR_EMBED

const void* sort_ids_kernel() { return reinterpret_cast<const void*>(&k_sort_ids); }

size_t sort_ids_smem()
{
    return ((size_t)(kSortThreads / 32) * (1 << kSortBits) + 2 * (1 << kSortBits) + (1 << kSortBits) / 32) * 4;
}

}  // namespace quasar
