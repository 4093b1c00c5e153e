// Instantiations of the embedding's kernels.
#include "embedding.cuh"

namespace quasar {

const void* embedding_kernel(bool vectors)
{
    return vectors ? reinterpret_cast<const void*>(&k_embedding<true>) : reinterpret_cast<const void*>(&k_embedding<false>);
}

const void* sort_ids_kernel() { return reinterpret_cast<const void*>(&k_sort_ids); }

size_t sort_ids_smem()
{
    return ((size_t)(kSortThreads / 32) * (1 << kSortBits) + (1 << kSortBits) + (1 << kSortBits) / 32) * 4;
}

const void* embedding_chunks_kernel(bool vectors)
{
    return vectors ? reinterpret_cast<const void*>(&k_embedding_chunks<true>)
                   : reinterpret_cast<const void*>(&k_embedding_chunks<false>);
}

const void* embedding_grad_kernel(bool vectors)
{
    return vectors ? reinterpret_cast<const void*>(&k_embedding_grad<true>)
                   : reinterpret_cast<const void*>(&k_embedding_grad<false>);
}

}  // namespace quasar
