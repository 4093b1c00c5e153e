// Instantiations of the layer norms.
#include "layer_norm.cuh"

namespace quasar {

namespace {

struct Shape {
    int t, nv;  // threads a row, vectors of 8 a thread
};

// Short rows share a CTA of 256 threads; from 65 vectors on a row has a CTA, of
// up to 4 vectors a thread (backward, where a vector takes more registers: 2).
Shape norm_shape(int64_t cols, bool grad)
{
    const int64_t vecs = (cols + 7) / 8;
    if (vecs <= 8) return {8, 1};
    if (vecs <= 16) return {8, 2};
    if (vecs <= 32) return {32, 1};
    if (vecs <= 64) return {32, 2};
    if (vecs <= 128) return {128, 1};
    if (vecs <= 256) return {128, 2};
    if (!grad) {
        if (vecs <= 512) return {128, 4};
        return vecs <= 1024 ? Shape{256, 4} : Shape{512, 4};
    }
    if (vecs <= 512) return {256, 2};
    return vecs <= 1024 ? Shape{512, 2} : Shape{512, 4};
}

template <int T, int NV>
const void* forward(bool vectors, bool wide)
{
    if (vectors)
        return wide ? reinterpret_cast<const void*>(&k_layer_norm<T, NV, true, true>)
                    : reinterpret_cast<const void*>(&k_layer_norm<T, NV, true, false>);
    return wide ? reinterpret_cast<const void*>(&k_layer_norm<T, NV, false, true>)
                : reinterpret_cast<const void*>(&k_layer_norm<T, NV, false, false>);
}

template <int T, int NV>
const void* backward(bool vectors, bool wide)
{
    if (vectors)
        return wide ? reinterpret_cast<const void*>(&k_layer_norm_grad<T, NV, true, true>)
                    : reinterpret_cast<const void*>(&k_layer_norm_grad<T, NV, true, false>);
    return wide ? reinterpret_cast<const void*>(&k_layer_norm_grad<T, NV, false, true>)
                : reinterpret_cast<const void*>(&k_layer_norm_grad<T, NV, false, false>);
}

}  // namespace

// The kernel of rows of this length (backward: of their gradients), its
// threads, how many rows a CTA takes at a time and how many CTAs an SM holds;
// nullptr for rows that registers do not hold.
const void* layer_norm_kernel(int64_t cols, bool vectors, bool grad, bool wide, int* threads, int* rows, int* per_sm)
{
    if (cols > kNormMostCols) return nullptr;
    const Shape s = norm_shape(cols, grad);
    *threads = s.t < 128 ? 256 : s.t;
    *rows = *threads / s.t;
    *per_sm = (s.nv == 1 ? 768 : 512) / *threads;
#define QUASAR_NORM(T, NV) \
    if (s.t == T && s.nv == NV) return grad ? backward<T, NV>(vectors, wide) : forward<T, NV>(vectors, wide);
#define QUASAR_NORM_FORWARD(T, NV) \
    if (s.t == T && s.nv == NV) return forward<T, NV>(vectors, wide);
    QUASAR_NORM(8, 1)
    QUASAR_NORM(8, 2)
    QUASAR_NORM(32, 1)
    QUASAR_NORM(32, 2)
    QUASAR_NORM(128, 1)
    QUASAR_NORM(128, 2)
    QUASAR_NORM(512, 4)
    if (grad) {
        if (s.t == 256) return backward<256, 2>(vectors, wide);
        return backward<512, 2>(vectors, wide);
    }
    QUASAR_NORM_FORWARD(128, 4)
    QUASAR_NORM_FORWARD(256, 4)
#undef QUASAR_NORM
#undef QUASAR_NORM_FORWARD
    return nullptr;
}

// The kernel of rows through shared memory (rows of whole vectors of 8 that
// start at 16-byte boundaries), its threads and CTAs an SM; nullptr for rows
// that a warp takes, or that registers do not hold (backward beyond 8192, where
// dw and db need them too: k_layer_norm_grad has such rows, with 348 to 808 bytes of
// spills a thread and no row on its way; 4096 x 16384 bf16 164 us, 2.5 TB/s, against
// 82, 4.9 TB/s, for 8192 x 8192 here).  Rows that are not whole vectors take the
// register kernels by single elements: 16384 x 4099 bf16 219 us forward and 310
// back, against 51 and 79 for 4096 columns.
const void* layer_norm_ring_kernel(int64_t cols, bool grad, bool wide, int* threads, int* per_sm)
{
    if (cols % 8 != 0 || cols <= 1024 || cols > (grad ? 8192 : kNormMostCols)) return nullptr;
#define QUASAR_RING(most, T, NV, kernel, grads)                                        \
    if (cols <= most) {                                                                \
        *threads = T, *per_sm = kNormRingPerSm<T, NV, grads>;                          \
        return wide ? reinterpret_cast<const void*>(&kernel<T, NV, true>)              \
                    : reinterpret_cast<const void*>(&kernel<T, NV, false>);            \
    }
    // few threads with many elements each: the reductions cost a warp as much
    // for 1 as for 4 vectors (16384 x 4096: 512 threads of one 75 us)
    if (grad) {
        QUASAR_RING(2048, 128, 2, k_layer_norm_grad_ring, true)
        QUASAR_RING(4096, 256, 2, k_layer_norm_grad_ring, true)
        QUASAR_RING(8192, 512, 2, k_layer_norm_grad_ring, true)
    }
    QUASAR_RING(2048, 128, 2, k_layer_norm_ring, false)
    QUASAR_RING(4096, 128, 4, k_layer_norm_ring, false)
    QUASAR_RING(8192, 256, 4, k_layer_norm_ring, false)
    QUASAR_RING(kNormMostCols, 512, 4, k_layer_norm_ring, false)
#undef QUASAR_RING
    return nullptr;
}

// Slots of a ring, by what the CTAs of an SM leave each other.
int layer_norm_slots(uint32_t slot_bytes, int threads, int per_sm, size_t* smem)
{
    int slots = 8;
    while (slots > 1 && norm_ring_smem(slots, slot_bytes, threads) > (size_t)216 * 1024 / per_sm) --slots;
    *smem = norm_ring_smem(slots, slot_bytes, threads);
    return slots;
}

const void* layer_norm_long_kernel() { return reinterpret_cast<const void*>(&k_layer_norm_long); }
const void* layer_norm_grad_long_kernel() { return reinterpret_cast<const void*>(&k_layer_norm_grad_long); }
const void* layer_norm_grad_columns_kernel() { return reinterpret_cast<const void*>(&k_layer_norm_grad_columns); }
const void* part_sum_kernel() { return reinterpret_cast<const void*>(&k_part_sum); }

}  // namespace quasar
