// One row of logits held in the shared memory of a cluster, so that a row is
// read from HBM once however often it is passed over.
//
// The row is cut at 16-byte addresses: vector 0 is the 16 bytes that hold the
// row's first element, and CTA c of the cluster holds the vectors [c vecs,
// (c + 1) vecs).  Rows may start at any element; the two vectors that the row
// fills only in part are loaded element by element and completed with -inf,
// the rest arrives by bulk copies.
#pragma once

#include <cuda_bf16.h>

#include "cluster.cuh"
#include "logits.h"

namespace quasar {

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xFF800000); }

template <typename T>
struct Vec16;  // 16 bytes of T as floats

template <>
struct Vec16<float> {
    static constexpr int kN = 4;
    static __device__ __forceinline__ void unpack(const uint4& x, float (&v)[4])
    {
        v[0] = __uint_as_float(x.x);
        v[1] = __uint_as_float(x.y);
        v[2] = __uint_as_float(x.z);
        v[3] = __uint_as_float(x.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&v)[4])
    {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                          __float_as_uint(v[3]));
    }
    static __device__ __forceinline__ float to_f32(float x) { return x; }
    static __device__ __forceinline__ float from_f32(float x) { return x; }
};

template <>
struct Vec16<__nv_bfloat16> {
    static constexpr int kN = 8;
    static __device__ __forceinline__ void unpack(const uint4& x, float (&v)[8])
    {
        v[0] = bf16lo(x.x), v[1] = bf16hi(x.x);
        v[2] = bf16lo(x.y), v[3] = bf16hi(x.y);
        v[4] = bf16lo(x.z), v[5] = bf16hi(x.z);
        v[6] = bf16lo(x.w), v[7] = bf16hi(x.w);
    }
    static __device__ __forceinline__ uint4 pack(const float (&v)[8])
    {
        return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]),
                          pack_bf16x2(v[6], v[7]));
    }
    static __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }
};

// Where a CTA's slice of one row lies.  Slots count elements from the 16-byte
// boundary at or before the row's start: element e of the row is slot lead + e.
template <typename T>
struct RowSlice {
    static constexpr int kN = Vec16<T>::kN;
    const T* row;      // element 0 of the row
    int lead;          // slots before the row in its first vector
    int64_t first;     // first slot of the slice
    int n_vecs;        // vectors of the slice (may be 0)
    int64_t begin;     // slots [begin, end) of the slice hold elements
    int64_t end;

    __device__ __forceinline__ RowSlice(const RowParams& p, int64_t r, int rank)
    {
        row = static_cast<const T*>(p.logits) + r * p.ld;
        lead = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        const int64_t slots = lead + p.vocab;
        const int64_t vecs = (slots + kN - 1) / kN;
        const int64_t v0 = (int64_t)rank * p.vecs;
        n_vecs = (int)(v0 >= vecs ? 0 : (vecs - v0 < p.vecs ? vecs - v0 : p.vecs));
        first = v0 * kN;
        begin = first < lead ? lead : first;
        end = first + (int64_t)n_vecs * kN < slots ? first + (int64_t)n_vecs * kN : slots;
        if (end < begin) end = begin;
    }

    // slot, relative to the slice, of element e; -1 if another CTA holds it
    __device__ __forceinline__ int slot_of(int64_t e) const
    {
        const int64_t s = lead + e;
        return s >= begin && s < end ? (int)(s - first) : -1;
    }

    __device__ __forceinline__ bool whole(int v) const
    {
        const int64_t s = first + (int64_t)v * kN;
        return s >= begin && s + kN <= end;
    }

    // Start loading the slice.  Bulk copies for the whole vectors, chunk c of
    // them on bars[c]; the (at most two) partial vectors by thread 0's warp.
    // Every thread of the CTA calls it, after the barriers' initialisation.
    __device__ __forceinline__ void load(T* smem, uint64_t* bars) const
    {
        int v0 = 0, v1 = n_vecs;
        if (v0 < v1 && !whole(v0)) ++v0;
        if (v0 < v1 && !whole(v1 - 1)) --v1;
        if (threadIdx.x == 0) {
            const int per = (v1 - v0 + kRowChunks - 1) / kRowChunks;
            for (int c = 0; c < kRowChunks; ++c) {
                const int a = v0 + c * per < v1 ? v0 + c * per : v1;
                const int b = a + per < v1 ? a + per : v1;
                mbar_arrive_expect_tx(bars + c, (uint32_t)(b - a) * 16u);
                if (b > a)
                    bulk_g2s(smem + (size_t)a * kN, row + (first + (int64_t)a * kN - lead),
                             (uint32_t)(b - a) * 16u, bars + c);
            }
        }
        const int t = threadIdx.x;
        if (t < 2 * kN) {
            const int v = t < kN ? 0 : n_vecs - 1;
            const bool second = t >= kN;
            if (v >= 0 && v < n_vecs && !whole(v) && !(second && v == 0)) {
                const int64_t s = first + (int64_t)v * kN + t % kN;
                smem[v * kN + t % kN] =
                    s >= begin && s < end ? row[s - lead] : Vec16<T>::from_f32(neg_inf());
            }
        }
    }
};

// Larger-of-maxima merge of two (maximum, sum of exp2((x - maximum) c)).
__device__ __forceinline__ void merge_sum(float& m, float& s, float m2, float s2, float c)
{
    const float top = fmaxf(m, m2);
    if (top == neg_inf()) return;
    s = s * exp2f((m - top) * c) + s2 * exp2f((m2 - top) * c);
    m = top;
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

}  // namespace quasar
