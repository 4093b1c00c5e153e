// Rows of bf16 or fp32 shared out to T threads, 8 elements at a time.
#pragma once

#include "device_common.cuh"

namespace quasar {

// Elements of thread t: with VECTORS runs of 8 (rows start at 16-byte
// boundaries), else single elements T apart.
template <int T, bool VECTORS>
__device__ __forceinline__ int row_at(int t, int j, int i)
{
    return VECTORS ? (j * T + t) * 8 + i : (j * 8 + i) * T + t;
}

// 8 elements as they lie in memory: the raw words of a row on its way.
// WIDE: fp32 is possible (the type is known at run time).
template <bool WIDE>
struct Raw8 {
    uint32_t w[WIDE ? 8 : 4];
};

template <int T, bool VECTORS, bool WIDE>
__device__ __forceinline__ void load_raw(Raw8<WIDE>& r, const void* row, bool f32, int t, int j, int cols)
{
    const __nv_bfloat16* h = static_cast<const __nv_bfloat16*>(row);
    const float* f = static_cast<const float*>(row);
#pragma unroll
    for (int q = 0; q < (WIDE ? 8 : 4); ++q) r.w[q] = 0;
    const int c0 = row_at<T, VECTORS>(t, j, 0);
    if (VECTORS && c0 + 8 <= cols) {
        if (WIDE && f32) {
            const uint4 a = __ldcs(reinterpret_cast<const uint4*>(f + c0));
            const uint4 b = __ldcs(reinterpret_cast<const uint4*>(f + c0) + 1);
            r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w;
            r.w[WIDE ? 4 : 0] = b.x, r.w[WIDE ? 5 : 0] = b.y, r.w[WIDE ? 6 : 0] = b.z, r.w[WIDE ? 7 : 0] = b.w;
        } else {
            const uint4 a = __ldcs(reinterpret_cast<const uint4*>(h + c0));
            r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = row_at<T, VECTORS>(t, j, i);
        if (c >= cols) continue;
        if (WIDE && f32) {
            r.w[WIDE ? i : 0] = __float_as_uint(f[c]);
        } else {
            const uint32_t bits = __bfloat16_as_ushort(h[c]);
            r.w[i / 2] |= i & 1 ? bits << 16 : bits;
        }
    }
}

template <bool WIDE>
__device__ __forceinline__ void unpack_raw(const Raw8<WIDE>& r, bool f32, float (&v)[8])
{
    if (WIDE && f32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[WIDE ? i : 0]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i & 1 ? bf16hi(r.w[i / 2]) : bf16lo(r.w[i / 2]);
    }
}

template <int T, bool VECTORS>
__device__ __forceinline__ void load_floats(float (&v)[8], const float* row, int t, int j, int cols, float none)
{
    const int c0 = row_at<T, VECTORS>(t, j, 0);
    if (VECTORS && row && c0 + 8 <= cols) {
        const float4 a = *reinterpret_cast<const float4*>(row + c0), b = *reinterpret_cast<const float4*>(row + c0 + 4);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = row_at<T, VECTORS>(t, j, i);
        v[i] = c < cols ? (row ? row[c] : none) : 0.0f;
    }
}

template <int T, bool VECTORS>
__device__ __forceinline__ void store_row(void* row, bool f32, int t, int j, int cols, const float (&v)[8])
{
    __nv_bfloat16* h = static_cast<__nv_bfloat16*>(row);
    float* f = static_cast<float*>(row);
    const int c0 = row_at<T, VECTORS>(t, j, 0);
    if (VECTORS && c0 + 8 <= cols) {
        if (f32) {
            reinterpret_cast<float4*>(f + c0)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(f + c0)[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint4*>(h + c0) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                           pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = row_at<T, VECTORS>(t, j, i);
        if (c >= cols) continue;
        if (f32)
            f[c] = v[i];
        else
            h[c] = __float2bfloat16_rn(v[i]);
    }
}

__device__ __forceinline__ const void* row_of(const void* p, bool f32, int64_t row, int64_t ld)
{
    return static_cast<const uint8_t*>(p) + row * ld * (f32 ? 4 : 2);
}

__device__ __forceinline__ void* row_of(void* p, bool f32, int64_t row, int64_t ld)
{
    return static_cast<uint8_t*>(p) + row * ld * (f32 ? 4 : 2);
}

}  // namespace quasar
