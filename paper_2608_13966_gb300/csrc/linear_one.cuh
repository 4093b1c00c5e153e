// The forward product for one token: r is read once, at the memory's rate, and
// multiplied on the FP32 pipe.
//
// A CTA takes 4 features and splits their rows over its 8 warps, so that the
// 32 KB of four rows of 4,096 are all on their way at once; x comes from L1.
// Bound by HBM: 14336 x 4096 takes 22.0 us, 5.3 TB/s.  (From two tokens on the
// tensor cores' kernel is faster: see the rule in the launch.)
#pragma once

#include "linear.cuh"

namespace quasar {

constexpr int kOneFeatures = 4;
constexpr int kOneWarps = 8;

__device__ __forceinline__ void unpack8(const uint4& x, float2 (&v)[4])
{
    v[0] = make_float2(bf16lo(x.x), bf16hi(x.x));
    v[1] = make_float2(bf16lo(x.y), bf16hi(x.y));
    v[2] = make_float2(bf16lo(x.z), bf16hi(x.z));
    v[3] = make_float2(bf16lo(x.w), bf16hi(x.w));
}

__global__ void __launch_bounds__(32 * kOneWarps) k_linear_one(const __grid_constant__ OneParams p)
{
    using bf16 = __nv_bfloat16;
    constexpr int kF = kOneFeatures;
    extern __shared__ uint8_t smem_raw[];
    float* parts = reinterpret_cast<float*>(smem_raw);  // [warps][features]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t f0 = (int64_t)blockIdx.x * kF;
    const int64_t vecs = p.inputs / 8;
    const bf16* x = static_cast<const bf16*>(p.x);
    // the last four may be fewer: a row beyond is the last again
    const uint4* row[kF];
    float2 acc[kF];
#pragma unroll
    for (int f = 0; f < kF; ++f) {
        row[f] = reinterpret_cast<const uint4*>(static_cast<const bf16*>(p.r) +
                                                (f0 + f < p.features ? f0 + f : p.features - 1) * p.ld_r);
        acc[f] = make_float2(0.0f, 0.0f);
    }
    wait_for_previous_grid();

#pragma unroll 2
    for (int64_t v = threadIdx.x; v < vecs; v += 32 * kOneWarps) {
        uint4 raw[kF];
#pragma unroll
        for (int f = 0; f < kF; ++f) raw[f] = __ldcs(row[f] + v);
        float2 xs[4];
        unpack8(reinterpret_cast<const uint4*>(x)[v], xs);
#pragma unroll
        for (int f = 0; f < kF; ++f) {
            float2 w[4];
            unpack8(raw[f], w);
#pragma unroll
            for (int q = 0; q < 4; ++q) acc[f] = __ffma2_rn(w[q], xs[q], acc[f]);
        }
    }
    // inputs beyond the last whole vector, one a thread
    const int64_t k = vecs * 8 + threadIdx.x;
    if (k < p.inputs) {
#pragma unroll
        for (int f = 0; f < kF; ++f)
            acc[f].x += __bfloat162float(reinterpret_cast<const bf16*>(row[f])[k]) * __bfloat162float(x[k]);
    }
#pragma unroll
    for (int f = 0; f < kF; ++f) {
        float s = acc[f].x + acc[f].y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) parts[warp * kF + f] = s;
    }
    __syncthreads();
    if (threadIdx.x < kF) {
        const int64_t i = f0 + threadIdx.x;
        float s[1] = {0.0f};
#pragma unroll
        for (int w = 0; w < kOneWarps; ++w) s[0] += parts[w * kF + threadIdx.x];
        finish(p.e, s, i, 0, p.features, 1, p.e.bias && i < p.features ? p.e.bias[i] : 0.0f);
    }
}

}  // namespace quasar
