// The pieces of the linear layers' backward pass beside the large products: the
// weight gradient of a few tokens, the bias gradient and the gradient through a
// layer's own activation.
#pragma once

#include "linear.cuh"

namespace quasar {

// dr = dz^T x and dbias for up to TOKENS tokens: a sum of that many outer
// products, bound by writing dr.  A thread keeps 8 inputs of every token in
// registers (in fp32 results two runs of 4, so that a warp's stores are 512
// consecutive bytes either way) and walks kOuterFeatures features.  1 to 4
// tokens through 14336 x 4096: 20 us in bf16, 5.9 TB/s, 8 tokens 24, where the
// tensor cores' kernels store 64 bytes a warp and step and take 36.
constexpr int kOuterThreads = 256;
constexpr int kOuterFeatures = 32;

template <int TOKENS, bool F32>
__global__ void __launch_bounds__(kOuterThreads) k_outer(const __grid_constant__ OuterParams p)
{
    using bf16 = __nv_bfloat16;
    extern __shared__ uint8_t smem_raw[];
    float* dz = reinterpret_cast<float*>(smem_raw);  // [kOuterFeatures][TOKENS]
    const int t = threadIdx.x, lane = t & 31;
    const int64_t n0 = (int64_t)blockIdx.y * kOuterFeatures;
    const int features = (int)(p.features - n0 < kOuterFeatures ? p.features - n0 : kOuterFeatures);
    // inputs of the warp from k0, of the thread's pair q at place(q)
    const int64_t k0 = ((int64_t)blockIdx.x * kOuterThreads + (t & ~31)) * 8;
    auto place = [&](int q) { return F32 ? (q >> 1) * 128 + lane * 4 + (q & 1) * 2 : lane * 8 + q * 2; };
    const bool whole = k0 + 256 <= p.inputs;
    wait_for_previous_grid();
    for (int i = t; i < kOuterFeatures * TOKENS; i += kOuterThreads) {
        const int n = i / TOKENS, m = i % TOKENS;
        dz[i] = n < features && m < p.tokens
                    ? __bfloat162float(static_cast<const bf16*>(p.dz)[m * p.ld_dz + n0 + n])
                    : 0.0f;
    }
    float2 x[TOKENS][4];
#pragma unroll
    for (int m = 0; m < TOKENS; ++m) {
#pragma unroll
        for (int q = 0; q < 4; ++q) x[m][q] = make_float2(0.0f, 0.0f);
        if (m >= p.tokens) continue;
        const bf16* from = static_cast<const bf16*>(p.x) + m * p.ld_x + k0;
        if (whole) {
            uint2 w[2];
            if constexpr (F32) {
                w[0] = *reinterpret_cast<const uint2*>(from + place(0));
                w[1] = *reinterpret_cast<const uint2*>(from + place(2));
            } else {
                const uint4 v = *reinterpret_cast<const uint4*>(from + place(0));
                w[0] = make_uint2(v.x, v.y);
                w[1] = make_uint2(v.z, v.w);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t u = q & 1 ? w[q / 2].y : w[q / 2].x;
                x[m][q] = make_float2(bf16lo(u), bf16hi(u));
            }
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (k0 + place(q) < p.inputs) x[m][q].x = __bfloat162float(from[place(q)]);
                if (k0 + place(q) + 1 < p.inputs) x[m][q].y = __bfloat162float(from[place(q) + 1]);
            }
        }
    }
    __syncthreads();
    if (p.dbias && blockIdx.x == 0 && t < features) {
        float s = 0.0f;
        for (int m = 0; m < p.tokens; ++m) s += dz[t * TOKENS + m];
        p.dbias[n0 + t] = s;
    }
    if (!p.dr || k0 >= p.inputs) return;
    using Out = std::conditional_t<F32, float, bf16>;
    Out* to = static_cast<Out*>(p.dr) + n0 * p.ld_dr + k0;
    const bool vectors = whole && (reinterpret_cast<uintptr_t>(to) & 15) == 0 && p.ld_dr * sizeof(Out) % 16 == 0;
#pragma unroll 2
    for (int n = 0; n < features; ++n, to += p.ld_dr) {
        float2 y[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) y[q] = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int m = 0; m < TOKENS; ++m) {
            const float d = dz[n * TOKENS + m];
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] = __ffma2_rn(make_float2(d, d), x[m][q], y[q]);
        }
        if (vectors) {
            if constexpr (F32) {
                __stcs(reinterpret_cast<float4*>(to + place(0)), make_float4(y[0].x, y[0].y, y[1].x, y[1].y));
                __stcs(reinterpret_cast<float4*>(to + place(2)), make_float4(y[2].x, y[2].y, y[3].x, y[3].y));
            } else {
                __stcs(reinterpret_cast<uint4*>(to + place(0)),
                       make_uint4(pack_bf16x2(y[0].x, y[0].y), pack_bf16x2(y[1].x, y[1].y),
                                  pack_bf16x2(y[2].x, y[2].y), pack_bf16x2(y[3].x, y[3].y)));
            }
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (k0 + place(q) < p.inputs) to[place(q)] = (Out)y[q].x;
                if (k0 + place(q) + 1 < p.inputs) to[place(q) + 1] = (Out)y[q].y;
            }
        }
    }
}

// dbias[j] = sum over rows of dz[row][j] in fp32.  64 columns per cluster of 8
// CTAs of 8 warps; warp w of CTA c takes the rows c + 8 w + 64 q, and the 64
// partial sums of a column are added in a fixed order.
__global__ void __launch_bounds__(256) k_column_sum(const __grid_constant__ ColumnSumParams p)
{
    extern __shared__ uint8_t smem_raw[];
    float2* part = reinterpret_cast<float2*>(smem_raw);  // [8 warps][32 lanes]
    float2* peers = part + 256;                          // [8 CTAs][32 lanes], used by rank 0
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank();
    const int64_t col = (int64_t)(blockIdx.x / 8) * 64 + 2 * lane;
    const __nv_bfloat16* in = static_cast<const __nv_bfloat16*>(p.in) + col;
    float2 s = make_float2(0.0f, 0.0f);
    cluster_arrive();
    wait_for_previous_grid();
    if (col + 1 < p.cols) {
#pragma unroll 8
        for (int64_t r = rank + 8 * warp; r < p.rows; r += 64) {
            const uint32_t x = *reinterpret_cast<const uint32_t*>(in + r * p.ld);
            s.x += bf16lo(x);
            s.y += bf16hi(x);
        }
    } else if (col < p.cols) {
        for (int64_t r = rank + 8 * warp; r < p.rows; r += 64) s.x += __bfloat162float(in[r * p.ld]);
    }
    part[warp * 32 + lane] = s;
    __syncthreads();
    cluster_wait();
    if (warp == 0) {
        for (int w = 1; w < 8; ++w) {
            s.x += part[w * 32 + lane].x;
            s.y += part[w * 32 + lane].y;
        }
        const uint32_t to = peer_addr(smem_u32(peers + rank * 32 + lane), 0);
        st_peer(to, s.x);
        st_peer(to + 4, s.y);
    }
    cluster_sync();
    if (rank == 0 && warp == 0) {
        s = peers[lane];
        for (int c = 1; c < 8; ++c) {
            s.x += peers[c * 32 + lane].x;
            s.y += peers[c * 32 + lane].y;
        }
        if (col < p.cols) p.out[col] = s.x;
        if (col + 1 < p.cols) p.out[col + 1] = s.y;
    }
}

// dz = dy act'(pre), rounded once to bf16 (pre NULL: a strided copy).  One
// element a thread, so bound by its loads' number: 4096 x 12288 takes 237 us
// with SiLU, 1.3 TB/s, and 199 us as a copy of odd rows.
__global__ void __launch_bounds__(256) k_activation_grad(const __grid_constant__ ActGradParams p)
{
    wait_for_previous_grid();
    const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (col >= p.cols) return;
    const __nv_bfloat16* dy = static_cast<const __nv_bfloat16*>(p.dy);
    const __nv_bfloat16* pre = static_cast<const __nv_bfloat16*>(p.pre);
    __nv_bfloat16* dz = static_cast<__nv_bfloat16*>(p.dz);
    for (int64_t r = blockIdx.y; r < p.rows; r += gridDim.y) {
        float d[1] = {__bfloat162float(dy[r * p.ld_dy + col])};
        if (pre) {
            const float z[1] = {__bfloat162float(pre[r * p.ld_pre + col])};
            times_slope(d, z, p.act);
        }
        dz[r * p.ld_dz + col] = __float2bfloat16_rn(d[0]);
    }
}

}  // namespace quasar
