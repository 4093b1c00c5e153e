// The pieces of the linear layers' backward pass that are not products: the
// bias gradient and the gradient through a layer's own activation.
#pragma once

#include "linear.cuh"

namespace quasar {

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

// dz = dy act'(pre), rounded once to bf16 (pre NULL: a strided copy).
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
