// Matrix products with the reconstructed weights: y = act(x r^T + bias) +
// residual and the two products of its backward pass, on the 5th-generation
// tensor cores.
//
// Every product is written as D[i][j] = sum_k A[i][k] B[j][k] with i the
// coordinate that is contiguous in the result's memory:
//
//   forward          i = feature, j = token, k = input    A = r,  B = x
//   input gradient   i = input,   j = token, k = feature  A = r^T, B = dz
//   weight gradient  i = input,   j = feature, k = token  A = x^T, B = dz^T
//
// so that an accumulator lane (a row of D in tensor memory) is a memory
// column: one accumulator column stored by a warp is 32 consecutive results.
// No result is staged through shared memory, and results may start at any
// element and have any row stride.  A transposed operand is read as it lies
// in memory (an MN-major tile); nothing is transposed on the way.
#pragma once

#include <type_traits>

#include "cluster.cuh"
#include "linear.h"
#include "quasar.h"
#include "tensor_core.cuh"

namespace quasar {

constexpr int kTileRows = 128;          // rows of D a CTA owns: the lanes of tensor memory
constexpr int kTileK = 64;              // 128 bytes of bf16: one swizzled row
constexpr uint32_t kTileABytes = kTileRows * kTileK * 2;

// -- activations -------------------------------------------------------------

__device__ __forceinline__ float ex2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float rcp_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 1 / (1 + e^-z), to 2^-22 of itself where it is not small: with the accurate
// exponential and division instead, the epilogue of a 256 x 256 tile took
// longer than its product at 4096 inputs.
__device__ __forceinline__ float sigmoid(float z) { return rcp_approx(1.0f + ex2_approx(-1.44269504f * z)); }

// The normal distribution Phi(z) and its density, from erfc(x) = e^(-x^2) t
// (a1 + t (a2 + ...)), t = 1 / (1 + 0.3275911 x), x >= 0 (Abramowitz and
// Stegun, Handbook of Mathematical Functions, 7.1.26: error 1.5e-7).
__device__ __forceinline__ void normal(float z, float& phi, float& density)
{
    const float x = fabsf(z) * 0.70710678f;
    const float t = rcp_approx(fmaf(0.3275911f, x, 1.0f));
    const float e = ex2_approx(-0.72134752f * z * z);
    float q = fmaf(1.061405429f, t, -1.453152027f);
    q = fmaf(q, t, 1.421413741f);
    q = fmaf(q, t, -0.284496736f);
    q = fmaf(q, t, 0.254829592f);
    const float tail = 0.5f * q * t * e;  // beyond |z|
    phi = z < 0.0f ? tail : 1.0f - tail;
    density = 0.39894228f * e;
}

template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int act)
{
    if (act == QUASAR_ACT_RELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] = v[c] < 0.0f ? 0.0f : v[c];  // (a NaN stays one)
    } else if (act == QUASAR_ACT_SILU) {
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] *= sigmoid(v[c]);
    } else if (act == QUASAR_ACT_GELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            float phi, density;
            normal(v[c], phi, density);
            v[c] *= phi;
        }
    }
}

// Infinities brought in, where the slopes' products have their limits 0 and 1
// (a NaN comes in too, and comes out again with the other factor).
__device__ __forceinline__ float bring_in(float z) { return fminf(fmaxf(z, -1e30f), 1e30f); }

// v *= act'(z)
template <int N>
__device__ __forceinline__ void times_slope(float (&v)[N], const float (&z)[N], int act)
{
    if (act == QUASAR_ACT_RELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] = z[c] > 0.0f ? v[c] : (z[c] <= 0.0f ? 0.0f : z[c]);
    } else if (act == QUASAR_ACT_SILU) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const float s = sigmoid(z[c]);
            v[c] *= s * fmaf(bring_in(z[c]), 1.0f - s, 1.0f);
        }
    } else if (act == QUASAR_ACT_GELU) {
#pragma unroll
        for (int c = 0; c < N; ++c) {
            float phi, density;
            normal(z[c], phi, density);
            v[c] *= fmaf(bring_in(z[c]), density, phi);
        }
    }
}

// -- epilogue ----------------------------------------------------------------

// Element (row j, column i) of a row-major matrix, walked down a column: the
// address is one addition a row.
template <typename T, int N, bool FULL>
__device__ __forceinline__ void load_column(const void* base, int64_t ld, int64_t j0, int64_t i, int n, float (&v)[N])
{
    const T* p = static_cast<const T*>(base) + j0 * ld + i;
#pragma unroll
    for (int c = 0; c < N; ++c, p += ld) {
        v[c] = 0.0f;
        if (FULL || c < n) {
            if constexpr (sizeof(T) == 2)
                v[c] = __bfloat162float(*p);
            else
                v[c] = *p;
        }
    }
}

template <typename T, int N, bool FULL>
__device__ __forceinline__ void store_column(void* base, int64_t ld, int64_t j0, int64_t i, int n, const float (&v)[N])
{
    T* p = static_cast<T*>(base) + j0 * ld + i;
#pragma unroll
    for (int c = 0; c < N; ++c, p += ld)
        if (FULL || c < n) {
            if constexpr (sizeof(T) == 2)
                *p = __float2bfloat16_rn(v[c]);
            else
                *p = v[c];
        }
}

template <int N, bool FULL>
__device__ __forceinline__ void finish_columns(const Epilogue& e, float (&v)[N], int64_t i, int64_t j0, int n, float bias)
{
    using bf16 = __nv_bfloat16;
    float res[N];
    if (e.residual) {
        if (e.out_f32)
            load_column<float, N, FULL>(e.residual, e.ld_res, j0, i, n, res);
        else
            load_column<bf16, N, FULL>(e.residual, e.ld_res, j0, i, n, res);
    }
    if (e.scale_pre) {
        float z[N];
        load_column<bf16, N, FULL>(e.scale_pre, e.ld_scale, j0, i, n, z);
        times_slope(v, z, e.act);
    } else {
        if (e.bias) {
#pragma unroll
            for (int c = 0; c < N; ++c) v[c] += bias;
        }
        if (e.pre) store_column<bf16, N, FULL>(e.pre, e.ld_pre, j0, i, n, v);
        activate(v, e.act);
    }
    if (e.residual) {
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] += res[c];
    }
    if (e.out_f32)
        store_column<float, N, FULL>(e.out, e.ld_out, j0, i, n, v);
    else
        store_column<bf16, N, FULL>(e.out, e.ld_out, j0, i, n, v);
}

// N consecutive columns j0.. (rows of memory) of one row i: bias, activation
// (or the input activation's slope), residual, one rounding to the output's
// type.
template <int N>
__device__ __forceinline__ void finish(const Epilogue& e, float (&v)[N], int64_t i, int64_t j0,
                                       int64_t rows, int64_t cols, float bias)
{
    if (i >= rows || j0 >= cols) return;
    if (cols - j0 >= N)
        finish_columns<N, true>(e, v, i, j0, N, bias);
    else
        finish_columns<N, false>(e, v, i, j0, (int)(cols - j0), bias);
}

// 4 consecutive rows i.. (consecutive in memory) of one column j: as finish,
// with one access for the four where they are aligned.
template <typename T>
__device__ __forceinline__ void finish_four(const Epilogue& e, float (&v)[4], int64_t i, int64_t j)
{
    using bf16 = __nv_bfloat16;
    auto vector = [](const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; };
    auto load = [&](auto* p, float (&x)[4]) {
        using E = std::remove_cv_t<std::remove_pointer_t<decltype(p)>>;
        if (vector(p, 4 * sizeof(E))) {
            if constexpr (sizeof(E) == 2) {
                const uint2 w = *reinterpret_cast<const uint2*>(p);
                x[0] = bf16lo(w.x), x[1] = bf16hi(w.x), x[2] = bf16lo(w.y), x[3] = bf16hi(w.y);
            } else {
                const float4 w = *reinterpret_cast<const float4*>(p);
                x[0] = w.x, x[1] = w.y, x[2] = w.z, x[3] = w.w;
            }
        } else {
            for (int q = 0; q < 4; ++q) x[q] = (float)p[q];
        }
    };
    auto store = [&](auto* p, const float (&x)[4]) {
        using E = std::remove_pointer_t<decltype(p)>;
        if (vector(p, 4 * sizeof(E))) {
            if constexpr (sizeof(E) == 2)
                *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
            else
                *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
        } else {
            for (int q = 0; q < 4; ++q) p[q] = (E)x[q];
        }
    };
    float res[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (e.residual) load(static_cast<const T*>(e.residual) + j * e.ld_res + i, res);
    if (e.scale_pre) {
        float z[4];
        load(static_cast<const bf16*>(e.scale_pre) + j * e.ld_scale + i, z);
        times_slope(v, z, e.act);
    } else {
        if (e.bias) {
            float b[4];
            load(e.bias + i, b);
            for (int q = 0; q < 4; ++q) v[q] += b[q];
        }
        if (e.pre) store(static_cast<bf16*>(e.pre) + j * e.ld_pre + i, v);
        activate(v, e.act);
    }
    for (int q = 0; q < 4; ++q) v[q] += res[q];
    store(static_cast<T*>(e.out) + j * e.ld_out + i, v);
}

__device__ __forceinline__ void finish_rows(const Epilogue& e, const float4& x, int64_t i, int64_t j, int64_t rows)
{
    float v[4] = {x.x, x.y, x.z, x.w};
    if (i + 4 <= rows) {
        if (e.out_f32)
            finish_four<float>(e, v, i, j);
        else
            finish_four<__nv_bfloat16>(e, v, i, j);
    } else {
        for (int q = 0; q < 4; ++q) {
            float one[1] = {v[q]};
            finish(e, one, i + q, j, rows, j + 1, e.bias && i + q < rows ? e.bias[i + q] : 0.0f);
        }
    }
}

// -- one tile per cluster ------------------------------------------------------

// BN columns (tokens, for the forward product) by 128 rows per cluster, the
// reduction split over the cluster's CTAs.  Each CTA multiplies its share
// into its own tensor memory; the partial tiles are then exchanged through
// distributed shared memory and summed in rank order (always the same order,
// so the result does not depend on timing), each CTA finishing BN / split of
// the columns.
//
// PROMOTE: fp32 results.  The tensor core truncates as it accumulates, an
// error that grows with the number of instructions (relative to the result's
// norm 9e-7 after 1024 products, 4.7e-7 after 512; a plain fp32 product of
// 4096 has 6e-7).  So every kPromoteBlocks blocks of the reduction go to a
// fresh accumulator, two taking turns, and the epilogue adds the parts up in
// registers, rounding to nearest.
//
// Bound by r's bytes for few columns (23 x 4096 x 14336: 23.4 us, 5.1 TB/s),
// by the operands' way from L2 for more (each byte serves 128 rows or columns:
// 1001 x 1003 x 4096 in fp32, 21.5 us); larger products go to the paired tiles.
//
// Warps: 0-3 epilogue (one per 32 lanes of tensor memory), 4 copies, 5
// matrix instructions.
constexpr int kPromoteBlocks = 8;

template <int BN, bool A_MN, bool B_MN, bool PROMOTE>
__global__ void __launch_bounds__(192, 2) k_product_tile(const __grid_constant__ ProductParams p)
{
    constexpr uint32_t kBBytes = BN * kTileK * 2;
    constexpr uint32_t kStageBytes = kTileABytes + kBBytes;
    constexpr uint32_t kColumns = (PROMOTE ? 2 : 1) * BN < 32 ? 32 : (PROMOTE ? 2 : 1) * BN;
    static_assert(!B_MN || BN % 64 == 0, "an MN-major tile is made of 64-wide blocks");

    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int stages = p.stages;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + (size_t)stages * kStageBytes);
    uint64_t* empty = full + stages;
    uint64_t* acc_full = empty + stages;   // [2]
    uint64_t* acc_empty = acc_full + 2;    // [2]: 4 epilogue warps
    uint64_t* drained = acc_empty + 2;
    uint64_t* never = drained + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(never + 1);
    volatile uint32_t* gone = tmem_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = p.split > 1 ? (int)cluster_rank() : 0;
    const int64_t tile = blockIdx.x / p.split;
    const int64_t row0 = (tile % p.tiles_row) * kTileRows;
    const int64_t col0 = (tile / p.tiles_row) * BN;
    const int kb0 = (int)((int64_t)p.k_blocks * rank / p.split);
    const int nkb = (int)((int64_t)p.k_blocks * (rank + 1) / p.split) - kb0;
    const int per_part = PROMOTE ? kPromoteBlocks : nkb;

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(full + s, 1);
            mbar_init(empty + s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full + b, 1);
            mbar_init(acc_empty + b, 4);
        }
        mbar_init(drained, 1);
        mbar_init(never, 1);
        *gone = 0;
        mbar_init_fence();
    }
    if (warp == 5) tmem_alloc<1>(tmem_slot, kColumns);
    if (warp == 4 && lane == 0 && p.k_blocks > 0) {  // (an empty reduction has no maps)
        prefetch_map(&p.a);
        prefetch_map(&p.b);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    wait_for_previous_grid();
    const uint32_t tmem = *tmem_slot;

    if (warp == 4 && lane == 0) {
        if (p.force_timeout_ns) role_wait(never, 0, gone, p.force_timeout_ns, p.status);
        int it = 0;
        for (; it < nkb; ++it) {
            const int s = it % stages;
            if (it >= stages && !role_wait(empty + s, (it / stages - 1) & 1, gone, p.timeout_ns, p.status)) break;
            if (*gone) break;
            const uint32_t a = smem_u32(smem + (size_t)s * kStageBytes), b = a + kTileABytes;
            const uint32_t bar = smem_u32(full + s);
            mbar_arrive_expect_tx(full + s, kStageBytes);
            const int k = (kb0 + it) * kTileK;
            if (A_MN) {
#pragma unroll
                for (int q = 0; q < kTileRows / 64; ++q) tile_g2s(a + q * 8192, &p.a, (int)row0 + 64 * q, k, bar);
            } else {
                tile_g2s(a, &p.a, k, (int)row0, bar);
            }
            if (B_MN) {
#pragma unroll
                for (int q = 0; q < BN / 64; ++q) tile_g2s(b + q * 8192, &p.b, (int)col0 + 64 * q, k, bar);
            } else {
                tile_g2s(b, &p.b, k, (int)col0, bar);
            }
        }
        // before the memory is let go: every slot's release has arrived; given
        // up, every copy in flight has landed
        for (int j = it > stages ? it - stages : 0; j < it; ++j)
            if (it < nkb || *gone)
                mbar_wait_bounded(full + j % stages, (j / stages) & 1, p.timeout_ns);
            else
                role_wait(empty + j % stages, (j / stages) & 1, gone, p.timeout_ns, p.status);
    } else if (warp == 5 && lane == 0) {
        constexpr uint32_t desc = mma_desc(kTileRows, BN, A_MN, B_MN);
        bool ok = true;
        int it = 0;
        for (int part = 0; it < nkb && ok; ++part) {
            const int buf = part & 1;
            if (part >= 2 && !role_wait(acc_empty + buf, (part / 2 - 1) & 1, gone, p.timeout_ns, p.status)) break;
            tc_fence_after();
            const int end = it + per_part < nkb ? it + per_part : nkb;
            for (bool add = false; it < end; ++it) {
                const int s = it % stages;
                if (!role_wait(full + s, (it / stages) & 1, gone, p.timeout_ns, p.status)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t a = smem_u32(smem + (size_t)s * kStageBytes);
                uint64_t da = operand_desc(a, A_MN), db = operand_desc(a + kTileABytes, B_MN);
#pragma unroll
                for (int k = 0; k < kTileK / 16; ++k) {
                    mma_bf16<1>(tmem + buf * BN, da, db, desc, add);
                    add = true;
                    da += k_step(A_MN);
                    db += k_step(B_MN);
                }
                mma_commit(smem_u32(empty + s));
            }
            if (ok) mma_commit(smem_u32(acc_full + buf));
        }
        // everything issued is finished before tensor memory is freed
        mma_commit(smem_u32(drained));
        mbar_wait_bounded(drained, 0, p.timeout_ns);
    }
    __syncwarp();
    if (warp < 4) {
        const int64_t i = row0 + 32 * warp + lane;
        const float bias = p.e.bias && i < p.rows ? p.e.bias[i] : 0.0f;
        const uint32_t mine = tmem + ((uint32_t)(32 * warp) << 16);
        float* part = reinterpret_cast<float*>(smem);
        const int n_parts = nkb > 0 ? (nkb + per_part - 1) / per_part : 0;
        uint32_t from = mine;
        float acc[PROMOTE ? BN : 1];
#pragma unroll
        for (float& x : acc) x = 0.0f;
#pragma unroll 1
        for (int q = 0; q < n_parts; ++q) {
            const bool ok = role_wait(acc_full + (q & 1), (q / 2) & 1, gone, p.timeout_ns, p.status);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            from = mine + (q & 1) * BN;
            if constexpr (PROMOTE) {
#pragma unroll
                for (int c = 0; c < BN; c += 16) {
                    float v[16];
                    tmem_ld16(from + c, v);
#pragma unroll
                    for (int x = 0; x < 16; ++x) acc[c + x] += v[x];
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(acc_empty + (q & 1));
            }
        }
        if (PROMOTE && n_parts > 1) {
            // the sums where the last part lay, for the loop below
#pragma unroll
            for (int c = 0; c < BN; c += 16) tmem_st16(from + c, acc + (PROMOTE ? c : 0));
            tmem_wait_st();
        }
#pragma unroll 1
        for (int c = 0; c < BN; c += 16) {
            float v[16];
            if (nkb > 0) {
                __syncwarp();
                tmem_ld16(from + c, v);
            } else {
#pragma unroll
                for (int q = 0; q < 16; ++q) v[q] = 0.0f;
            }
            if (p.split == 1) {
                if (col0 + c < p.cols) finish(p.e, v, i, col0 + c, p.rows, p.cols, bias);
            } else {
                // the operands' memory is free: every product is done
#pragma unroll
                for (int q = 0; q < 16; ++q) part[(c + q) * kTileRows + 32 * warp + lane] = v[q];
            }
        }
    }
    if (p.split > 1) {
        __syncthreads();
        cluster_sync();
        if (warp < 4) {
            // 4 rows of two columns a thread at a time: 16 bytes from each CTA
            const int stop = BN * (rank + 1) / p.split;
            const uint32_t base = smem_u32(smem) + (uint32_t)lane * 16;
            for (int c = BN * rank / p.split + warp; c < stop && col0 + c < p.cols; c += 8) {
                const bool two = c + 4 < stop && col0 + c + 4 < p.cols;
                float4 a[8], b[8];
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < p.split) {
                        const uint32_t from = peer_addr(base, (uint32_t)r) + (uint32_t)c * kTileRows * 4;
                        a[r] = ld_peer4(from);
                        if (two) b[r] = ld_peer4(from + 4 * kTileRows * 4);
                    }
#pragma unroll
                for (int r = 1; r < 8; ++r)
                    if (r < p.split) {
                        a[0].x += a[r].x, a[0].y += a[r].y, a[0].z += a[r].z, a[0].w += a[r].w;
                        if (two) b[0].x += b[r].x, b[0].y += b[r].y, b[0].z += b[r].z, b[0].w += b[r].w;
                    }
                finish_rows(p.e, a[0], row0 + 4 * lane, col0 + c, p.rows);
                if (two) finish_rows(p.e, b[0], row0 + 4 * lane, col0 + c + 4, p.rows);
            }
        }
        cluster_sync();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 5) tmem_free<1>(tmem, kColumns);
}

// -- pairs of CTAs ---------------------------------------------------------------

// 256 x 256 tiles, two CTAs (one on each SM of a pair) a tile, persistent.
// Each CTA keeps its 128 rows of A and half of B's columns in shared memory;
// one thread of the pair's first CTA issues the matrix instructions of both,
// which read the two halves of B from both memories, so an operand byte is
// fetched from L2 once for 256 rows or columns.  The accumulators (128 lanes x
// 256 columns a CTA) use half of tensor memory: the next tile is multiplied
// into the other half while the epilogue drains this one.
//
// PROMOTE: fp32 results, parts of the reduction added up in registers as in
// k_product_tile (8192 x 14336 x 4096 with parts of 512: 667 us against 521
// us for bf16 results, one input set over and over).  Its 64 sums a thread
// leave some of the epilogue's values in local memory; with 8 warps none are,
// and it takes 661.
//
// Bound by the tensor cores and the power they draw: 8192 x 14336 x 4096 with
// bias, SiLU and kept pre-activation takes 615 us, 1.56 PFLOP/s, 0.83 of the
// measured burst rate and 0.91 of the sustained (536 to 572 us, where one input
// set is used over and over).  With a short reduction, by the epilogue: the
// weight gradient of 32 tokens, 14336 x 4096, takes 36 to 45 us.
//
// Warps: 0-15 epilogue (lane quadrant w % 4, 64 columns w / 4; with 8 warps of
// 128 columns 32 tokens' gradient took 56 us against 45, 2560 x 2560 x 1024 with
// SiLU 19.2 against 18.5, the large products the same), 16 copies, 17 matrix
// instructions and, in the second CTA, the drained accumulators' messages.
constexpr int kPairCols = 256;
constexpr int kPairEpilogue = 16;  // warps
constexpr int kPairThreads = (kPairEpilogue + 2) * 32;
constexpr int kPairSpan = 4 * kPairCols / kPairEpilogue;  // columns of an epilogue warp
constexpr int kPairStages = 6;
constexpr int kPairGroup = 8;  // column tiles walked together, for operand reuse in L2
constexpr uint32_t kPairStageBytes = 2 * kTileABytes;

__device__ __forceinline__ void arrive_peer(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

template <bool A_MN, bool B_MN, bool PROMOTE>
__global__ void __launch_bounds__(kPairThreads, 1) k_product_pair(const __grid_constant__ ProductParams p)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + kPairStages * kPairStageBytes);  // first CTA's: both halves landed
    uint64_t* empty = full + kPairStages;   // each CTA's
    uint64_t* acc_full = empty + kPairStages;  // [2], each CTA's
    uint64_t* acc_empty = acc_full + 2;        // [2], each CTA's: its epilogue warps
    uint64_t* peer_empty = acc_empty + 2;      // [2], first CTA's: the second's acc_empty, passed on
    uint64_t* drained = peer_empty + 2;
    uint64_t* never = drained + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(never + 1);
    volatile uint32_t* gone = tmem_slot + 1;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int pair = (int)(blockIdx.x >> 1), n_pairs = (int)(gridDim.x >> 1);
    const int64_t n_tiles = (int64_t)p.tiles_row * p.tiles_col;
    const int nkb = p.k_blocks;
    const int per_part = PROMOTE ? kPromoteBlocks : nkb;
    const int n_parts = (nkb + per_part - 1) / per_part;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; ++s) {
            mbar_init(full + s, 1);
            mbar_init(empty + s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(acc_full + b, 1);
            mbar_init(acc_empty + b, kPairEpilogue);
            mbar_init(peer_empty + b, 1);
        }
        mbar_init(drained, 1);
        mbar_init(never, 1);
        *gone = 0;
        mbar_init_fence();
    }
    if (warp == kPairEpilogue + 1) tmem_alloc<2>(tmem_slot, 512);
    if (warp == kPairEpilogue && lane == 0) {
        prefetch_map(&p.a);
        prefetch_map(&p.b);
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
    wait_for_previous_grid();
    const uint32_t tmem = *tmem_slot;

    // tile t: groups of kPairGroup column tiles, row tiles within a group
    auto tile_at = [&](int64_t t, int64_t& row0, int64_t& col0) {
        const int64_t group = t / ((int64_t)kPairGroup * p.tiles_row);
        const int64_t in = t - group * kPairGroup * p.tiles_row;
        const int64_t left = p.tiles_col - group * kPairGroup;
        const int wide = (int)(left < kPairGroup ? left : kPairGroup);
        row0 = in / wide * 256 + 128 * rank;  // of this CTA
        col0 = (group * kPairGroup + in % wide) * kPairCols;
    };

    if (warp == kPairEpilogue && lane == 0) {
        if (p.force_timeout_ns) role_wait(never, 0, gone, p.force_timeout_ns, p.status);
        uint32_t it = 0;
        for (int64_t t = pair; t < n_tiles && !*gone; t += n_pairs) {
            int64_t row0, col0;
            tile_at(t, row0, col0);
            const int bcol = (int)col0 + 128 * (int)rank;
            for (int kb = 0; kb < nkb; ++kb, ++it) {
                const int s = it % kPairStages;
                if (it >= kPairStages &&
                    !role_wait(empty + s, (it / kPairStages - 1) & 1, gone, p.timeout_ns, p.status))
                    break;
                const uint32_t a = smem_u32(smem + (size_t)s * kPairStageBytes), b = a + kTileABytes;
                const uint32_t bar = peer_addr(smem_u32(full + s), 0);
                if (rank == 0) mbar_arrive_expect_tx(full + s, 2 * kPairStageBytes);
                const int k = kb * kTileK;
                if (A_MN) {
                    tile_g2s_pair(a, &p.a, (int)row0, k, bar);
                    tile_g2s_pair(a + 8192, &p.a, (int)row0 + 64, k, bar);
                } else {
                    tile_g2s_pair(a, &p.a, k, (int)row0, bar);
                }
                if (B_MN) {
                    tile_g2s_pair(b, &p.b, bcol, k, bar);
                    tile_g2s_pair(b + 8192, &p.b, bcol + 64, k, bar);
                } else {
                    tile_g2s_pair(b, &p.b, k, bcol, bar);
                }
            }
        }
        // before the memory is let go: every slot's release has arrived, which
        // the first CTA's instructions send to both; given up, what is in
        // flight has landed (the second CTA's copies report to the first, which
        // waits for both)
        for (uint32_t j = it > kPairStages ? it - kPairStages : 0; j < it; ++j)
            if (!*gone)
                role_wait(empty + j % kPairStages, (j / kPairStages) & 1, gone, p.timeout_ns, p.status);
            else if (rank == 0)
                mbar_wait_bounded(full + j % kPairStages, (j / kPairStages) & 1, p.timeout_ns);
    } else if (warp == kPairEpilogue + 1 && lane == 0 && rank == 0) {
        constexpr uint32_t desc = mma_desc(256, kPairCols, A_MN, B_MN);
        uint32_t it = 0, part = 0;
        bool ok = true;
        for (int64_t t = pair; t < n_tiles && ok; t += n_pairs) {
            for (int kb = 0; kb < nkb && ok; ++part) {
                const uint32_t buf = part & 1;
                const uint32_t before = (part / 2 - 1) & 1;
                if (part >= 2 && !(role_wait(acc_empty + buf, before, gone, p.timeout_ns, p.status) &&
                                   role_wait(peer_empty + buf, before, gone, p.timeout_ns, p.status))) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t d = tmem + buf * kPairCols;
                const int end = kb + per_part < nkb ? kb + per_part : nkb;
                for (bool add = false; kb < end; ++kb, ++it) {
                    const int s = it % kPairStages;
                    if (!role_wait(full + s, (it / kPairStages) & 1, gone, p.timeout_ns, p.status)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t a = smem_u32(smem + (size_t)s * kPairStageBytes);
                    uint64_t da = operand_desc(a, A_MN), db = operand_desc(a + kTileABytes, B_MN);
#pragma unroll
                    for (int k = 0; k < kTileK / 16; ++k) {
                        mma_bf16<2>(d, da, db, desc, add);
                        add = true;
                        da += k_step(A_MN);
                        db += k_step(B_MN);
                    }
                    mma_commit_pair(smem_u32(empty + s));
                }
                if (ok) mma_commit_pair(smem_u32(acc_full + buf));
            }
        }
        mma_commit_local_pair(smem_u32(drained));
        mbar_wait_bounded(drained, 0, p.timeout_ns);
    } else if (warp == kPairEpilogue + 1 && lane == 0) {
        // The second CTA's drained accumulators, passed on.  (An arrival at the
        // other CTA waits for its thread's earlier stores to global memory: done
        // by the epilogue's warps it cost the gradient of 32 tokens 10 us.)
        uint32_t part = 0;
        bool ok = true;
        for (int64_t t = pair; t < n_tiles && ok; t += n_pairs)
            for (int q = 0; q < n_parts && ok; ++q, ++part) {
                ok = role_wait(acc_empty + (part & 1), (part / 2) & 1, gone, p.timeout_ns, p.status);
                tc_fence_after();
                tc_fence_before();
                if (ok) arrive_peer(peer_addr(smem_u32(peer_empty + (part & 1)), 0));
            }
    } else if (warp < kPairEpilogue) {
        const int quad = warp & 3, span = warp >> 2;
        const uint32_t mine = tmem + ((uint32_t)(32 * quad) << 16) + kPairSpan * span;
        uint32_t part = 0;
        for (int64_t t = pair; t < n_tiles; t += n_pairs) {
            int64_t row0, col0;
            tile_at(t, row0, col0);
            col0 += kPairSpan * span;
            const int64_t i = row0 + 32 * quad + lane;
            const float bias = p.e.bias && i < p.rows ? p.e.bias[i] : 0.0f;
            float acc[PROMOTE ? kPairSpan : 1];
#pragma unroll
            for (float& x : acc) x = 0.0f;
            bool ok = true;
            uint32_t from = mine;
#pragma unroll 1
            for (int q = 0; q < n_parts && ok; ++q, ++part) {
                const uint32_t buf = part & 1;
                ok = role_wait(acc_full + buf, (part / 2) & 1, gone, p.timeout_ns, p.status);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                tc_fence_after();
                from = mine + buf * kPairCols;
                if constexpr (PROMOTE) {
#pragma unroll
                    for (int c = 0; c < kPairSpan; c += 16) {
                        float v[16];
                        tmem_ld16(from + c, v);
#pragma unroll
                        for (int x = 0; x < 16; ++x) acc[c + x] += v[x];
                    }
                    if (q + 1 < n_parts) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(acc_empty + buf);
                    }
                }
            }
            if (!ok) break;
            if constexpr (PROMOTE) {
                // the sums back where the last part lay, for the epilogue's loop
#pragma unroll
                for (int c = 0; c < kPairSpan; c += 16) tmem_st16(from + c, acc + c);
                tmem_wait_st();
            }
#pragma unroll 1
            for (int c = 0; c < kPairSpan; c += 16) {
                float v[16];
                __syncwarp();
                tmem_ld16(from + c, v);
                if (c == kPairSpan - 16) {  // drained: the next part may be multiplied into it
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(acc_empty + ((part - 1) & 1));
                }
                finish(p.e, v, i, col0 + c, p.rows, p.cols, bias);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    cluster_sync();  // neither CTA leaves while the other may still signal it
    if (warp == kPairEpilogue + 1) tmem_free<2>(tmem, 512);
}

}  // namespace quasar
