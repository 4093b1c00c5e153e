// Layer normalisation and its gradients.
//
//   y = (x - mean) rstd w + b,   rstd = (mean((x - mean)^2) + eps)^-1/2
//   (not centered: mean = 0 throughout, the root-mean-square norm)
//
//   xh = (x - mean) rstd,  u = dy w
//   dx = rstd (u - mean(u) - xh mean(u xh)) + residual
//   dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Bound by memory: a row is read once and kept in registers.  T threads share
// a row, NV times 8 elements each; 8 or 32 threads where rows are short (a CTA
// then takes 32 or 8 of them at a time), a whole CTA else.  The backward
// kernel's CTAs are persistent, so that a thread's columns stay the same and dw
// and db accumulate in registers over the CTA's rows.
//
// The variance is summed about the mean: of each warp's elements about their
// own mean, the warps' then joined (M2 = sum M2_w + n_w (mean_w - mean)^2),
// which takes one exchange through shared memory instead of two.
#pragma once

#include "layers.h"
#include "row_access.cuh"

namespace quasar {

template <int T>
constexpr int kNormThreads = T < 128 ? 256 : T;

// CTAs an SM of the kernels whose rows come through shared memory: 512 threads
// have 128 registers each (forward with two vectors a thread: 768).
template <int T, int NV, bool GRAD>
constexpr int kNormRingPerSm = (NV == 2 && !GRAD ? 768 : 512) / T;

// CTAs an SM of the backward kernel, by its registers.
template <int T, int NV>
constexpr int kNormPerSm = (NV == 1 ? 768 : 512) / kNormThreads<T>;  // 512 threads have 128 each

// Sum over the W (at most 32) threads of an aligned part of a warp.
template <int W>
__device__ __forceinline__ float lanes_sum(float x)
{
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// -- forward ---------------------------------------------------------------------

// Several CTAs an SM, no more than a row each in hand, keep the memory busy; the
// weights come from L1.  65536 x 128 bf16, statistics: 12 us, 1.4 TB/s of what L2
// takes and HBM gives, which is mostly the grid's start and end.
template <int T, int NV, bool VECTORS, bool WIDE>
__global__ void __launch_bounds__(kNormThreads<T>, 1024 / kNormThreads<T>) k_layer_norm(const __grid_constant__ NormParams p)
{
    constexpr int kGroups = kNormThreads<T> / T, kWarps = T / 32, kLanes = T < 32 ? T : 32;
    __shared__ float2 red[T > 32 ? kWarps : 1];
    const int t = threadIdx.x % T, lane = threadIdx.x & 31;
    const int n_cols = (int)p.cols;  // (what registers hold)
    const bool whole = n_cols == T * NV * 8;
    const float cols = (float)n_cols;
    const int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / T;
    const bool live = row < p.rows;
    wait_for_previous_grid();

    Raw8<WIDE> raw[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j)
        load_raw<T, VECTORS>(raw[j], row_of(p.x, p.x_f32, row, p.ld_x), p.x_f32, t, j, live ? n_cols : 0);
    float v[NV][8];
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        unpack_raw(raw[j], p.x_f32, v[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[j][i];
    }
    float n = cols;  // this warp's elements (its part of the row)
    if (T > 32) {
        n = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int left = n_cols - row_at<T, VECTORS>(t & ~31, j, 0);
            if (VECTORS)
                n += (float)max(0, min(256, left));
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) n += (float)max(0, min(32, left - i * T));
        }
    }
    // (divisions: a row of one value then has no variance at all)
    float mean = p.center && n > 0.0f ? lanes_sum<kLanes>(sum) / n : 0.0f;
    float m2 = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = whole || row_at<T, VECTORS>(t, j, i) < n_cols ? v[j][i] - mean : 0.0f;
            m2 = fmaf(d, d, m2);
        }
    m2 = lanes_sum<kLanes>(m2);
    if constexpr (T > 32) {
        __shared__ float counts[kWarps];
        if (lane == 0) red[threadIdx.x >> 5] = make_float2(mean, m2), counts[threadIdx.x >> 5] = n;
        __syncthreads();
        const float2 part = lane < kWarps ? red[lane] : make_float2(0.0f, 0.0f);
        n = lane < kWarps ? counts[lane] : 0.0f;
        mean = lanes_sum<kWarps>(n * part.x) / cols;
        const float d = part.x - mean;
        m2 = lanes_sum<kWarps>(fmaf(n * d, d, part.y));
        mean = __shfl_sync(0xffffffffu, mean, 0);  // (of the lanes that hold a warp's part)
        m2 = __shfl_sync(0xffffffffu, m2, 0);
    }
    const float rstd = rsqrtf(m2 / cols + p.eps);
    if (!live) return;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float w[8], b[8];
        load_floats<T, VECTORS>(w, p.weight, t, j, n_cols, 1.0f);
        load_floats<T, VECTORS>(b, p.bias, t, j, n_cols, 0.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = fmaf((v[j][i] - mean) * rstd, w[i], b[i]);
        store_row<T, VECTORS>(row_of(p.y, p.y_f32, row, p.ld_y), p.y_f32, t, j, n_cols, v[j]);
    }
    if (p.stats && t == 0) {
        p.stats[2 * row] = mean;
        p.stats[2 * row + 1] = rstd;
    }
}

// -- rows through shared memory ----------------------------------------------------
//
// Rows of whole 16-byte vectors that start at 16-byte boundaries, longer than
// what a warp takes: persistent CTAs keep their columns' weights in registers
// and bulk copies bring the next rows (up to 8) into a ring.  A slot is free
// once every thread has taken its part, which the reduction's barrier says.
//
// 16384 x 4096 bf16 with weight, bias and statistics: 48 us, 5.6 TB/s, 0.83 of the
// copy rate (weights from L1, a row a CTA: 60 us; rows in registers, fetched one
// ahead by two CTAs of 512 threads an SM: 79 us); with 63% of the issue slots in use
// the warps' two reductions a row are what is left.  The gradient with dw, db and a
// residual: 85 us, 6.3 TB/s, 0.93 of it.

struct NormRing {
    uint8_t* rows;
    uint64_t* full;         // [slots]
    uint64_t* never;
    volatile uint32_t* gone;
    float2* red;            // [2][warps]
    float* counts;          // [warps]
    int slots;
    uint32_t slot_bytes;
};

__host__ __device__ constexpr size_t norm_ring_smem(int slots, uint32_t slot_bytes, int threads)
{
    return (size_t)slots * slot_bytes + (slots + 2) * 8 + threads / 32 * 20;
}

__device__ __forceinline__ NormRing norm_ring(uint8_t* smem, int slots, uint32_t slot_bytes, int warps)
{
    NormRing r;
    r.rows = smem;
    r.full = reinterpret_cast<uint64_t*>(smem + (size_t)slots * slot_bytes);
    r.never = r.full + slots;
    r.gone = reinterpret_cast<volatile uint32_t*>(r.never + 1);
    r.red = reinterpret_cast<float2*>(r.never + 2);
    r.counts = reinterpret_cast<float*>(r.red + 2 * warps);
    r.slots = slots;
    r.slot_bytes = slot_bytes;
    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) mbar_init(r.full + i, 1);
        mbar_init(r.never, 1);
        *r.gone = 0;
        mbar_init_fence();
    }
    __syncthreads();
    return r;
}

// A wait that ran out is said to all behind the next barrier.
__device__ __forceinline__ void norm_wait(const NormRing& r, uint64_t* bar, uint32_t parity, uint64_t limit_ns,
                                          unsigned int* status)
{
    if (!mbar_wait_bounded(bar, parity, limit_ns)) {
        *r.gone = 1;
        record_timeout(status);
    }
}

// Given up: what is in flight of `sent` rows has landed before the memory is
// let go.
__device__ __forceinline__ void norm_drain(const NormRing& r, int64_t sent, uint64_t limit_ns)
{
    for (int64_t k = sent > r.slots ? sent - r.slots : 0; k < sent; ++k)
        mbar_wait_bounded(r.full + k % r.slots, (uint32_t)(k / r.slots) & 1, limit_ns);
}

template <bool WIDE>
__device__ __forceinline__ void from_shared(Raw8<WIDE>& r, const uint8_t* row, bool f32, int c0)
{
#pragma unroll
    for (int q = 0; q < (WIDE ? 8 : 4); ++q) r.w[q] = 0;
    if (WIDE && f32) {
        const uint4 a = *reinterpret_cast<const uint4*>(row + (size_t)c0 * 4);
        const uint4 b = *reinterpret_cast<const uint4*>(row + (size_t)c0 * 4 + 16);
        r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w;
        r.w[WIDE ? 4 : 0] = b.x, r.w[WIDE ? 5 : 0] = b.y, r.w[WIDE ? 6 : 0] = b.z, r.w[WIDE ? 7 : 0] = b.w;
    } else {
        const uint4 a = *reinterpret_cast<const uint4*>(row + (size_t)c0 * 2);
        r.w[0] = a.x, r.w[1] = a.y, r.w[2] = a.z, r.w[3] = a.w;
    }
}

template <int T, int NV, bool WIDE>
__global__ void __launch_bounds__(T, kNormRingPerSm<T, NV, false>) k_layer_norm_ring(const __grid_constant__ NormParams p)
{
    constexpr int kWarps = T / 32;
    extern __shared__ __align__(16) uint8_t smem[];
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const int n_cols = (int)p.cols;  // a multiple of 8 (of 4 in fp32)
    const float cols = (float)n_cols;
    const uint32_t bytes = (uint32_t)n_cols * (p.x_f32 ? 4 : 2);
    const NormRing ring = norm_ring(smem, p.slots, bytes, kWarps);
    float n = 0.0f;  // this warp's elements
#pragma unroll
    for (int j = 0; j < NV; ++j) n += (float)max(0, min(256, n_cols - row_at<T, true>(t & ~31, j, 0)));
    if (lane == 0) ring.counts[warp] = n;
    wait_for_previous_grid();
    int64_t sent = 0;  // rows asked for (thread 0)
    auto fetch = [&](int64_t row, int slot) {
        mbar_arrive_expect_tx(ring.full + slot, bytes);
        bulk_g2s(ring.rows + (size_t)slot * bytes, row_of(p.x, p.x_f32, row, p.ld_x), bytes, ring.full + slot);
        ++sent;
    };
    if (t == 0) {
        if (p.force_timeout_ns) norm_wait(ring, ring.never, 0, p.force_timeout_ns, p.status);
        int64_t row = blockIdx.x;
        for (int s = 0; s < ring.slots && row < p.rows; ++s, row += gridDim.x) fetch(row, s);
    }
    float w[NV][8], b[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        load_floats<T, true>(w[j], p.weight, t, j, n_cols, 1.0f);
        load_floats<T, true>(b[j], p.bias, t, j, n_cols, 0.0f);
    }
    int slot = 0, turn = 0;
    uint32_t parity = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
        norm_wait(ring, ring.full + slot, parity, p.timeout_ns, p.status);
        float v[NV][8];
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c0 = row_at<T, true>(t, j, 0);
            Raw8<WIDE> raw{};
            if (c0 < n_cols) from_shared(raw, ring.rows + (size_t)slot * bytes, p.x_f32, c0);
            unpack_raw(raw, p.x_f32, v[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += v[j][i];
        }
        float mean = p.center && n > 0.0f ? lanes_sum<32>(sum) / n : 0.0f;
        float m2 = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const bool in = row_at<T, true>(t, j, 0) < n_cols;  // (whole runs of 8)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = in ? v[j][i] - mean : 0.0f;
                m2 = fmaf(d, d, m2);
            }
        }
        m2 = lanes_sum<32>(m2);
        if (lane == 0) ring.red[turn * kWarps + warp] = make_float2(mean, m2);
        __syncthreads();
        if (*ring.gone) break;
        if (t == 0 && row + (int64_t)ring.slots * gridDim.x < p.rows) fetch(row + (int64_t)ring.slots * gridDim.x, slot);
        const float2 part = lane < kWarps ? ring.red[turn * kWarps + lane] : make_float2(0.0f, 0.0f);
        const float k = lane < kWarps ? ring.counts[lane] : 0.0f;
        mean = lanes_sum<32>(k * part.x) / cols;
        const float d = part.x - mean;
        m2 = lanes_sum<32>(fmaf(k * d, d, part.y));
        const float rstd = rsqrtf(m2 / cols + p.eps);
        void* y = row_of(p.y, p.y_f32, row, p.ld_y);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = fmaf((v[j][i] - mean) * rstd, w[j][i], b[j][i]);
            store_row<T, true>(y, p.y_f32, t, j, n_cols, v[j]);
        }
        if (p.stats && t == 0) {
            p.stats[2 * row] = mean;
            p.stats[2 * row + 1] = rstd;
        }
        if (++slot == ring.slots) slot = 0, parity ^= 1;
    }
    if (*ring.gone && t == 0) norm_drain(ring, sent, p.timeout_ns);
}

// Sum over the CTA (512 threads), the same value in every thread.
__device__ __forceinline__ float cta_sum(float x, float* red)
{
    x = lanes_sum<32>(x);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
    __syncthreads();
    return lanes_sum<32>((threadIdx.x & 31) < 16 ? red[threadIdx.x & 31] : 0.0f);
}

__device__ __forceinline__ float element(const void* row, bool f32, int64_t c)
{
    return f32 ? static_cast<const float*>(row)[c] : __bfloat162float(static_cast<const __nv_bfloat16*>(row)[c]);
}

__device__ __forceinline__ void put_element(void* row, bool f32, int64_t c, float v)
{
    if (f32)
        static_cast<float*>(row)[c] = v;
    else
        static_cast<__nv_bfloat16*>(row)[c] = __float2bfloat16_rn(v);
}

// Rows that registers do not hold: read once for the mean, once for the
// variance and once for y (from L2, where they fit it).
__global__ void __launch_bounds__(512) k_layer_norm_long(const __grid_constant__ NormParams p)
{
    __shared__ float red[16];
    wait_for_previous_grid();
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const void* x = row_of(p.x, p.x_f32, row, p.ld_x);
        const float cols = (float)p.cols;
        float mean = 0.0f;
        if (p.center) {
            float s = 0.0f;
#pragma unroll 4
            for (int64_t c = threadIdx.x; c < p.cols; c += 512) s += element(x, p.x_f32, c);
            mean = cta_sum(s, red) / cols;
        }
        float s = 0.0f;
#pragma unroll 4
        for (int64_t c = threadIdx.x; c < p.cols; c += 512) {
            const float d = element(x, p.x_f32, c) - mean;
            s = fmaf(d, d, s);
        }
        const float rstd = rsqrtf(cta_sum(s, red) / cols + p.eps);
        void* y = row_of(p.y, p.y_f32, row, p.ld_y);
#pragma unroll 4
        for (int64_t c = threadIdx.x; c < p.cols; c += 512)
            put_element(y, p.y_f32, c,
                        fmaf((element(x, p.x_f32, c) - mean) * rstd, p.weight ? p.weight[c] : 1.0f,
                             p.bias ? p.bias[c] : 0.0f));
        if (p.stats && threadIdx.x == 0) {
            p.stats[2 * row] = mean;
            p.stats[2 * row + 1] = rstd;
        }
    }
}

// -- backward --------------------------------------------------------------------

// A row's elements stay as they lie in memory between the two passes over
// them; dw and db take the registers.
template <int T, int NV, bool VECTORS, bool WIDE>
__global__ void __launch_bounds__(kNormThreads<T>, kNormPerSm<T, NV>)
    k_layer_norm_grad(const __grid_constant__ NormGradParams p)
{
    constexpr int kGroups = kNormThreads<T> / T, kWarps = T / 32, kLanes = T < 32 ? T : 32;
    __shared__ float2 red[2][T > 32 ? kWarps : 1];
    __shared__ float sums[kGroups > 1 ? kGroups * T * NV * 8 : 1];
    const int t = threadIdx.x % T, lane = threadIdx.x & 31;
    const int n_cols = (int)p.cols;
    const float per = 1.0f / (float)n_cols;
    wait_for_previous_grid();

    float dw[NV][8], db[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = db[j][i] = 0.0f;
    const int64_t step = (int64_t)gridDim.x * kGroups;
    int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / T;
    int turn = 0;
    for (int64_t first = (int64_t)blockIdx.x * kGroups; first < p.rows; first += step, row += step, turn ^= 1) {
        const bool live = row < p.rows;
        Raw8<WIDE> raw_x[NV], raw_dy[NV], raw_res[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            load_raw<T, VECTORS>(raw_x[j], row_of(p.x, p.x_f32, row, p.ld_x), p.x_f32, t, j, live ? n_cols : 0);
            load_raw<T, VECTORS>(raw_dy[j], row_of(p.dy, p.dy_f32, row, p.ld_dy), p.dy_f32, t, j, live ? n_cols : 0);
            if (p.residual)
                load_raw<T, VECTORS>(raw_res[j], row_of(p.residual, p.dx_f32, row, p.ld_res), p.dx_f32, t, j,
                                     live ? n_cols : 0);
        }
        const float mean = live && p.center ? p.stats[2 * row] : 0.0f, rstd = live ? p.stats[2 * row + 1] : 0.0f;
        float su = 0.0f, sux = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float x[8], u[8], w[8];
            unpack_raw(raw_x[j], p.x_f32, x);
            unpack_raw(raw_dy[j], p.dy_f32, u);
            load_floats<T, VECTORS>(w, p.weight, t, j, n_cols, 1.0f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // (beyond the row dy is 0, which keeps x's part out of every sum)
                const float xh = (x[i] - mean) * rstd;
                dw[j][i] = fmaf(u[i], xh, dw[j][i]);
                db[j][i] += u[i];
                u[i] *= w[i];
                su += u[i];
                sux = fmaf(u[i], xh, sux);
            }
        }
        if (!p.dx) continue;
        su = lanes_sum<kLanes>(su);
        sux = lanes_sum<kLanes>(sux);
        if constexpr (T > 32) {
            if (lane == 0) red[turn][threadIdx.x >> 5] = make_float2(su, sux);
            __syncthreads();
            const float2 part = lane < kWarps ? red[turn][lane] : make_float2(0.0f, 0.0f);
            su = lanes_sum<32>(part.x);
            sux = lanes_sum<32>(part.y);
        }
        const float mu = p.center ? su * per : 0.0f, mux = sux * per;
        if (live) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float x[8], u[8], w[8], res[8];
                unpack_raw(raw_x[j], p.x_f32, x);
                unpack_raw(raw_dy[j], p.dy_f32, u);
                load_floats<T, VECTORS>(w, p.weight, t, j, n_cols, 1.0f);
                if (p.residual) {
                    unpack_raw(raw_res[j], p.dx_f32, res);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) res[i] = 0.0f;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    u[i] = fmaf(fmaf(-(x[i] - mean) * rstd, mux, fmaf(u[i], w[i], -mu)), rstd, res[i]);
                store_row<T, VECTORS>(row_of(p.dx, p.dx_f32, row, p.ld_dx), p.dx_f32, t, j, n_cols, u);
            }
        }
    }
    // this CTA's share of dw and db
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* part = which ? p.part_b : p.part_w;
        if (!part) continue;
        float(&mine)[NV][8] = which ? db : dw;
        part += (int64_t)blockIdx.x * p.cols;
        if constexpr (kGroups > 1) {
            constexpr int kSpan = T * NV * 8;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    sums[threadIdx.x / T * kSpan + row_at<T, VECTORS>(t, j, i)] = mine[j][i];
            __syncthreads();
            for (int c = threadIdx.x; c < n_cols; c += kNormThreads<T>) {
                float s = sums[c];
#pragma unroll 8
                for (int g = 1; g < kGroups; ++g) s += sums[g * kSpan + c];
                part[c] = s;
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = row_at<T, VECTORS>(t, j, i);
                    if (c < n_cols) part[c] = mine[j][i];
                }
        }
    }
}

template <int T, int NV, bool WIDE>
__global__ void __launch_bounds__(T, kNormRingPerSm<T, NV, true>)
    k_layer_norm_grad_ring(const __grid_constant__ NormGradParams p)
{
    constexpr int kWarps = T / 32;
    extern __shared__ __align__(16) uint8_t smem[];
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const int n_cols = (int)p.cols;
    const float per = 1.0f / (float)n_cols;
    // a slot: the rows of x, dy and the residual
    const uint32_t x_bytes = (uint32_t)n_cols * (p.x_f32 ? 4 : 2), dy_bytes = (uint32_t)n_cols * (p.dy_f32 ? 4 : 2);
    const uint32_t res_bytes = p.residual ? (uint32_t)n_cols * (p.dx_f32 ? 4 : 2) : 0;
    const uint32_t slot_bytes = x_bytes + dy_bytes + res_bytes;
    const NormRing ring = norm_ring(smem, p.slots, slot_bytes, kWarps);
    wait_for_previous_grid();
    int64_t sent = 0;
    auto fetch = [&](int64_t row, int slot) {
        uint8_t* to = ring.rows + (size_t)slot * slot_bytes;
        mbar_arrive_expect_tx(ring.full + slot, slot_bytes);
        bulk_g2s(to, row_of(p.x, p.x_f32, row, p.ld_x), x_bytes, ring.full + slot);
        bulk_g2s(to + x_bytes, row_of(p.dy, p.dy_f32, row, p.ld_dy), dy_bytes, ring.full + slot);
        if (res_bytes)
            bulk_g2s(to + x_bytes + dy_bytes, row_of(p.residual, p.dx_f32, row, p.ld_res), res_bytes, ring.full + slot);
        ++sent;
    };
    if (t == 0) {
        if (p.force_timeout_ns) norm_wait(ring, ring.never, 0, p.force_timeout_ns, p.status);
        int64_t row = blockIdx.x;
        for (int s = 0; s < ring.slots && row < p.rows; ++s, row += gridDim.x) fetch(row, s);
    }
    float w[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        load_floats<T, true>(w[j], p.weight, t, j, n_cols, 1.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = db[j][i] = 0.0f;
    }
    auto stats_of = [&](int64_t row) {
        if (row >= p.rows) return make_float2(0.0f, 0.0f);
        return make_float2(p.center ? p.stats[2 * row] : 0.0f, p.stats[2 * row + 1]);
    };
    float2 next = stats_of(blockIdx.x);
    int slot = 0, turn = 0;
    uint32_t parity = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, turn ^= 1) {
        const float mean = next.x, rstd = next.y;
        next = stats_of(row + gridDim.x);
        norm_wait(ring, ring.full + slot, parity, p.timeout_ns, p.status);
        const uint8_t* at = ring.rows + (size_t)slot * slot_bytes;
        float xh[NV][8], u[NV][8];
        Raw8<WIDE> res[NV];
        float su = 0.0f, sux = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c0 = row_at<T, true>(t, j, 0);
            Raw8<WIDE> x{}, dy{};
            res[j] = Raw8<WIDE>{};
            if (c0 < n_cols) {
                from_shared(x, at, p.x_f32, c0);
                from_shared(dy, at + x_bytes, p.dy_f32, c0);
                if (res_bytes) from_shared(res[j], at + x_bytes + dy_bytes, p.dx_f32, c0);
            }
            unpack_raw(x, p.x_f32, xh[j]);
            unpack_raw(dy, p.dy_f32, u[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // (beyond the row dy is 0, which keeps x's part out of every sum)
                xh[j][i] = (xh[j][i] - mean) * rstd;
                dw[j][i] = fmaf(u[j][i], xh[j][i], dw[j][i]);
                db[j][i] += u[j][i];
                u[j][i] *= w[j][i];
                su += u[j][i];
                sux = fmaf(u[j][i], xh[j][i], sux);
            }
        }
        su = lanes_sum<32>(su);
        sux = lanes_sum<32>(sux);
        if (lane == 0) ring.red[turn * kWarps + warp] = make_float2(su, sux);
        __syncthreads();  // (every thread has its part of the row: dx may take its place)
        if (*ring.gone) break;
        if (t == 0 && row + (int64_t)ring.slots * gridDim.x < p.rows) fetch(row + (int64_t)ring.slots * gridDim.x, slot);
        if (p.dx) {
            const float2 part = lane < kWarps ? ring.red[turn * kWarps + lane] : make_float2(0.0f, 0.0f);
            const float mu = p.center ? lanes_sum<32>(part.x) * per : 0.0f, mux = lanes_sum<32>(part.y) * per;
            void* dx = row_of(p.dx, p.dx_f32, row, p.ld_dx);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float r[8];
                unpack_raw(res[j], p.dx_f32, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) u[j][i] = fmaf(fmaf(-xh[j][i], mux, u[j][i] - mu), rstd, r[i]);
                store_row<T, true>(dx, p.dx_f32, t, j, n_cols, u[j]);
            }
        }
        if (++slot == ring.slots) slot = 0, parity ^= 1;
    }
    if (*ring.gone) {
        if (t == 0) norm_drain(ring, sent, p.timeout_ns);
        return;
    }
    // (of one row they are the caller's dweight and dbias, which start at any float)
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* part = which ? p.part_b : p.part_w;
        if (!part) continue;
        float(&mine)[NV][8] = which ? db : dw;
        const bool vectors = (reinterpret_cast<uintptr_t>(part) & 15) == 0;
        part += (int64_t)blockIdx.x * p.cols;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (vectors) {
                store_row<T, true>(part, true, t, j, n_cols, mine[j]);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int c = row_at<T, true>(t, j, i);
                    if (c < n_cols) part[c] = mine[j][i];
                }
            }
        }
    }
}

// dx of rows that registers do not hold.
__global__ void __launch_bounds__(512) k_layer_norm_grad_long(const __grid_constant__ NormGradParams p)
{
    __shared__ float red[16];
    wait_for_previous_grid();
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const void* x = row_of(p.x, p.x_f32, row, p.ld_x);
        const void* dy = row_of(p.dy, p.dy_f32, row, p.ld_dy);
        const float mean = p.center ? p.stats[2 * row] : 0.0f, rstd = p.stats[2 * row + 1];
        const float per = 1.0f / (float)p.cols;
        float su = 0.0f, sux = 0.0f;
#pragma unroll 4
        for (int64_t c = threadIdx.x; c < p.cols; c += 512) {
            const float u = element(dy, p.dy_f32, c) * (p.weight ? p.weight[c] : 1.0f);
            su += u;
            sux = fmaf(u, (element(x, p.x_f32, c) - mean) * rstd, sux);
        }
        const float mu = p.center ? cta_sum(su, red) * per : 0.0f, mux = cta_sum(sux, red) * per;
        void* dx = row_of(p.dx, p.dx_f32, row, p.ld_dx);
#pragma unroll 4
        for (int64_t c = threadIdx.x; c < p.cols; c += 512) {
            const float u = element(dy, p.dy_f32, c) * (p.weight ? p.weight[c] : 1.0f);
            const float xh = (element(x, p.x_f32, c) - mean) * rstd;
            const float res = p.residual ? element(row_of(p.residual, p.dx_f32, row, p.ld_res), p.dx_f32, c) : 0.0f;
            put_element(dx, p.dx_f32, c, fmaf(fmaf(-xh, mux, u - mu), rstd, res));
        }
    }
}

// dw and db of such rows: a column a thread, a share of the rows a CTA.
__global__ void __launch_bounds__(256) k_layer_norm_grad_columns(const __grid_constant__ NormGradParams p)
{
    wait_for_previous_grid();
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= p.cols) return;
    float dw = 0.0f, db = 0.0f;
#pragma unroll 4
    for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const float d = element(row_of(p.dy, p.dy_f32, row, p.ld_dy), p.dy_f32, c);
        const float mean = p.center ? p.stats[2 * row] : 0.0f;
        dw = fmaf(d, (element(row_of(p.x, p.x_f32, row, p.ld_x), p.x_f32, c) - mean) * p.stats[2 * row + 1], dw);
        db += d;
    }
    if (p.part_w) p.part_w[(int64_t)blockIdx.y * p.cols + c] = dw;
    if (p.part_b) p.part_b[(int64_t)blockIdx.y * p.cols + c] = db;
}

// The CTAs' shares added up, always in the same order: 32 columns a CTA, the
// parts over its 32 warps (with 8 warps 304 parts of 4096 columns took 10 us).
__global__ void __launch_bounds__(1024) k_part_sum(const __grid_constant__ PartSumParams p)
{
    __shared__ float red[32][33];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    wait_for_previous_grid();
    const float* part = p.part[blockIdx.y];
    float s = 0.0f;
    if (c < p.cols) {
#pragma unroll 8
        for (int q = warp; q < p.parts; q += 32) s += part[q * p.cols + c];
    }
    red[warp][lane] = s;
    __syncthreads();
    // column `warp`, its 32 sums in a tree
    s = lanes_sum<32>(red[lane][warp]);
    if (lane == 0 && (int64_t)blockIdx.x * 32 + warp < p.cols) p.out[blockIdx.y][(int64_t)blockIdx.x * 32 + warp] = s;
}

}  // namespace quasar
