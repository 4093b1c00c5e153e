// A row's k largest logits, in order, with their indices, and the row's
// log-sum-exp: what a teacher hands to the distillation.
//
// Elements are compared as 64-bit keys: the value's bits, reordered so that
// unsigned comparison follows the floats', above the complement of the index,
// so that equal values rank by the lowest index and no two keys are equal.
//
// Each CTA of a row's cluster finds the k largest of its slice.  A bound on
// the k-th comes from the threads' own maxima: the k-th largest of the 512
// maxima has at least k elements at or above it, and not many more unless
// the row is made of ties.  The elements at or above the bound are gathered
// and ranked by counting.  A slice with more of them than the list holds is
// settled by bisection on the 64-bit keys, which is exact for any data.  The
// slices' lists, sorted, are merged by rank 0: an entry's rank is its place
// in its own list plus, by binary search, the entries above it in the others.
#pragma once

#include "distill.cuh"

namespace quasar {

constexpr int kTopThreads = 512;
constexpr int kTopList = 1024;  // elements a slice may gather before bisection

// Both zeros are one value, and NaN ranks above everything.
__device__ __forceinline__ uint32_t ordered_bits(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return x != x ? 0xFFFFFFFFu : (b & 0x80000000u ? ~b : b | 0x80000000u);
}

__device__ __forceinline__ float from_ordered(uint32_t o)
{
    return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}

__device__ __forceinline__ uint64_t top_key(float x, int64_t e)
{
    return ((uint64_t)ordered_bits(x) << 32) | (uint32_t)~(uint32_t)e;
}

template <typename T>
__global__ void __launch_bounds__(kTopThreads) k_top_logits(const __grid_constant__ TopParams p)
{
    using V = Vec16<T>;
    constexpr int kN = V::kN;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    T* slice = reinterpret_cast<T*>(smem_raw);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem_raw + (size_t)p.row.vecs * 16);
    uint64_t* never = bars + kRowChunks;
    uint64_t* list = never + 1;                        // [kTopList]
    uint64_t* merged = list + kTopList;                // rank 0: [kRowCtas][k]
    float(*parts)[2] = reinterpret_cast<float(*)[2]>(merged + (size_t)kRowCtas * p.k);
    float* scratch = reinterpret_cast<float*>(parts + kRowCtas);
    int* count = reinterpret_cast<int*>(scratch + 32);

    const int t = threadIdx.x;
    const int rank = (int)(blockIdx.x % p.row.ctas);
    const int64_t r = blockIdx.x / p.row.ctas;
    const RowSlice<T> S(p.row, r, rank);
    if (t == 0) {
        for (int c = 0; c < kRowChunks; ++c) mbar_init(bars + c, 1);
        mbar_init(never, 1);
        mbar_init_fence();
        *count = 0;
    }
    cluster_arrive();
    __syncthreads();
    S.load(slice, bars);
    if (t == 0 && p.row.force_timeout_ns && !mbar_wait_bounded(never, 0, p.row.force_timeout_ns))
        record_timeout(p.row.status);
    for (int c = 0; c < kRowChunks; ++c)
        if (!mbar_wait_bounded(bars + c, 0, p.row.timeout_ns)) record_timeout(p.row.status);
    __syncthreads();
    cluster_wait();  // every CTA of the row has started: its shared memory may be written

    // maximum and sum of this thread's elements, and its largest element
    const float c2 = kLog2e / p.temperature;
    float m = neg_inf(), s = 0.0f;
    bool any = false;
    for (int v = t; v < S.n_vecs; v += kTopThreads) {
        float x[kN];
        V::unpack(reinterpret_cast<const uint4*>(slice)[v], x);
        float top = x[0];
#pragma unroll
        for (int j = 1; j < kN; ++j) top = fmaxf(top, x[j]);
        if (top > m) {
            s *= ex2((m - top) * c2);
            m = top;
        }
        const float base = m == neg_inf() ? 0.0f : m;
#pragma unroll
        for (int j = 0; j < kN; ++j) s += ex2((x[j] - base) * c2);
        any = true;
    }
    if (p.lse) {
        const float top = block_max(m, scratch);
        const float sum = block_sum(top == neg_inf() ? s : s * ex2((m - top) * c2), scratch);
        if (t == 0) {
            const uint32_t to = peer_addr(smem_u32(&parts[rank][0]), 0);
            st_peer(to, top);
            st_peer(to + 4, sum);
        }
    }
    // this thread's largest element (or less): a NaN leaves its mark in the sum
    uint32_t best = 0;
    if (any) best = s != s && m != __int_as_float(0x7F800000) ? 0xFFFFFFFFu : ordered_bits(m);

    const int have = (int)(S.end - S.begin);
    const int want = have < p.k ? have : p.k;
    // the want-th largest of the threads' maxima, bit by bit
    uint32_t bound = 0;
    if (have > kTopThreads)
        for (int b = 31; b >= 0; --b) {
            const uint32_t trial = bound | (1u << b);
            if (__syncthreads_count(best >= trial) >= want) bound = trial;
        }
    for (int v = t; v < S.n_vecs; v += kTopThreads) {
        float x[kN];
        V::unpack(reinterpret_cast<const uint4*>(slice)[v], x);
        const int64_t at = S.first + (int64_t)v * kN;
#pragma unroll
        for (int j = 0; j < kN; ++j)
            if (ordered_bits(x[j]) >= bound && at + j >= S.begin && at + j < S.end) {
                const int n = atomicAdd(count, 1);
                if (n < kTopList) list[n] = top_key(x[j], at + j - S.lead);
            }
    }
    __syncthreads();
    int n = *count;
    if (n > kTopList) {
        // exact: the want-th largest key, and the keys from it up
        uint64_t floor_key = 0;
        for (int b = 63; b >= 0; --b) {
            const uint64_t trial = floor_key | (1ull << b);
            int c = 0;
            for (int v = t; v < S.n_vecs; v += kTopThreads) {
                float x[kN];
                V::unpack(reinterpret_cast<const uint4*>(slice)[v], x);
                const int64_t at = S.first + (int64_t)v * kN;
#pragma unroll
                for (int j = 0; j < kN; ++j)
                    c += at + j >= S.begin && at + j < S.end && top_key(x[j], at + j - S.lead) >= trial;
            }
            c = __reduce_add_sync(0xffffffffu, c);
            __syncthreads();
            if (t == 0) *count = 0;
            __syncthreads();
            if ((t & 31) == 0) atomicAdd(count, c);
            __syncthreads();
            if (*count >= want) floor_key = trial;
        }
        __syncthreads();
        if (t == 0) *count = 0;
        __syncthreads();
        for (int v = t; v < S.n_vecs; v += kTopThreads) {
            float x[kN];
            V::unpack(reinterpret_cast<const uint4*>(slice)[v], x);
            const int64_t at = S.first + (int64_t)v * kN;
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                const uint64_t key = top_key(x[j], at + j - S.lead);
                if (at + j >= S.begin && at + j < S.end && key >= floor_key) {
                    const int i = atomicAdd(count, 1);
                    if (i < kTopList) list[i] = key;
                }
            }
        }
        __syncthreads();
        n = *count < kTopList ? *count : kTopList;
    }
    // sorted into rank 0's row of the merge: the place is the number above
    const uint32_t to = peer_addr(smem_u32(merged + (size_t)rank * p.k), 0);
    for (int i = t; i < n; i += kTopThreads) {
        const uint64_t key = list[i];
        int above = 0;
        for (int j = 0; j < n; ++j) above += list[j] > key;
        if (above < p.k) st_peer(to + (uint32_t)above * 8, key);
    }
    for (int i = n + t; i < p.k; i += kTopThreads) st_peer(to + (uint32_t)i * 8, (uint64_t)0);
    cluster_sync();
    if (rank != 0) return;

    for (int i = t; i < p.row.ctas * p.k; i += kTopThreads) {
        const int c = i / p.k;
        const uint64_t key = merged[i];
        if (key == 0) continue;
        int place = i - c * p.k;
        for (int o = 0; o < p.row.ctas && place < p.k; ++o) {
            if (o == c) continue;
            const uint64_t* other = merged + (size_t)o * p.k;
            int lo = 0, hi = p.k;  // other[lo - 1] > key >= other[hi]
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (other[mid] > key)
                    lo = mid + 1;
                else
                    hi = mid;
            }
            place += lo;
        }
        if (place < p.k) {
            p.values[r * p.k + place] = from_ordered((uint32_t)(key >> 32));
            p.indices[r * p.k + place] = (int32_t)~(uint32_t)key;
        }
    }
    if (p.lse && t == 0) {
        float top = neg_inf(), sum = 0.0f;
        for (int c = 0; c < p.row.ctas; ++c) merge_sum(top, sum, parts[c][0], parts[c][1], c2);
        p.lse[r] = sum > 0.0f || sum != sum ? top / p.temperature + logf(sum) : neg_inf();
    }
}

}  // namespace quasar
