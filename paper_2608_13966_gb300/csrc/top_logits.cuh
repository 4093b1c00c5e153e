// A row's k largest logits, in order, with their indices, and the row's
// log-sum-exp: what a teacher hands to the distillation.
//
// Elements are compared as 64-bit keys: the value's bits, reordered so that
// unsigned comparison follows the floats', above the complement of the index,
// so that equal values rank by the lowest index and no two keys are equal.
//
// Each CTA of a row's cluster finds the k largest of its slice.  A bound on
// the k-th comes from the threads' own maxima: the k-th largest of them (in
// 16 bits, rounded down) has at least k elements at or above it, and not many
// more unless the row is made of ties.  One warp settles the bound; then, in
// the pass that sums the exponentials, each 16-byte vector's maximum is
// compared with it, and the few vectors that reach it are looked into
// afterwards, an element a thread.  The elements found are ranked by counting.
// A slice with more of them than the lists hold is settled by bisection on
// the 64-bit keys, which is exact for any data.  The slices' lists, sorted,
// are merged by rank 0: an entry's rank is its place in its own list plus, by
// binary search, the entries above it in the others.
#pragma once

#include "distill.cuh"

namespace quasar {

constexpr int kTopThreads = 512;
constexpr int kTopList = 512;  // vectors or elements a slice may gather before bisection
constexpr int kTopBounds = kTopThreads;  // maxima the bound is taken from

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

// The want-th largest of the kTopBounds 16-bit maxima (0 if there are fewer),
// by one warp, a bit a step.
__device__ __forceinline__ uint32_t kth_largest(const uint16_t* maxima, int want)
{
    constexpr int kEach = kTopBounds / 32;
    const int lane = threadIdx.x & 31;
    uint32_t key[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) key[i] = maxima[32 * i + lane];
    // the bits above the highest in which any two differ are settled already
    uint32_t high = key[0], low = key[0];
#pragma unroll
    for (int i = 1; i < kEach; ++i) {
        high = max(high, key[i]);
        low = min(low, key[i]);
    }
    high = __reduce_max_sync(0xffffffffu, high);
    low = __reduce_min_sync(0xffffffffu, low);
    int b = 31 - __clz(high ^ low);
    uint32_t bound = high >> (b + 1) << (b + 1);
#pragma unroll 1
    for (; b >= 0; --b) {
        const uint32_t trial = bound | (1u << b);
        int c = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) c += key[i] >= trial;
        if (__reduce_add_sync(0xffffffffu, c) >= want) bound = trial;
    }
    return bound;
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
    uint64_t* merged = list + kTopList;                // rank 0: [ctas][k]
    float(*parts)[2] = reinterpret_cast<float(*)[2]>(merged + (size_t)p.row.ctas * p.k);
    float* scratch = reinterpret_cast<float*>(parts + kRowCtas);      // [2][warps]
    uint16_t* maxima = reinterpret_cast<uint16_t*>(scratch + 32);     // [kTopBounds]
    uint16_t* found = maxima + kTopBounds;                            // [kTopList] vectors
    int* count = reinterpret_cast<int*>(found + kTopList);  // elements, vectors
    uint32_t* shared_bound = reinterpret_cast<uint32_t*>(count + 2);

    const int t = threadIdx.x;
    const int rank = (int)(blockIdx.x % p.row.ctas);
    const int64_t r = blockIdx.x / p.row.ctas;
    const RowSlice<T> S(p.row, r, rank);
    cluster_arrive();
    wait_for_previous_grid();
    if (t == 0) count[0] = count[1] = 0;
    S.load(slice, bars, never);
    __syncthreads();
    if (t == 0 && p.row.force_timeout_ns && !mbar_wait_bounded(never, 0, p.row.force_timeout_ns))
        record_timeout(p.row.status);

    const float c2 = kLog2e / p.temperature;
    const uint4* vecs = reinterpret_cast<const uint4*>(slice);
    const int warp = t >> 5, lane = t & 31;
    const int have = S.end - S.begin;
    const int want = have < p.k ? have : p.k;
    const float mine = S.largest(slice, bars, p.row);
    cluster_wait();  // every CTA of the row has started: its shared memory may be written
    // 0 where a thread held nothing: it must not count towards the bound
    maxima[t] = (uint16_t)(S.holds(t) ? ordered_bits(mine) >> 16 : 0);
    const float m = block_max(mine, scratch);
    // one warp settles the bound while the others sum the exponentials
    if (warp == 0) {
        const uint32_t b = kth_largest(maxima, want) << 16;
        if (lane == 0) *shared_bound = b;
    } else if (p.lse) {
        const ExpBase at(m, c2);
        const float s = warp_sum(sum_exponentials(slice, S.n_vecs, t - 32, kTopThreads - 32, c2, at)) * at.fix;
        if (lane == 0) scratch[16 + warp] = s;
    }
    __syncthreads();
    if (p.lse && warp == 1) {
        const float sum = warp_sum(lane > 0 && lane < kTopThreads / 32 ? scratch[16 + lane] : 0.0f);
        if (lane == 0) {
            const uint32_t to = peer_addr(smem_u32(&parts[rank][0]), 0);
            st_peer(to, m);
            st_peer(to + 4, sum);
        }
    }
    // the vectors that hold an element at or above the bound (a NaN compares
    // as if it did)
    const uint32_t bound = *shared_bound;
    const float least = from_ordered(bound);
#pragma unroll 4
    for (int v = t; v < S.n_vecs; v += kTopThreads)
        if (!(V::value(V::larger(vecs[v])) < least)) {
            const int i = atomicAdd(count + 1, 1);
            if (i < kTopList) found[i] = (uint16_t)v;
        }
    __syncthreads();
    // an element a thread of the vectors found
    const int n_found = count[1];
    for (int i = t; i < min(n_found, kTopList) * kN; i += kTopThreads) {
        const int at_slot = found[i / kN] * kN + i % kN;
        const float x = V::to_f32(slice[at_slot]);
        if (ordered_bits(x) >= bound && at_slot >= S.begin && at_slot < S.end) {
            const int j = atomicAdd(count, 1);
            if (j < kTopList) list[j] = top_key(x, S.element0 + at_slot);
        }
    }
    __syncthreads();
    int n = n_found > kTopList ? kTopList + 1 : *count;
    if (n > kTopList) {
        // exact: the want-th largest key, and the keys from it up
        uint64_t floor_key = 0;
        for (int b = 63; b >= 0; --b) {
            const uint64_t trial = floor_key | (1ull << b);
            int c = 0;
            for (int i = t; i < have; i += kTopThreads)
                c += top_key(V::to_f32(slice[S.begin + i]), S.element0 + S.begin + i) >= trial;
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
        for (int i = t; i < have; i += kTopThreads) {
            const uint64_t key = top_key(V::to_f32(slice[S.begin + i]), S.element0 + S.begin + i);
            if (key >= floor_key) {
                const int j = atomicAdd(count, 1);
                if (j < kTopList) list[j] = key;
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
        p.lse[r] = top == neg_inf() && sum == 0.0f ? neg_inf() : top / p.temperature + logf(sum);
    }
}

}  // namespace quasar
