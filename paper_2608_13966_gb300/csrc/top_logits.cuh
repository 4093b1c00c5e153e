// A row's k largest logits, in order, with their indices, and the row's
// log-sum-exp: what a teacher hands to the distillation.
//
// Elements are compared as 64-bit keys: the value's bits, reordered so that
// unsigned comparison follows the floats', above the complement of the index,
// so that equal values rank by the lowest index and no two keys are equal.
//
// A row is read once.  The threads' maxima over the first vectors they hold (8
// each; in fours where an eighth of the threads is k or more) bound the k-th
// largest: the k-th largest of those maxima (a CTA has k threads or more), in
// 16 bits rounded down, has at least k elements at or above it.  A vector of the rest is put aside only if
// its maximum reaches the bound; with 131,072 bf16 logits, k = 64 and values
// in no particular order that is about 350 of 16,384 vectors.  Over a long row
// the bound is renewed, each time the part read has doubled, from the maxima
// of what lies aside.  In the end the elements at or above the bound are
// gathered, a second bound among them (a bit a step) leaves little more than
// k, and those are ranked by counting.  A row that puts aside more than the
// lists hold (rising order, ties, fewer than k that are not -inf) is settled
// by bisection on the k-th value, which is exact for any data and reads the
// row once more for each bit.  Where a cluster shares a row, its lists,
// sorted, are merged by rank 0: an entry's rank is its place in its own list
// plus, by binary search, the entries above it in the others.
//
// Bound by instructions, some 11 an element at 2.6 a cycle: the top 64 of 2048
// x 131072 bf16 rows with their log-sum-exps take 125 us, 4.3 TB/s.  The 256 of
// 4096 x 8184 take 186 us, the 128 (128 threads a CTA) 122.  A row that is
// settled by bisection is what its call waits for: 2048 x 131072 fp32 rows of
// normal values take 209 us, and 755 in the batches, about every second, where
// one or two of them put more aside than the lists hold.
#pragma once

#include "row_stream.cuh"

namespace quasar {

constexpr int kTopVectors = 1024;  // vectors a share may put aside before bisection
constexpr int kTopKeys = 2048;     // elements of them at or above the bound
constexpr int kTopShort = 512;     // ... that one warp finds the second bound of

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

// The largest 16-bit value that at least `want` of 32 EACH values reach (the
// want-th largest), by one warp, a bit a step from the highest in which the
// largest differs from `low`: a value that many are known to reach, or 0 (then
// from the smallest present, which takes want <= 32 EACH).
template <int EACH>
__device__ __forceinline__ uint32_t kth_largest(const uint16_t* values, int want, uint32_t low)
{
    const int lane = threadIdx.x & 31;
    uint32_t key[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) key[i] = values[32 * i + lane];
    uint32_t high = key[0], least = key[0];
#pragma unroll
    for (int i = 1; i < EACH; ++i) {
        high = max(high, key[i]);
        least = min(least, key[i]);
    }
    high = __reduce_max_sync(0xffffffffu, high);
    low = max(low, __reduce_min_sync(0xffffffffu, least));
    int b = 31 - __clz(high ^ low);
    uint32_t bound = high >> (b + 1) << (b + 1);
#pragma unroll 1
    for (; b >= 0; --b) {
        const uint32_t trial = bound | (1u << b);
        int c[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < EACH; ++i) c[i & 3] += key[i] >= trial;
        if (__reduce_add_sync(0xffffffffu, (c[0] + c[1]) + (c[2] + c[3])) >= want) bound = trial;
    }
    return bound;
}

// The same of n values, get(i) each, by the whole CTA: for the longer lists.
template <int THREADS, typename Get>
__device__ __noinline__ uint32_t block_kth_largest(int n, int want, uint32_t low, Get get)
{
    uint32_t bound = 0;
    for (int b = 15; b >= 0; --b) {
        const uint32_t trial = bound | (1u << b);
        int c = want;
        if (trial > low) {
            c = 0;
            for (int i = threadIdx.x; i < (n + THREADS - 1) / THREADS * THREADS; i += THREADS)
                c += __syncthreads_count(i < n && get(i) >= trial);
        }
        if (c >= want) bound = trial;
    }
    return max(bound, low);
}

// A place in a list for each lane with `want`, one atomic a warp; the lanes
// of the warp that call it do so together.
__device__ __forceinline__ int take_place(int* count, bool want)
{
    const unsigned active = __activemask();
    const unsigned who = __ballot_sync(active, want);
    if (who == 0) return 0;
    const int lane = threadIdx.x & 31, leader = __ffs(who) - 1;
    int first = 0;
    if (lane == leader) first = atomicAdd(count, __popc(who));
    return __shfl_sync(active, first, leader) + __popc(who & ((1u << lane) - 1));
}

// The keys of the share's `want` largest elements into few[], unordered, by
// bisection on the value: exact for any data, a pass over the row a bit.
// `list` and `scratch` are room to work in; returns how many there are.  (Kept
// out of line: inlined, its registers were spilled in the loops that run.)
template <typename T, int THREADS>
__device__ __noinline__ int exact_top(const RowStream<T, THREADS> S, int want, uint64_t* few, uint64_t* list,
                                      int* found, float* scratch)
{
    using V = Vec16<T>;
    constexpr int kN = V::kN;
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const int groups = S.groups();
    constexpr int kLow = sizeof(T) == 2 ? 16 : 0;  // a bf16 is its 16 high bits
    auto count_from = [&](uint32_t trial) {
        const float f = from_ordered(trial);
        int c = 0;
        for (int g = 0; g < groups; ++g)
#pragma unroll
            for (int u = 0; u < kHand; ++u) {
                const int v = S.vec(g, u);
                if (v >= S.v1) break;
                const uint4 x = S.load(v);
                if (V::value(V::larger(x)) < f) continue;
#pragma unroll
                for (int j = 0; j < kN; ++j)
                    c += ordered_bits(V::get(x, j)) >= trial && S.holds((int64_t)v * kN + j);
            }
        c = __reduce_add_sync(0xffffffffu, c);
        __syncthreads();
        if (t == 0) *found = 0;
        __syncthreads();
        if (lane == 0) atomicAdd(found, c);
        __syncthreads();
        return *found;
    };
    uint32_t value = 0;
    for (int b = 31; b >= kLow; --b)
        if (count_from(value | (1u << b)) >= want) value |= 1u << b;
    // (bf16: the bits below, as ordered_bits leaves them)
    if (kLow && (!(value & 0x80000000u) || value == 0xFFFF0000u)) value |= 0xFFFFu;
    // the keys above it, and of those that tie the lowest indices: the
    // threads' vectors of one step lie in order, so the ties of a step
    // are numbered by a scan over the CTA
    __syncthreads();
    if (t == 0) *found = 0;
    __syncthreads();
    int ties = 0;  // found so far
    int32_t* warps = reinterpret_cast<int32_t*>(scratch);
    for (int g = 0; g < groups; ++g)
        for (int u = 0; u < kHand; ++u) {
            const int v = S.vec(g, u);
            const uint4 x = S.load(v);
            unsigned equal = 0;
            for (int j = 0; j < kN; ++j) {
                const int64_t slot = (int64_t)v * kN + j;
                if (v >= S.v1 || !S.holds(slot)) continue;
                const float f = V::get(x, j);
                const uint32_t o = ordered_bits(f);
                if (o > value) {
                    const int i = atomicAdd(found, 1);
                    if (i < kTopKeys / 2) few[i] = top_key(f, slot - S.begin);
                } else if (o == value) {
                    equal |= 1u << j;
                }
            }
            if (ties >= want) continue;
            const int mine = __popc(equal);
            int upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int y = __shfl_up_sync(0xffffffffu, upto, o);
                upto += lane >= o ? y : 0;
            }
            __syncthreads();
            if (lane == 31) warps[warp] = upto;
            __syncthreads();
            int at = ties + upto - mine;
            for (int w = 0; w < THREADS / 32; ++w) {
                if (w < warp) at += warps[w];
                ties += warps[w];
            }
            for (; equal; equal &= equal - 1, ++at) {
                const int j = __ffs(equal) - 1;
                if (at < want) list[at] = top_key(V::get(x, j), (int64_t)v * kN + j - S.begin);
            }
        }
    __syncthreads();
    // fewer than `want` are above; the first ties complete them
    const int above = min(*found, want);
    ties = min(ties, want - above);
    for (int i = t; i < ties; i += THREADS) few[above + i] = list[i];
    __syncthreads();
    return above + ties;
}

template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_top_logits(const __grid_constant__ TopParams p)
{
    using V = Vec16<T>;
    constexpr int kN = V::kN;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    uint4* aside = reinterpret_cast<uint4*>(smem_raw);               // [kTopVectors]
    uint64_t* list = reinterpret_cast<uint64_t*>(aside + kTopVectors);  // [kTopKeys]
    uint64_t* few = reinterpret_cast<uint64_t*>(aside);              // [kTopKeys], once the vectors are done with
    int32_t* aside_at = reinterpret_cast<int32_t*>(list + kTopKeys);  // [kTopVectors]
    uint64_t* merged = reinterpret_cast<uint64_t*>(aside_at + kTopVectors);  // rank 0: [ctas][k]
    uint64_t* never = merged + (p.row.ctas > 1 ? (size_t)p.row.ctas * p.k : 0);
    float(*parts)[2] = reinterpret_cast<float(*)[2]>(never + 1);     // [kRowCtas]
    float* scratch = reinterpret_cast<float*>(parts + kRowCtas);     // [2][32]
    int* count = reinterpret_cast<int*>(scratch + 64);               // vectors, keys, survivors
    uint32_t* bounds = reinterpret_cast<uint32_t*>(count + 3);       // [2]
    uint16_t* maxima = reinterpret_cast<uint16_t*>(bounds + 3);      // [THREADS]
    // [kTopVectors]: maxima of what lies aside, then the keys' values, in 16 bits
    uint16_t* high16 = maxima + THREADS;

    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const bool alone = p.row.ctas == 1;
    const int rank = alone ? 0 : (int)(blockIdx.x % p.row.ctas);
    const int64_t r = alone ? blockIdx.x : blockIdx.x / p.row.ctas;
    const RowStream<T, THREADS> S(p.row, r, rank);
    if (!alone) cluster_arrive();
    wait_for_previous_grid();
    uint4 raw[kHand], next[kHand];
    S.load_group(raw, 0);
    S.load_group(next, 1);
    if (t == 0 && p.row.force_timeout_ns) {
        mbar_init(never, 1);
        if (!mbar_wait_bounded(never, 0, p.row.force_timeout_ns)) record_timeout(p.row.status);
    }

    const float c2 = kLog2e / p.temperature;
    auto top_of = [](const uint4 (&x)[kHand]) {
        typename V::Max m = V::larger(x[0]);
#pragma unroll
        for (int u = 1; u < kHand; ++u) m = V::larger(m, V::larger(x[u]));
        return m;
    };

    const int groups = S.groups();
    // elements of this share, and how many of its largest are wanted
    const int64_t first = max((int64_t)S.v0 * kN, (int64_t)S.begin);
    const int have = (int)max((int64_t)0, min((int64_t)S.v1 * kN, S.end) - first);
    const int want = min(have, p.k);

    const typename V::Max top0 = top_of(raw), top1 = top_of(next);
    // (0 from a thread that holds nothing: it must not count)
    uint32_t best = t < S.v1 - S.v0 ? ordered_bits(V::value(V::larger(top0, top1))) >> 16 : 0;
    const bool fours = p.k * 8 <= THREADS;
    if (fours) {
        best = max(best, __shfl_xor_sync(0xffffffffu, best, 1));
        best = max(best, __shfl_xor_sync(0xffffffffu, best, 2));
        if ((t & 3) == 0) maxima[t / 4] = (uint16_t)best;
    } else {
        maxima[t] = (uint16_t)best;
    }
    if (t < 3) count[t] = 0;
    __syncthreads();
    // one warp settles the bound while the others begin the sum
    if (warp == 0) {
        const uint32_t b = fours ? kth_largest<THREADS / 128>(maxima, want, 0) : kth_largest<THREADS / 32>(maxima, want, 0);
        if (t == 0) bounds[0] = b << 16;
    }
    RunningSum run;
    if (p.lse) {
        run.template add<T>(raw, top0, c2);
        run.template add<T>(next, top1, c2);
    }
    __syncthreads();
    uint32_t bound = bounds[0];
    float least = from_ordered(bound);

    // put a vector aside if its maximum reaches the bound (a NaN, or a bound
    // that is none, compares as if it did)
    auto keep = [&](const uint4& x, int v) {
        if (!(V::value(V::larger(x)) < least) && v < S.v1) {
            const int i = atomicAdd(count, 1);
            if (i < kTopVectors) {
                aside[i] = x;
                aside_at[i] = v;
            }
        }
    };
#pragma unroll
    for (int u = 0; u < kHand; ++u) keep(raw[u], S.vec(0, u));
#pragma unroll
    for (int u = 0; u < kHand; ++u) keep(next[u], S.vec(1, u));
    // each doubling of the part read puts some k vectors more aside
    const bool renew = p.k * groups > 1200;
    for (int g = 2, stop = renew ? 4 : groups;; stop = min(2 * stop, groups)) {
        stop = min(stop, groups);
        if (g < stop) S.load_group(raw, g);
        for (; g < stop; ++g) {
            if (g + 1 < stop) S.load_group(next, g + 1);
#pragma unroll
            for (int u = 0; u < kHand; ++u) keep(raw[u], S.vec(g, u));
            if (p.lse) run.template add<T>(raw, top_of(raw), c2);
#pragma unroll
            for (int u = 0; u < kHand; ++u) raw[u] = next[u];
        }
        if (g >= groups) break;
        __syncthreads();
        const int n = count[0];
        for (int i = t; i < min(n, kTopVectors); i += THREADS)
            high16[i] = (uint16_t)(ordered_bits(V::value(V::larger(aside[i]))) >> 16);
        __syncthreads();
        if (n <= kTopVectors)
            bound = block_kth_largest<THREADS>(n, want, bound >> 16, [=](int i) { return (uint32_t)high16[i]; }) << 16;
        least = from_ordered(bound);
    }
    float m = neg_inf(), s = 0.0f;
    if (p.lse) {
        block_sum<THREADS>(run, c2, scratch, m, s);
        if (is_far(m, c2)) s = far_sum(S, m, c2, scratch, [](uint4&, int, int) {});
        if (alone && t == 0)
            p.lse[r] = m == neg_inf() && s == 0.0f ? neg_inf() : m / p.temperature + logf(s);
    }
    __syncthreads();

    const int n_aside = count[0];
    int n = kTopKeys + 1;
    for (int i = t; i < kTopShort; i += THREADS) high16[i] = 0;
    __syncthreads();
    if (n_aside <= kTopVectors) {
        // a vector a thread: its elements at or above the bound
        for (int i = t; i < (n_aside + 31) / 32 * 32; i += THREADS) {
            const uint4 x = aside[i < n_aside ? i : 0];
            const int64_t slot = (int64_t)aside_at[i < n_aside ? i : 0] * kN;
            unsigned hits = 0;
            if (i < n_aside) {
#pragma unroll
                for (int j = 0; j < kN; ++j)
                    hits |= (unsigned)(ordered_bits(V::get(x, j)) >= bound && S.holds(slot + j)) << j;
            }
            const int mine = __popc(hits);
            int upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) {
                const int y = __shfl_up_sync(0xffffffffu, upto, o);
                upto += lane >= o ? y : 0;
            }
            int at = 0;
            if (lane == 31) at = atomicAdd(count + 1, upto);
            at = __shfl_sync(0xffffffffu, at, 31) + upto - mine;
            for (; hits; hits &= hits - 1, ++at) {
                const int j = __ffs(hits) - 1;
                const uint64_t key = top_key(V::get(x, j), slot + j - S.begin);
                if (at < kTopKeys) list[at] = key;
                if (at < kTopShort) high16[at] = (uint16_t)(key >> 48);
            }
        }
        __syncthreads();
        n = count[1];
    }
    if (n >= want && n <= kTopKeys) {
        // the want-th largest in 16 bits
        uint32_t second;
        if (n <= kTopShort) {
            if (warp == 0) {
                const uint32_t b = kth_largest<kTopShort / 32>(high16, want, bound >> 16);
                if (t == 0) bounds[1] = b;
            }
            __syncthreads();
            second = bounds[1];
        } else {
            second = block_kth_largest<THREADS>(n, want, bound >> 16, [=](int i) { return (uint32_t)(list[i] >> 48); });
        }
        const uint64_t least_key = (uint64_t)second << 48;
        for (int i = t; i < (n + 31) / 32 * 32; i += THREADS) {
            const uint64_t key = i < n ? list[i] : 0;
            const bool in = i < n && key >= least_key;
            const int j = take_place(count + 2, in);
            if (in) few[j] = key;
        }
        __syncthreads();
        n = count[2];
    } else {
        n = exact_top<T, THREADS>(S, want, few, list, count + 2, scratch);
    }

    // in order: a key's place is the number above it
    if (!alone) cluster_wait();  // every CTA of the row has started: its shared memory may be written
    const uint32_t to = alone ? 0 : peer_addr(smem_u32(merged + (size_t)rank * p.k), 0);
    for (int i = t; i < (4 * n + 31) / 32 * 32; i += THREADS) {
        // four threads a key, a quarter of the others each
        const uint64_t key = i < 4 * n ? few[i / 4] : ~0ull;
        int above = 0;
#pragma unroll 4
        for (int j = i & 3; j < n; j += 4) above += few[j] > key;
        above += __shfl_xor_sync(0xffffffffu, above, 1);
        above += __shfl_xor_sync(0xffffffffu, above, 2);
        if (i >= 4 * n || (i & 3) != 0 || above >= p.k) continue;
        if (alone) {
            p.values[r * p.k + above] = from_ordered((uint32_t)(key >> 32));
            p.indices[r * p.k + above] = (int32_t)~(uint32_t)key;
        } else {
            st_peer(to + (uint32_t)above * 8, key);
        }
    }
    if (alone) return;
    for (int i = n + t; i < p.k; i += THREADS) st_peer(to + (uint32_t)i * 8, (uint64_t)0);
    if (p.lse && t == 0) {
        const uint32_t part = peer_addr(smem_u32(&parts[rank][0]), 0);
        st_peer(part, m);
        st_peer(part + 4, s);
    }
    cluster_sync();
    if (rank != 0) return;

    for (int i = t; i < p.row.ctas * p.k; i += THREADS) {
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
