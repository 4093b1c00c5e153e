// Rows of logits streamed through registers.
//
// A row is read as 16-byte vectors from the 16-byte boundary at or before its
// first element: rows may start anywhere, and the two vectors that a row fills
// only in part are read element by element and completed with -inf.  A CTA
// takes a row (a cluster of CTAs takes one, a contiguous share each, where
// rows are few).  Each thread keeps four vectors in hand and the next four on
// their way.
//
// A row is not kept in shared memory between passes: that ties its bytes to a
// chain of reductions and barriers, and with at most 228 KB an SM the copies
// wait for it (the 4096 x 131072 distillation took 457 us that way, 372 so).
// A second pass finds most of the row in L2.
#pragma once

#include <cuda_bf16.h>

#include "cluster.cuh"
#include "logits.h"

namespace quasar {

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xFF800000); }

// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// 16 bytes of T: as pairs of floats, and their maximum (bf16: two at a time,
// four instructions a vector).
template <typename T>
struct Vec16;

template <>
struct Vec16<float> {
    static constexpr int kN = 4;
    static constexpr uint32_t kNone = 0xFF800000u;  // -inf
    using Max = float;
    static __device__ __forceinline__ uint32_t replace(uint32_t, int, float x) { return __float_as_uint(x); }
    static __device__ __forceinline__ void put(uint32_t (&w)[4], int j, float x) { w[j] = __float_as_uint(x); }
    static __device__ __forceinline__ float get(const uint4& x, int j)
    {
        return __uint_as_float(j & 2 ? (j & 1 ? x.w : x.z) : (j & 1 ? x.y : x.x));
    }
    static __device__ __forceinline__ void unpack(const uint4& x, float2 (&v)[2])
    {
        v[0] = make_float2(__uint_as_float(x.x), __uint_as_float(x.y));
        v[1] = make_float2(__uint_as_float(x.z), __uint_as_float(x.w));
    }
    static __device__ __forceinline__ uint4 pack(const float2 (&v)[2])
    {
        return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x),
                          __float_as_uint(v[1].y));
    }
    static __device__ __forceinline__ Max larger(const uint4& x)
    {
        return max_nan(max_nan(__uint_as_float(x.x), __uint_as_float(x.y)),
                       max_nan(__uint_as_float(x.z), __uint_as_float(x.w)));
    }
    static __device__ __forceinline__ Max larger(Max m, Max n) { return max_nan(m, n); }
    static __device__ __forceinline__ float value(Max m) { return m; }
    static __device__ __forceinline__ float to_f32(float x) { return x; }
    static __device__ __forceinline__ float from_f32(float x) { return x; }
};

template <>
struct Vec16<__nv_bfloat16> {
    static constexpr int kN = 8;
    static constexpr uint32_t kNone = 0xFF80FF80u;  // two of -inf
    using Max = __nv_bfloat162;
    static __device__ __forceinline__ uint32_t replace(uint32_t word, int j, __nv_bfloat16 x)
    {
        const uint32_t bits = __bfloat16_as_ushort(x);
        return j & 1 ? (word & 0xFFFFu) | bits << 16 : (word & 0xFFFF0000u) | bits;
    }
    static __device__ __forceinline__ void put(uint32_t (&w)[4], int j, __nv_bfloat16 x)
    {
        w[j / 2] = replace(w[j / 2], j, x);
    }
    static __device__ __forceinline__ float get(const uint4& x, int j)
    {
        const uint32_t w = j & 4 ? (j & 2 ? x.w : x.z) : (j & 2 ? x.y : x.x);
        return j & 1 ? bf16hi(w) : bf16lo(w);
    }
    static __device__ __forceinline__ Max pair(uint32_t x) { return *reinterpret_cast<const Max*>(&x); }
    static __device__ __forceinline__ void unpack(const uint4& x, float2 (&v)[4])
    {
        v[0] = make_float2(bf16lo(x.x), bf16hi(x.x));
        v[1] = make_float2(bf16lo(x.y), bf16hi(x.y));
        v[2] = make_float2(bf16lo(x.z), bf16hi(x.z));
        v[3] = make_float2(bf16lo(x.w), bf16hi(x.w));
    }
    static __device__ __forceinline__ uint4 pack(const float2 (&v)[4])
    {
        return make_uint4(pack_bf16x2(v[0].x, v[0].y), pack_bf16x2(v[1].x, v[1].y),
                          pack_bf16x2(v[2].x, v[2].y), pack_bf16x2(v[3].x, v[3].y));
    }
    static __device__ __forceinline__ Max larger(const uint4& x)
    {
        return __hmax2_nan(__hmax2_nan(pair(x.x), pair(x.y)), __hmax2_nan(pair(x.z), pair(x.w)));
    }
    static __device__ __forceinline__ Max larger(Max m, Max n) { return __hmax2_nan(m, n); }
    static __device__ __forceinline__ float value(Max m)
    {
        const uint32_t x = *reinterpret_cast<const uint32_t*>(&m);
        return max_nan(bf16lo(x), bf16hi(x));
    }
    static __device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 from_f32(float x) { return __float2bfloat16_rn(x); }
};

// A load that is issued where it stands (the compiler would move it down to
// its use, and the next vectors would no longer be on their way).  An ordinary
// load, not a read-only one: a gradient may take the logits' place within the
// launch, each vector written after its thread has read it.
// KEEP: the line may be wanted again, and stays in L2 before others (the
// distillation's first pass asks so whether a gradient follows or not);
// otherwise it goes first.
template <bool KEEP>
__device__ __forceinline__ uint4 load_now(const uint4* p)
{
    uint4 x;
    if constexpr (KEEP)
        asm volatile(
            "{\n\t.reg .b64 keep;\n\tcreatepolicy.fractional.L2::evict_last.b64 keep, 1.0;\n\t"
            "ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], keep;\n\t}"
            : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
            : "l"(p));
    else
        asm volatile(
            "{\n\t.reg .b64 drop;\n\tcreatepolicy.fractional.L2::evict_first.b64 drop, 1.0;\n\t"
            "ld.global.L1::no_allocate.L2::cache_hint.v4.u32 {%0, %1, %2, %3}, [%4], drop;\n\t}"
            : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
            : "l"(p));
    return x;
}

__device__ __forceinline__ float load_one(const float* p)
{
    float x;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(x) : "l"(p));
    return x;
}

__device__ __forceinline__ __nv_bfloat16 load_one(const __nv_bfloat16* p)
{
    unsigned short x;
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(x) : "l"(p));
    return __ushort_as_bfloat16(x);
}

constexpr float kLog2e = 1.44269504f;
constexpr int kHand = 4;  // vectors a thread works on at a time

// One CTA's share of a row.  Slots count elements from vector 0.
template <typename T, int THREADS>
struct RowStream {
    static constexpr int kN = Vec16<T>::kN;
    const T* slot0;      // the 16-byte boundary at or before the row
    int begin;           // slot of element 0
    int64_t end;         // slot after the last element
    int v0, v1;          // this CTA's vectors
    int whole0, whole1;  // of those, the ones the row fills
    bool ragged;         // not all

    __device__ __forceinline__ RowStream(const RowParams& p, int64_t r, int rank)
    {
        const T* row = static_cast<const T*>(p.logits) + r * p.ld;
        begin = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        slot0 = row - begin;
        end = begin + p.vocab;
        const int vecs = (int)((end + kN - 1) / kN);
        v0 = min(rank * p.vecs, vecs);
        v1 = min(v0 + p.vecs, vecs);
        whole0 = v0 == 0 && begin > 0 ? 1 : v0;
        whole1 = v1 == vecs && end < (int64_t)vecs * kN ? v1 - 1 : v1;
        if (whole1 < whole0) whole1 = whole0;
        ragged = whole0 > v0 || whole1 < v1;
    }

    __device__ __forceinline__ bool whole(int v) const
    {
        return (unsigned)(v - whole0) < (unsigned)(whole1 - whole0);
    }

    __device__ __forceinline__ bool holds(int64_t slot) const { return slot >= begin && slot < end; }

    // vector u of this thread's group g
    __device__ __forceinline__ int vec(int g, int u) const
    {
        return v0 + (g * kHand + u) * THREADS + (int)threadIdx.x;
    }

    __device__ __forceinline__ int groups() const { return (v1 - v0 + kHand * THREADS - 1) / (kHand * THREADS); }

    // A vector that the row fills in part: what lies outside it as -inf.  (A
    // loop, inlined: a call from the loops over groups would spill their
    // registers, and unrolled it is most of their code.)
    __device__ __forceinline__ uint4 load_part(int v) const
    {
        uint4 x = none();
#pragma unroll 1
        for (int j = 0; j < kN; ++j) {
            const int64_t s = (int64_t)v * kN + j;
            if (!holds(s)) continue;
            const int word = j * (int)sizeof(T) / 4;
            uint32_t old = word == 0 ? x.x : word == 1 ? x.y : word == 2 ? x.z : x.w;
            old = Vec16<T>::replace(old, j, slot0[s]);
            if (word == 0) x.x = old;
            if (word == 1) x.y = old;
            if (word == 2) x.z = old;
            if (word == 3) x.w = old;
        }
        return x;
    }

    __device__ __forceinline__ static uint4 none()
    {
        return make_uint4(Vec16<T>::kNone, Vec16<T>::kNone, Vec16<T>::kNone, Vec16<T>::kNone);
    }

    __device__ __forceinline__ uint4 load(int v) const
    {
        if (whole(v)) return load_now<false>(reinterpret_cast<const uint4*>(slot0) + v);
        return v >= v0 && v < v1 ? load_part(v) : none();
    }

    template <bool KEEP = false>
    __device__ __forceinline__ void load_group(uint4 (&raw)[kHand], int g) const
    {
        const int v = vec(g, 0);
        const uint4* p = reinterpret_cast<const uint4*>(slot0) + v;
        const unsigned at = (unsigned)(v - whole0), n = (unsigned)(whole1 - whole0);
        if (at < n && at + (kHand - 1) * THREADS < n) {
#pragma unroll
            for (int u = 0; u < kHand; ++u) raw[u] = load_now<KEEP>(p + u * THREADS);
            return;
        }
#pragma unroll
        for (int u = 0; u < kHand; ++u) {
            raw[u] = none();
            if (at + u * THREADS < n) raw[u] = load_now<KEEP>(p + u * THREADS);
        }
        if (ragged) {
#pragma unroll
            for (int u = 0; u < kHand; ++u) {
                const int w = v + u * THREADS;
                if (at + u * THREADS >= n && w >= v0 && w < v1) raw[u] = load_part(w);
            }
        }
    }

    // Where the vectors of this thread's group all lie within the row.
    __device__ __forceinline__ bool whole_group(int g) const
    {
        const unsigned at = (unsigned)(vec(g, 0) - whole0), n = (unsigned)(whole1 - whole0);
        return at < n && at + (kHand - 1) * THREADS < n;
    }
};

// Sums of exponentials are kept as (m, s), meaning sum e^(x / tau) = s e^(m /
// tau) with m one of the logits; c = log2(e) / tau.  m = -inf: nothing was
// added (s = 0), or nothing but NaN (s = NaN; m does not see one); m = inf: s is
// inf, or NaN.
__device__ __forceinline__ void merge_sum(float& m, float& s, float m2, float s2, float c)
{
    const float top = fmaxf(m, m2);
    if (top == neg_inf()) {
        s += s2;
        return;
    }
    s = (m == top ? s : s * exp2f((m - top) * c)) + (m2 == top ? s2 : s2 * exp2f((m2 - top) * c));
    m = top;
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float warp_sum(float x)
{
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// 2^((x - m) c) as one multiply-add and one exponential: 2^(x c - base) times
// fix(), with base = m c as rounded and fix what that rounding took away: at
// most one half up to kFar, where the base stays.  Rows whose largest logit
// lies farther out (masked with -1e10, or with the type's lowest value) take
// the subtraction first, by is_far: a product's ulp of its own would be worth
// powers of two there.
constexpr float kFar = 16777216.0f;  // 2^24

__device__ __forceinline__ float exp_base(float m, float c) { return fminf(fmaxf(m * c, -kFar), kFar); }
__device__ __forceinline__ float exp_fix(float m, float c, float base) { return exp2f(-fmaf(m, c, -base)); }

// A thread's running sum: s = sum of 2^(x c - base).
struct RunningSum {
    float m, base, s;

    __device__ __forceinline__ RunningSum() : m(neg_inf()), base(-kFar), s(0.0f) {}

    template <typename T>
    __device__ __forceinline__ void add(const uint4 (&raw)[kHand], typename Vec16<T>::Max top, float c)
    {
        constexpr int kP = Vec16<T>::kN / 2;
        m = fmaxf(m, Vec16<T>::value(top));
        const float next = exp_base(m, c);
        s *= ex2(base - next);
        base = next;
        const float2 cc = make_float2(c, c), bb = make_float2(-base, -base);
        float2 sum = make_float2(s, 0.0f);
#pragma unroll
        for (int u = 0; u < kHand; ++u) {
            float2 x[kP];
            Vec16<T>::unpack(raw[u], x);
#pragma unroll
            for (int j = 0; j < kP; ++j) {
                x[j] = __ffma2_rn(x[j], cc, bb);
                x[j] = make_float2(ex2(x[j].x), ex2(x[j].y));
            }
#pragma unroll
            for (int j = 0; j < kP; ++j) sum = __fadd2_rn(sum, x[j]);
        }
        s = sum.x + sum.y;
    }
};

// Over the CTA: (m, s) as merge_sum keeps them, the same in every thread.
// `scratch` holds two floats a warp; a barrier separates its uses.
template <int THREADS>
__device__ __forceinline__ void block_sum(const RunningSum& r, float c, float* scratch, float& m, float& s)
{
    constexpr int kW = THREADS / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float top = lanes_max(r.m, 0xffffffffu);
    const float part = warp_sum(r.s * ex2(r.base - exp_base(top, c)));
    if (lane == 0) {
        scratch[warp] = top;
        scratch[kW + warp] = part;
    }
    __syncthreads();
    const float w = lane < kW ? scratch[lane] : neg_inf();
    m = lanes_max(w, 0xffffffffu);
    const float base = exp_base(m, c);
    s = warp_sum(lane < kW ? scratch[kW + lane] * ex2(exp_base(w, c) - base) : 0.0f);
    s = isinf(m) ? s : s * exp_fix(m, c, base);
}

// Where the largest logit lies so far out that the base stopped at kFar: the
// sum again, the subtraction first.  `drop` replaces what a thread's vector (g, u) must
// not count.
// (Out of line, and its arguments by value: a reference would keep the caller's
// variables in memory.)
template <typename T, int THREADS, typename Drop>
__device__ __noinline__ float far_sum(const RowStream<T, THREADS> S, float m, float c, float* scratch, Drop drop)
{
    constexpr int kP = Vec16<T>::kN / 2;
    float s = 0.0f;
    for (int g = 0; g < S.groups(); ++g)
        for (int u = 0; u < kHand; ++u) {
            uint4 raw = S.load(S.vec(g, u));
            drop(raw, g, u);
            float2 x[kP];
            Vec16<T>::unpack(raw, x);
#pragma unroll
            for (int j = 0; j < kP; ++j) s += ex2((x[j].x - m) * c) + ex2((x[j].y - m) * c);
        }
    s = warp_sum(s);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = s;
    __syncthreads();
    s = warp_sum((threadIdx.x & 31) < THREADS / 32 ? scratch[threadIdx.x & 31] : 0.0f);
    __syncthreads();
    return s;
}

__device__ __forceinline__ bool is_far(float m, float c) { return !isinf(m) && fabsf(m * c) > kFar; }

}  // namespace quasar
