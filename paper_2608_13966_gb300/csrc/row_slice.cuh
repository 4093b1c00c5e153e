// One row of logits held in the shared memory of a cluster, so that a row is
// read from HBM once however often it is passed over.
//
// The row is cut at 16-byte addresses: vector 0 is the 16 bytes that hold the
// row's first element, and CTA c of the cluster holds the vectors [c vecs,
// (c + 1) vecs).  Rows may start at any element; the two vectors that the row
// fills only in part are loaded element by element and completed with -inf,
// the rest arrives by bulk copies.
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
    using Max = float;
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
    static __device__ __forceinline__ Max lowest() { return neg_inf(); }
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
    using Max = __nv_bfloat162;
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
    static __device__ __forceinline__ Max lowest() { return pair(0xFF80FF80u); }
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

// Where a CTA's slice of one row lies.  Slots count elements from the 16-byte
// boundary at or before the slice's first element.
template <typename T>
struct RowSlice {
    static constexpr int kN = Vec16<T>::kN;
    const T* base;     // slot 0 (the row itself may start after it)
    int64_t element0;  // element of the row at slot 0 (negative: the row starts after it)
    int n_vecs;        // vectors of the slice (may be 0)
    int begin, end;    // slots that hold elements
    int whole0, whole1;  // vectors the row fills
    int per_chunk;     // whole vectors a copy brings

    __device__ __forceinline__ RowSlice(const RowParams& p, int64_t r, int rank)
    {
        const T* row = static_cast<const T*>(p.logits) + r * p.ld;
        const int lead = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
        const int64_t slots = lead + p.vocab;
        const int64_t vecs = (slots + kN - 1) / kN;
        const int64_t v0 = (int64_t)rank * p.vecs;
        n_vecs = (int)(v0 >= vecs ? 0 : (vecs - v0 < p.vecs ? vecs - v0 : p.vecs));
        element0 = v0 * kN - lead;
        base = row + element0;
        begin = element0 < 0 ? (int)-element0 : 0;
        const int64_t left = p.vocab - element0;
        end = left < (int64_t)n_vecs * kN ? (int)left : n_vecs * kN;
        if (n_vecs == 0) begin = end = 0;
        whole0 = begin > 0 ? 1 : 0;
        whole1 = end < n_vecs * kN ? n_vecs - 1 : n_vecs;
        if (whole1 < whole0) whole1 = whole0;
        per_chunk = (whole1 - whole0 + kRowChunks - 1) / kRowChunks;
    }

    // slot of element e; -1 if another CTA holds it
    __device__ __forceinline__ int slot_of(int e) const
    {
        const int64_t s = e - element0;
        return s >= begin && s < end ? (int)s : -1;
    }

    __device__ __forceinline__ bool whole(int v) const
    {
        return (unsigned)(v - whole0) < (unsigned)(whole1 - whole0);
    }

    // whether largest() gives thread t any element
    __device__ __forceinline__ bool holds(int t) const
    {
        return t < min(per_chunk, whole1 - whole0) || (t == 0 && whole0 == 1 && n_vecs > 0) ||
               (t == 1 && whole1 < n_vecs);
    }

    // Start loading the slice; every thread calls it, and a barrier follows
    // before the slice is touched.  Thread 0 initialises the chunks' barriers
    // and issues the copies of the whole vectors; the (at most two) partial
    // ones are loaded and completed with -inf by the first warp.
    __device__ __forceinline__ void load(T* smem, uint64_t* bars, uint64_t* never) const
    {
        const int t = threadIdx.x;
        if (t == 0) {
            for (int c = 0; c < kRowChunks; ++c) mbar_init(bars + c, 1);
            mbar_init(never, 1);
            mbar_init_fence();
            for (int c = 0; c < kRowChunks; ++c) {
                const int a = min(whole0 + c * per_chunk, whole1), b = min(a + per_chunk, whole1);
                mbar_arrive_expect_tx(bars + c, (uint32_t)(b - a) * 16u);
                if (b > a) bulk_g2s(smem + (size_t)a * kN, base + (size_t)a * kN, (uint32_t)(b - a) * 16u, bars + c);
            }
        }
        if (t < 2 * kN) {
            const int v = t < kN ? 0 : n_vecs - 1;
            if (v >= 0 && v < n_vecs && !whole(v) && !(t >= kN && v == 0)) {
                const int s = v * kN + t % kN;
                smem[s] = s >= begin && s < end ? base[s] : Vec16<T>::from_f32(neg_inf());
            }
        }
    }

    // This thread's largest logit, chunk by chunk as the copies land.
    // Records a timeout where one does not.
    __device__ __forceinline__ float largest(const T* smem, uint64_t* bars, const RowParams& p) const
    {
        const uint4* vecs = reinterpret_cast<const uint4*>(smem);
        typename Vec16<T>::Max m = Vec16<T>::lowest();
        for (int c = 0; c < kRowChunks; ++c) {
            if (!mbar_wait_bounded(bars + c, 0, p.timeout_ns)) record_timeout(p.status);
            const int stop = min(whole0 + (c + 1) * per_chunk, whole1);
#pragma unroll 4
            for (int v = whole0 + c * per_chunk + threadIdx.x; v < stop; v += blockDim.x)
                m = Vec16<T>::larger(m, Vec16<T>::larger(vecs[v]));
        }
        if (threadIdx.x == 0 && whole0 == 1 && n_vecs > 0) m = Vec16<T>::larger(m, Vec16<T>::larger(vecs[0]));
        if (threadIdx.x == 1 && whole1 < n_vecs) m = Vec16<T>::larger(m, Vec16<T>::larger(vecs[n_vecs - 1]));
        return Vec16<T>::value(m);
    }
};

constexpr float kLog2e = 1.44269504f;
constexpr float kLn2 = 0.69314718f;

// Sums of exponentials are kept as (m, s), meaning sum e^(x / tau) = s e^(m /
// tau) with m one of the logits; c = log2(e) / tau.  m = -inf: nothing was
// added.
__device__ __forceinline__ void merge_sum(float& m, float& s, float m2, float s2, float c)
{
    const float top = fmaxf(m, m2);
    if (top == neg_inf()) return;
    s = s * exp2f((m - top) * c) + s2 * exp2f((m2 - top) * c);
    m = top;
}

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Maximum and sum over the CTA.  `scratch` holds a float per warp and is not
// reused without a barrier in between.
__device__ __forceinline__ float block_max(float x, float* scratch)
{
    x = lanes_max(x, 0xffffffffu);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = x;
    __syncthreads();
    return lanes_max(scratch[threadIdx.x & (blockDim.x / 32 - 1)], 0xffffffffu);
}

__device__ __forceinline__ float warp_sum(float x)
{
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// 2^((x - m) c) as one multiply-add and one exponential: 2^(x c - base) times
// fix, with base = m c as rounded and fix = 2^(base - m c), what that rounding
// took away.  m = -inf (nothing to add): base 0.  Where m c leaves fp32's
// range (a row masked with the type's lowest value) the subtraction comes
// first instead.
struct ExpBase {
    float base, fix, shift;
    __device__ __forceinline__ ExpBase(float m, float c)
    {
        base = m == neg_inf() ? 0.0f : m * c;
        fix = m == neg_inf() ? 1.0f : exp2f(-fmaf(m, c, -base));
        shift = 0.0f;
        if (isinf(base)) {
            base = 0.0f;
            fix = 1.0f;
            shift = -m;
        }
    }

    // the pairs x -> 2^(x c - base)
    template <int N>
    __device__ __forceinline__ void apply(float2 (&x)[N], float c) const
    {
        const float2 cc = make_float2(c, c), mm = make_float2(-base, -base);
        if (shift != 0.0f) {
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] = __fadd2_rn(x[j], make_float2(shift, shift));
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            x[j] = __ffma2_rn(x[j], cc, mm);
            x[j] = make_float2(ex2(x[j].x), ex2(x[j].y));
        }
    }
};

// The sum of 2^(x c - base) over this thread's vectors v = first, first + step, ...
template <typename T>
__device__ __forceinline__ float sum_exponentials(const T* slice, int n_vecs, int first, int step, float c,
                                                  const ExpBase& at)
{
    const uint4* vecs = reinterpret_cast<const uint4*>(slice);
    float2 s = make_float2(0.0f, 0.0f);
#pragma unroll 2
    for (int v = first; v < n_vecs; v += step) {
        float2 x[Vec16<T>::kN / 2];
        Vec16<T>::unpack(vecs[v], x);
        at.apply(x, c);
#pragma unroll
        for (int j = 0; j < Vec16<T>::kN / 2; ++j) s = __fadd2_rn(s, x[j]);
    }
    return s.x + s.y;
}

// This thread's largest logit of a slice that has landed.
template <typename T>
__device__ __forceinline__ float largest(const T* slice, int n_vecs)
{
    const uint4* vecs = reinterpret_cast<const uint4*>(slice);
    typename Vec16<T>::Max m = Vec16<T>::lowest();
#pragma unroll 4
    for (int v = threadIdx.x; v < n_vecs; v += blockDim.x)
        m = Vec16<T>::larger(m, Vec16<T>::larger(vecs[v]));
    return Vec16<T>::value(m);
}

}  // namespace quasar
