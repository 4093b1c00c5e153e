// Distillation from a teacher's top logits: the forward KL divergence of a
// row of student logits and its gradient.
//
// With z = logits / temperature, q = softmax(z) over the vocabulary, p the
// teacher's probabilities of its k listed entries, and the "rest" everything
// that is not listed (student mass q_r, teacher mass p_r):
//
//   loss = sum_k p_k log(p_k / q_k) + p_r log(p_r / q_r)
//        = sum of p log(p / q) - p + q over the entries and the rest,
//
// the second form because both sides sum to one: no term is negative, so
// nothing cancels.  With P = sum p_k + p_r and u_j = e^{z_j} / sum over the
// rest of e^z, the student's share of unlisted entry j within the rest,
//
//   dloss/dz_k = P q_k - p_k            (listed)
//   dloss/dz_j = u_j (P q_r - p_r)      (unlisted),
//
// which never divides by q_r.  The rest's sum is formed on its own (a listed
// logit is replaced by -inf in shared memory once it has been read), not as
// the difference of two sums.
#pragma once

#include "row_slice.cuh"

namespace quasar {

constexpr int kDistillThreads = 512;

// x / tau - y: the quotient is not rounded before the subtraction (inv_tau is
// 1 / tau rounded, the second step its remainder)
__device__ __forceinline__ float scaled_less(float x, float tau, float inv_tau, float y)
{
    const float low = fmaf(-tau, inv_tau, 1.0f) * inv_tau;
    const float d = fmaf(x, inv_tau, -y);
    return low == 0.0f ? d : fmaf(x, low, d);
}

// p log(p / q) - p + q from p, log p and log q
__device__ __forceinline__ float kl_term(float p, float log_p, float log_q)
{
    if (!(p > 0.0f)) return expf(log_q);
    const float d = log_p - log_q;
    return d > -1.0f ? p * (d + expm1f(-d)) : p * (d - 1.0f) + expf(log_q);
}

// Teacher side of a row, by one warp: log p of each entry into logp[] (-inf
// where absent), returns sum p; n_listed counts the entries present.
__device__ __forceinline__ float teacher_side(const DistillParams& p, int64_t r, float inv_tau,
                                              float* logp, int32_t* entry, int* n_listed)
{
    const int lane = threadIdx.x & 31;
    const int32_t* idx = p.indices + r * p.k;
    const float* val = p.values + r * p.k;
    float top = neg_inf();
    int n = 0;
    for (int k = lane; k < p.k; k += 32) {
        const int32_t e = idx[k];
        const bool here = e >= 0 && e < p.row.vocab;
        const float t = here ? val[k] * inv_tau : neg_inf();
        entry[k] = here ? e : -1;
        logp[k] = t;
        top = fmaxf(top, t);
        n += here;
    }
    *n_listed = __reduce_add_sync(0xffffffffu, n);
    float norm;
    if (p.teacher_lse) {
        norm = p.teacher_lse[r];
    } else {
        top = lanes_max(top, 0xffffffffu);
        float s = 0.0f;
        for (int k = lane; k < p.k; k += 32) s += top == neg_inf() ? 0.0f : expf(logp[k] - top);
        s = warp_sum(s);
        norm = s > 0.0f ? top + logf(s) : 0.0f;
    }
    float sum = 0.0f;
    for (int k = lane; k < p.k; k += 32) {
        logp[k] -= norm;
        sum += expf(logp[k]);
    }
    return warp_sum(sum);
}

// BACKWARD: the gradient from kept statistics (log-sum-exp of z over the
// vocabulary and over the rest).  Otherwise the loss, the statistics and, if
// asked, the gradient, the row staying in shared memory in between.
template <typename T, bool BACKWARD>
__global__ void __launch_bounds__(kDistillThreads) k_distill_top(const __grid_constant__ DistillParams p)
{
    using V = Vec16<T>;
    constexpr int kN = V::kN;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    T* slice = reinterpret_cast<T*>(smem_raw);
    uint64_t* bars = reinterpret_cast<uint64_t*>(smem_raw + (size_t)p.row.vecs * 16);
    uint64_t* never = bars + kRowChunks;
    float* logp = reinterpret_cast<float*>(never + 1);      // [kMaxTop]
    float* all = logp + kMaxTop;                            // rank 0: the entries' student logits
    float(*parts)[4] = reinterpret_cast<float(*)[4]>(all + kMaxTop);  // [kRowCtas]
    float* scratch = reinterpret_cast<float*>(parts + kRowCtas);      // [4][warps]
    float* teacher = scratch + 64;                          // P, p_r
    int32_t* entry = reinterpret_cast<int32_t*>(teacher + 4);  // [kMaxTop]

    const int t = threadIdx.x;
    const int rank = (int)(blockIdx.x % p.row.ctas);
    const int64_t r = blockIdx.x / p.row.ctas;
    const RowSlice<T> S(p.row, r, rank);
    wait_for_previous_grid();
    const float weight = p.row_weight ? p.row_weight[r] : 1.0f;
    T* grad = p.grad ? static_cast<T*>(p.grad) + r * p.ld_grad : nullptr;

    if (weight == 0.0f) {  // a row that counts nothing is not read
        if (grad)
            for (int s = S.begin + t; s < S.end; s += kDistillThreads) grad[S.element0 + s] = V::from_f32(0.0f);
        if (!BACKWARD && rank == 0 && t == 0) {
            p.loss[r] = 0.0f;
            if (p.stats) p.stats[2 * r] = p.stats[2 * r + 1] = 0.0f;
        }
        return;
    }

    if (!BACKWARD) cluster_arrive();
    S.load(slice, bars, never);
    const float inv_tau = 1.0f / p.temperature;
    if (t < 32) {
        int n_listed;
        const float sum = teacher_side(p, r, inv_tau, logp, entry, &n_listed);
        if (t == 0) {
            float rest = p.teacher_lse && n_listed < p.row.vocab ? fmaxf(1.0f - sum, 0.0f) : 0.0f;
            teacher[0] = sum + rest;
            teacher[1] = rest;
        }
    }
    __syncthreads();
    if (t == 0 && p.row.force_timeout_ns && !mbar_wait_bounded(never, 0, p.row.force_timeout_ns))
        record_timeout(p.row.status);

    const float mass = teacher[0], p_rest = teacher[1];
    const float c2 = kLog2e * inv_tau;
    float mine = 0.0f;  // this thread's largest logit, listed or not
    if (BACKWARD) {
        for (int c = 0; c < kRowChunks; ++c)
            if (!mbar_wait_bounded(bars + c, 0, p.row.timeout_ns)) record_timeout(p.row.status);
    } else {
        mine = S.largest(slice, bars, p.row);
        cluster_wait();  // every CTA of the row has started: its shared memory may be written
        __syncthreads();
    }
    // take the listed entry of this thread out of the slice
    const int listed = t < p.k && entry[t] >= 0 ? S.slot_of(entry[t]) : -1;
    float own = neg_inf();
    if (listed >= 0) {
        own = V::to_f32(slice[listed]);
        slice[listed] = V::from_f32(neg_inf());
        if (!BACKWARD) st_peer(peer_addr(smem_u32(all + t), 0), own);
    }

    float m_rest, coef, q_rest;          // of the whole row (backward: m_rest is the rest's lse)
    float m_all, log_s = 0.0f;           // lse = m_all / tau + log_s (backward: lse = m_all)
    if constexpr (!BACKWARD) {
        const int warp = t >> 5, lane = t & 31;
        // the base is the largest logit, even a listed one: the rest's sum is
        // fine about it unless the rest lies far below, which is then redone
        float m = block_max(mine, scratch);
        ExpBase at(m, c2);
        float s = warp_sum(sum_exponentials(slice, S.n_vecs, t, kDistillThreads, c2, at)) * at.fix;
        // the listed entries held here, as a second sum (one a thread)
        float m_in = neg_inf(), s_in = 0.0f;
        if (t < kMaxTop) {
            m_in = lanes_max(own, 0xffffffffu);
            s_in = warp_sum(own == neg_inf() ? 0.0f : exp2f((own - m_in) * c2));
        }
        if (lane == 0) {
            scratch[16 + warp] = s;
            scratch[32 + warp] = m_in;
            scratch[48 + warp] = s_in;
        }
        __syncthreads();
        constexpr int kW = kDistillThreads / 32;
        float sum = warp_sum(lane < kW ? scratch[16 + lane] : 0.0f);
        if (sum < 1e-20f) {
            m = block_max(largest(slice, S.n_vecs), scratch);
            at = ExpBase(m, c2);
            s = warp_sum(sum_exponentials(slice, S.n_vecs, t, kDistillThreads, c2, at)) * at.fix;
            if (lane == 0) scratch[16 + warp] = s;
            __syncthreads();
            sum = warp_sum(lane < kW ? scratch[16 + lane] : 0.0f);
        }
        if (warp == 0) {
            const float x = lane < kW ? scratch[32 + lane] : neg_inf();
            m_in = lanes_max(x, 0xffffffffu);
            s_in = warp_sum(x == neg_inf() ? 0.0f : scratch[48 + lane] * exp2f((x - m_in) * c2));
            if (lane < p.row.ctas) {
                const uint32_t to = peer_addr(smem_u32(&parts[rank][0]), (uint32_t)lane);
                st_peer(to, m);
                st_peer(to + 4, sum);
                st_peer(to + 8, m_in);
                st_peer(to + 12, s_in);
            }
        }
        cluster_sync();
        float m_listed = neg_inf(), s_listed = 0.0f, s_rest = 0.0f;
        m_rest = neg_inf();
        for (int c = 0; c < p.row.ctas; ++c) {
            merge_sum(m_rest, s_rest, parts[c][0], parts[c][1], c2);
            merge_sum(m_listed, s_listed, parts[c][2], parts[c][3], c2);
        }
        float s_all = s_rest;
        m_all = m_rest;
        merge_sum(m_all, s_all, m_listed, s_listed, c2);
        log_s = logf(s_all);
        const bool some = m_rest != neg_inf();
        const float log_q_rest = some ? (m_rest - m_all) * inv_tau + (logf(s_rest) - log_s) : neg_inf();
        q_rest = expf(log_q_rest);
        coef = some ? (mass * q_rest - p_rest) / s_rest : 0.0f;
        if (rank == 0 && t < 32) {
            float loss = 0.0f;
            for (int k = t; k < p.k; k += 32)
                if (entry[k] >= 0)
                    loss += kl_term(expf(logp[k]), logp[k], (all[k] - m_all) * inv_tau - log_s);
            loss = warp_sum(loss);
            if (t == 0) {
                loss += kl_term(p_rest, logf(p_rest), log_q_rest);
                if (m_all == neg_inf()) loss = __int_as_float(0x7F800000);  // q is 0 everywhere
                p.loss[r] = mass > 0.0f ? loss : 0.0f;
                if (p.stats) {
                    p.stats[2 * r] = m_all / p.temperature + log_s;
                    p.stats[2 * r + 1] = some ? m_rest / p.temperature + logf(s_rest) : neg_inf();
                }
            }
        }
        if (!grad) return;
    } else {
        m_all = p.stats[2 * r];
        const float lse_rest = p.stats[2 * r + 1];
        const bool some = lse_rest != neg_inf();
        q_rest = some ? expf(lse_rest - m_all) : 0.0f;
        coef = some ? mass * q_rest - p_rest : 0.0f;
        m_rest = some ? lse_rest : 0.0f;
    }
    // a row without teacher mass, or without a finite logit, has no gradient
    const bool none = !(mass > 0.0f) || m_all == neg_inf();
    const float scale = none ? 0.0f : weight * inv_tau;
    coef *= scale;

    // the unlisted entries: coef 2^(x c - base), or coef e^(z - lse) from
    // kept statistics
    T* out = grad + S.element0;  // of slot 0
    const bool vectors = (reinterpret_cast<uintptr_t>(out) & 15) == 0;
    const ExpBase at(BACKWARD ? 0.0f : m_rest, c2);
    coef *= at.fix;
    const float2 kk = make_float2(coef, coef);
    if (BACKWARD) __syncthreads();
#pragma unroll 2
    for (int v = t; v < S.n_vecs; v += kDistillThreads) {
        constexpr int kP = kN / 2;
        float2 x[kP];
        V::unpack(reinterpret_cast<const uint4*>(slice)[v], x);
        if constexpr (BACKWARD) {
#pragma unroll
            for (int j = 0; j < kP; ++j)
                x[j] = make_float2(ex2(scaled_less(x[j].x, p.temperature, inv_tau, m_rest) * kLog2e),
                                   ex2(scaled_less(x[j].y, p.temperature, inv_tau, m_rest) * kLog2e));
        } else {
            at.apply(x, c2);
        }
#pragma unroll
        for (int j = 0; j < kP; ++j) x[j] = __fmul2_rn(kk, x[j]);
        if (vectors && S.whole(v)) {
            __stcs(reinterpret_cast<uint4*>(out) + v, V::pack(x));
        } else {
#pragma unroll
            for (int j = 0; j < kN; ++j) {
                const int s = v * kN + j;
                if (s >= S.begin && s < S.end) out[s] = V::from_f32(j & 1 ? x[j / 2].y : x[j / 2].x);
            }
        }
    }
    __syncthreads();
    // then the listed ones over the zeros left in their places
    if (listed >= 0) {
        const float log_q = BACKWARD ? scaled_less(own, p.temperature, inv_tau, m_all)
                                     : (own - m_all) * inv_tau - log_s;
        out[listed] = V::from_f32(none ? 0.0f : scale * (mass * expf(log_q) - expf(logp[t])));
    }
}

}  // namespace quasar
