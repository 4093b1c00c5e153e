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
// logit counts as -inf there), not as the difference of two sums.
//
// The row is passed over twice: the rest's sum of exponentials about a running
// maximum, then the gradient, from the row's end.  4096 x 131072 bf16 (a tenth
// of the rows padding) takes 372 us: 2.04 GB read and written at 5.5 TB/s, 0.81
// of the measured copy rate.  Of the second pass 0.2 GB comes from HBM again
// and the rest from L2, where the first pass asks for its lines to stay.
// Exponentials are the hardware's, about a base that loses nothing to rounding;
// every sum is fp32 and a bf16 gradient is rounded once.  The listed
// logits, k scattered elements, are read on the way.  A byte a vector in
// shared memory says which of its elements are listed; the four vectors a
// thread has in hand have theirs in one word.
#pragma once

#include "row_stream.cuh"

namespace quasar {

// x / tau - y: the quotient is not rounded before the subtraction (inv_tau is
// 1 / tau rounded, inv_low what that leaves out; x = -inf must not meet an
// inv_low of the other sign)
__device__ __forceinline__ float scaled_less(float x, float inv_tau, float inv_low, float y)
{
    const float d = fmaf(x, inv_tau, -y);
    return fmaf(fmaxf(x, -1e30f), inv_low, d);
}

// p log(p / q) - p + q from p, log p and log q (a NaN stays one)
__device__ __forceinline__ float kl_term(float p, float log_p, float log_q)
{
    if (p == 0.0f) return expf(log_q);
    const float d = log_p - log_q;
    return d > -1.0f ? p * (d + expm1f(-d)) : p * (d - 1.0f) + expf(log_q);
}

// Teacher side of a row, by one warp: log p of each entry replaces its value
// in logp[] (-inf where absent); returns sum p, NaN if the teacher is not a
// number anywhere: that must reach loss and gradient, not pass for no mass.
// A teacher_lse of -inf is that of a row without mass: not even the rest has
// any (`rest` says so).
__device__ __forceinline__ float teacher_side(const DistillParams& p, int64_t r, float inv_tau, float* logp, bool& rest)
{
    const int lane = threadIdx.x & 31;
    float norm;
    if (p.teacher_lse) {
        norm = p.teacher_lse[r];
    } else {
        float top = neg_inf();
        for (int k = lane; k < p.k; k += 32) top = fmaxf(top, logp[k] * inv_tau);
        top = lanes_max(top, 0xffffffffu);
        float s = 0.0f;
        for (int k = lane; k < p.k; k += 32) s += top == neg_inf() ? 0.0f : expf(logp[k] * inv_tau - top);
        s = warp_sum(s);
        norm = s == 0.0f ? 0.0f : top + logf(s);  // (NaN from a value that is NaN or infinite)
    }
    rest = p.teacher_lse && norm != neg_inf();
    float sum = 0.0f;
    for (int k = lane; k < p.k; k += 32) {
        const float z = logp[k] * inv_tau;
        logp[k] = z == neg_inf() && norm == neg_inf() ? z : z - norm;
        sum += expf(logp[k]);
    }
    return warp_sum(sum);
}

// BACKWARD: the gradient from kept statistics (log-sum-exp of z over the
// vocabulary and over the rest).  Otherwise the loss, the statistics and, if
// asked, the gradient.
template <typename T, int THREADS, bool BACKWARD>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) k_distill_top(const __grid_constant__ DistillParams p)
{
    using V = Vec16<T>;
    constexpr int kN = V::kN, kP = kN / 2;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    // a word for each thread's group: of its vectors, the listed elements
    uint32_t* mask = reinterpret_cast<uint32_t*>(smem_raw);
    const int mask_words = (p.row.vecs + kHand * THREADS - 1) / (kHand * THREADS) * THREADS;
    float* logp = reinterpret_cast<float*>(mask + mask_words);  // [kMaxTop]
    float* own = logp + kMaxTop;                              // the entries' student logits
    int32_t* entry = reinterpret_cast<int32_t*>(own + kMaxTop);  // -1: absent
    float* scratch = reinterpret_cast<float*>(entry + kMaxTop);  // [2][32]
    float* teacher = scratch + 64;                            // sum p, whether the rest may have mass
    float(*parts)[2] = reinterpret_cast<float(*)[2]>(teacher + 4);  // [kRowCtas]
    uint64_t* never = reinterpret_cast<uint64_t*>(parts + kRowCtas);  // nothing signals it: see quasar_debug_force_timeout
    int* n_listed = reinterpret_cast<int*>(never + 1);

    const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
    const int rank = p.row.ctas > 1 ? (int)(blockIdx.x % p.row.ctas) : 0;
    const int64_t r = blockIdx.x / p.row.ctas;
    const RowStream<T, THREADS> S(p.row, r, rank);
    const bool exchange = !BACKWARD && p.row.ctas > 1;
    wait_for_previous_grid();
    const float weight = p.row_weight ? p.row_weight[r] : 1.0f;
    T* grad = p.grad ? static_cast<T*>(p.grad) + r * p.ld_grad - S.begin : nullptr;  // of slot 0
    const bool vectors = (reinterpret_cast<uintptr_t>(grad) & 15) == 0;

    if (weight == 0.0f) {  // a row that counts nothing is not read
        if (grad)
            for (int v = S.v0 + t; v < S.v1; v += THREADS) {
                if (vectors && S.whole(v)) {
                    __stcs(reinterpret_cast<uint4*>(grad) + v, make_uint4(0, 0, 0, 0));
                } else {
                    for (int j = 0; j < kN; ++j)
                        if (S.holds((int64_t)v * kN + j)) grad[(int64_t)v * kN + j] = V::from_f32(0.0f);
                }
            }
        if (!BACKWARD && rank == 0 && t == 0) {
            p.loss[r] = 0.0f;
            if (p.stats) p.stats[2 * r] = p.stats[2 * r + 1] = 0.0f;
        }
        return;
    }

    if (exchange) cluster_arrive();
    uint4 raw[kHand];
    S.template load_group<!BACKWARD>(raw, 0);
    for (int w = t; w < mask_words; w += THREADS) mask[w] = 0;
    if (t == 0) *n_listed = 0;
    for (int k = t; k < p.k; k += THREADS) {
        const int32_t e = p.indices[r * p.k + k];
        const bool here = e >= 0 && e < p.row.vocab;
        entry[k] = here ? e : -1;
        logp[k] = here ? p.values[r * p.k + k] : neg_inf();
    }
    __syncthreads();
    const float inv_tau = 1.0f / p.temperature;
    const float inv_low = fmaf(-p.temperature, inv_tau, 1.0f) * inv_tau;
    const float c2 = kLog2e * inv_tau;
    // the student's logits of the entries are on their way during the first
    // pass (a backward call needs only its own share's: another CTA may already
    // have put the gradient in the place of the others)
    constexpr int kMine = kMaxTop / THREADS > 0 ? kMaxTop / THREADS : 1;
    T own_mine[kMine];
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
        const int k = q * THREADS + t;
        own_mine[q] = V::from_f32(neg_inf());
        if (k >= p.k || entry[k] < 0) continue;
        const int64_t s = (int64_t)S.begin + entry[k];
        const int v = (int)(s / kN) - S.v0;
        const bool held = v >= 0 && v < S.v1 - S.v0;
        if (!BACKWARD || held) own_mine[q] = load_one(S.slot0 + s);
        atomicAdd(n_listed, 1);
        if (held)  // vector v of the share is vector v / THREADS % kHand of a group of thread v % THREADS
            atomicOr(mask + v / (kHand * THREADS) * THREADS + v % THREADS,
                     1u << (v / THREADS % kHand * 8 + (int)(s % kN)));
    }
    if (warp == THREADS / 32 - 1) {
        bool rest;
        const float sum = teacher_side(p, r, inv_tau, logp, rest);
        if (lane == 0) {
            teacher[0] = sum;
            teacher[1] = rest ? 1.0f : 0.0f;
        }
    }
    if (t == 0 && p.row.force_timeout_ns) {
        mbar_init(never, 1);
        if (!mbar_wait_bounded(never, 0, p.row.force_timeout_ns)) record_timeout(p.row.status);
    }
    __syncthreads();
    const float sum_p = teacher[0];
    const float p_rest = teacher[1] != 0.0f && *n_listed < p.row.vocab ? max_nan(1.0f - sum_p, 0.0f) : 0.0f;
    const float mass = sum_p + p_rest;
    const int groups = S.groups();

    // -inf in the places of a vector's listed elements
    auto drop_from = [](uint4& x, unsigned listed) {
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int j = 0; j < kN; ++j)
            if (listed >> j & 1) V::put(w, j, V::from_f32(neg_inf()));
        x = make_uint4(w[0], w[1], w[2], w[3]);
    };
    auto drop_group = [=](uint4 (&x)[kHand], int g) {
        const uint32_t listed = mask[g * THREADS + t];
        if (listed) {
#pragma unroll
            for (int u = 0; u < kHand; ++u) drop_from(x[u], listed >> 8 * u);
        }
    };
    auto drop = [=](uint4& x, int g, int u) { drop_from(x, mask[g * THREADS + t] >> 8 * u); };

    auto put_own = [&] {
#pragma unroll
        for (int q = 0; q < kMine; ++q)
            if (q * THREADS + t < p.k) own[q * THREADS + t] = V::to_f32(own_mine[q]);
    };

    float m_rest, coef, q_rest;  // of the whole row (backward: m_rest is the rest's lse)
    float m_all, log_s = 0.0f;   // lse = m_all / tau + log_s (backward: lse = m_all)
    bool nothing;                // every logit is -inf (a NaN beside them shows in the sum alone)
    if constexpr (!BACKWARD) {
        RunningSum run;
        for (int g = 0; g < groups; ++g) {
            uint4 next[kHand];
            if (g + 1 < groups) S.template load_group<!BACKWARD>(next, g + 1);
            drop_group(raw, g);
            typename V::Max top = V::larger(raw[0]);
#pragma unroll
            for (int u = 1; u < kHand; ++u) top = V::larger(top, V::larger(raw[u]));
            run.template add<T>(raw, top, c2);
            if (g + 1 < groups) {
#pragma unroll
                for (int u = 0; u < kHand; ++u) raw[u] = next[u];
            }
        }
        // (the last group stays in hand for the second pass)
        float s_rest;
        put_own();
        block_sum<THREADS>(run, c2, scratch, m_rest, s_rest);
        // the listed entries' own sum of exponentials, by every warp
        float m_in = neg_inf(), s_in = 0.0f;
        for (int k = lane; k < p.k; k += 32) m_in = fmaxf(m_in, own[k]);
        m_in = lanes_max(m_in, 0xffffffffu);
        for (int k = lane; k < p.k; k += 32) s_in += own[k] == neg_inf() ? 0.0f : exp2f((own[k] - m_in) * c2);
        s_in = warp_sum(s_in);
        if (is_far(m_rest, c2)) s_rest = far_sum(S, m_rest, c2, scratch, drop);
        if (exchange) {
            cluster_wait();  // every CTA of the row has started: its shared memory may be written
            if (t < p.row.ctas) {
                const uint32_t to = peer_addr(smem_u32(&parts[rank][0]), (uint32_t)t);
                st_peer(to, m_rest);
                st_peer(to + 4, s_rest);
            }
            cluster_sync();
            m_rest = neg_inf();
            s_rest = 0.0f;
            for (int c = 0; c < p.row.ctas; ++c) merge_sum(m_rest, s_rest, parts[c][0], parts[c][1], c2);
        }
        m_all = m_rest;
        float s_all = s_rest;
        merge_sum(m_all, s_all, m_in, s_in, c2);
        log_s = isinf(s_all) ? s_all - s_all : logf(s_all);  // (softmax of a +inf logit is NaN)
        nothing = m_all == neg_inf() && s_all == 0.0f;
        const bool some = m_rest != neg_inf() || s_rest != 0.0f;
        const float log_q_rest = some ? (m_rest - m_all) * inv_tau + (logf(s_rest) - log_s) : neg_inf();
        q_rest = expf(log_q_rest);
        coef = some ? (mass * q_rest - p_rest) / s_rest : (s_all == s_all ? 0.0f * mass : s_all);
        if (rank == 0 && warp == 0) {
            float loss = 0.0f;
            for (int k = lane; k < p.k; k += 32)
                if (entry[k] >= 0) loss += kl_term(expf(logp[k]), logp[k], (own[k] - m_all) * inv_tau - log_s);
            loss = warp_sum(loss);
            if (lane == 0) {
                loss += kl_term(p_rest, logf(p_rest), log_q_rest);
                if (nothing) loss = mass + __int_as_float(0x7F800000);  // q is 0 everywhere
                p.loss[r] = mass == 0.0f ? 0.0f : loss;
                if (p.stats) {
                    p.stats[2 * r] = m_all / p.temperature + log_s;
                    p.stats[2 * r + 1] = some ? m_rest / p.temperature + logf(s_rest) : neg_inf();
                }
            }
        }
        if (!grad) return;
    } else {
        m_all = p.stats[2 * r];
        nothing = m_all == neg_inf();
        const float lse_rest = p.stats[2 * r + 1];
        const bool some = lse_rest != neg_inf();
        q_rest = some ? expf(lse_rest - m_all) : 0.0f;
        coef = some ? mass * q_rest - p_rest : (m_all == m_all ? 0.0f * mass : m_all);
        m_rest = some ? lse_rest : 0.0f;
    }
    // a row without teacher mass, or without a finite logit, has no gradient
    const bool none = mass == 0.0f || (nothing && mass == mass);
    const float scale = none ? 0.0f : weight * inv_tau;
    coef = none ? 0.0f : coef * scale;

    // the unlisted entries: coef 2^(x c - base), or coef e^(z - lse) from kept
    // statistics
    const float base = m_rest == neg_inf() ? 0.0f : exp_base(m_rest, c2);
    const bool far = !BACKWARD && fabsf(base) == kFar;  // the subtraction first: see exp_base
    if (!BACKWARD && !far) coef *= m_rest == neg_inf() ? 1.0f : exp_fix(m_rest, c2, base);
    const float2 cc = make_float2(c2, c2), bb = make_float2(far ? 0.0f : -base, far ? 0.0f : -base),
                 kk = make_float2(coef, coef);
    // from the end of the row: what was read last is the likeliest to be in L2
    if (BACKWARD) {
        put_own();
        if (groups > 1) S.load_group(raw, groups - 1);
    }
    for (int g = groups - 1; g >= 0; --g) {
        uint4 next[kHand];
        if (g > 0) S.load_group(next, g - 1);
        if (BACKWARD || far) drop_group(raw, g);
        const bool whole = vectors && S.whole_group(g);
        uint4* to = reinterpret_cast<uint4*>(grad) + S.vec(g, 0);
#pragma unroll
        for (int u = 0; u < kHand; ++u) {
            float2 x[kP];
            V::unpack(raw[u], x);
            if constexpr (BACKWARD) {
                // scaled_less, two at a time
#pragma unroll
                for (int j = 0; j < kP; ++j) {
                    const float2 z = x[j];
                    x[j] = __ffma2_rn(z, make_float2(inv_tau, inv_tau), make_float2(-m_rest, -m_rest));
                    if (inv_low != 0.0f)
                        x[j] = __ffma2_rn(make_float2(fmaxf(z.x, -1e30f), fmaxf(z.y, -1e30f)),
                                          make_float2(inv_low, inv_low), x[j]);
                    x[j] = __fmul2_rn(x[j], make_float2(kLog2e, kLog2e));
                    x[j] = make_float2(ex2(x[j].x), ex2(x[j].y));
                }
            } else {
                if (far) {
#pragma unroll
                    for (int j = 0; j < kP; ++j) x[j] = __fadd2_rn(x[j], make_float2(-m_rest, -m_rest));
                }
#pragma unroll
                for (int j = 0; j < kP; ++j) {
                    x[j] = __ffma2_rn(x[j], cc, bb);
                    x[j] = make_float2(ex2(x[j].x), ex2(x[j].y));
                }
            }
#pragma unroll
            for (int j = 0; j < kP; ++j) x[j] = __fmul2_rn(kk, x[j]);
            if (whole) {
                __stcs(to + u * THREADS, V::pack(x));
            } else {
                const int v = S.vec(g, u);
                if (v >= S.v1) continue;
                if (vectors && S.whole(v)) {
                    __stcs(to + u * THREADS, V::pack(x));
                    continue;
                }
#pragma unroll
                for (int j = 0; j < kN; ++j) {
                    const int64_t s = (int64_t)v * kN + j;
                    if (S.holds(s)) grad[s] = V::from_f32(j & 1 ? x[j / 2].y : x[j / 2].x);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kHand; ++u) raw[u] = next[u];
    }
    __syncthreads();
    // then the listed ones over what was left in their places
    for (int k = t; k < p.k; k += THREADS) {
        if (entry[k] < 0) continue;
        const int64_t s = (int64_t)S.begin + entry[k];
        if (s / kN < S.v0 || s / kN >= S.v1) continue;
        const float log_q = BACKWARD ? scaled_less(own[k], inv_tau, inv_low, m_all)
                                     : (own[k] - m_all) * inv_tau - log_s;
        grad[s] = V::from_f32(none ? 0.0f : scale * (mass * expf(log_q) - expf(logp[k])));
    }
}

}  // namespace quasar
