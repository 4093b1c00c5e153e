// The gradients of attention.  With p = exp(scale s - lse) made again from q,
// k and the row's log-sum-exp, and D the row's sum of dy y:
//
//   dv = p^T dy,   dp = dy v^T,   ds = p (dp - D)
//   dq = scale ds k,   dk = scale ds^T q
//
// Two kernels of one form, so that every sum has one owner and one order (no
// atomics, no second copy of dq): 128 rows stay in shared memory, the other
// side streams past in steps of 64 columns, and the gradients of the rows grow
// in tensor memory.
//
//   keys stay:    S = K Q^T, dP = V dY^T (transposed scores), dv += P dY, dk += dS Q
//   queries stay: S = Q K^T, dP = dY V^T,                      dq += dS K
//
// S and dP are made twice, 7 products where 5 would do; what a single kernel
// would need besides is fp32 additions to dq in memory from every key tile, in
// an order that timing decides.
//
// Rows and columns of queries are (token, head) pairs, the heads that share keys
// side by side, so dk and dv of shared keys are one sum over all of their heads.
// P and dS go through tensor memory as bf16, in the place of S and dP: each is
// rounded once for its matrix product (2^-8 of it), sums are fp32.
//
// Warps: 0-7 and 8-15 make P and dS of every other step, two threads a row (with
// one, their dependent instructions took 2,700 cycles a step, and 4 x 4096
// causal, 32 heads of 128 over 8, 1815 us in all); 16 copies, 17 and 18 matrix
// instructions (S and dv; dP and dk or dq), 19 brings the columns' statistics
// (keys stay).
// Tensor memory: two gradients of 128 columns, S and dP twice of 64.
#pragma once

#include "attention.cuh"

namespace quasar {

constexpr int kGradThreads = 640;
constexpr int kGradCopies = 16, kGradProducts = 17, kGradStats = 19;  // warps (of products two)
constexpr int kGradSlots = 4;

// The rows' statistics: 8 or 16 threads a (token, head) pair.
template <int LANES>
__global__ void __launch_bounds__(256) k_attention_stats(const __grid_constant__ AttnStatsParams p)
{
    wait_for_previous_grid();
    const int64_t pairs = p.tokens * p.heads;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;
    const int c = threadIdx.x % LANES;
    float sum = 0.0f;
    const int64_t token = at / p.heads;
    const int head = (int)(at % p.heads);
    if (at < pairs && 8 * c < p.d) {
        const int64_t col = (int64_t)head * p.d + 8 * c;
        const uint4 a = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.dy) + token * p.ld_dy + col);
        const uint4 b = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.y) + token * p.ld_y + col);
        const uint32_t aw[4] = {a.x, a.y, a.z, a.w}, bw[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            sum = fmaf(bf16lo(aw[i]), bf16lo(bw[i]), sum);
            sum = fmaf(bf16hi(aw[i]), bf16hi(bw[i]), sum);
        }
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (at < pairs && c == 0) {
        // (a row without keys: p = exp2(s - inf) = 0)
        const float lse = p.lse[at];
        p.stats[at] = make_float2(lse == minus_inf() ? -minus_inf() : lse * 1.44269504f, sum);
    }
}

template <int DB, bool KEYS>
__global__ void __launch_bounds__(kGradThreads, 1) k_attention_grad(const __grid_constant__ AttnGradParams p)
{
    constexpr int D = 64 * DB;
    constexpr uint32_t kRowTile = DB * kAttnBlock;        // bytes of the rows' x1 or x2
    constexpr uint32_t kColBlock = kGradCols * 128;
    constexpr uint32_t kColTile = DB * kColBlock;         // of a step's z1 or z2
    constexpr uint32_t kSlot = 2 * kColTile;
    constexpr uint32_t kAcc2 = 128, kScores = 256, kDp = 384;  // columns of tensor memory
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring = smem + 2 * kRowTile;
    float2* col_stats = reinterpret_cast<float2*>(ring + kGradSlots * kSlot);  // [slots][64]
    uint64_t* x_full = reinterpret_cast<uint64_t*>(col_stats + kGradSlots * kGradCols);
    uint64_t* full = x_full + 1;               // [slots]
    uint64_t* empty = full + kGradSlots;       // [slots]
    uint64_t* stat_full = empty + kGradSlots;  // [slots]
    uint64_t* s_full = stat_full + kGradSlots; // [2]
    uint64_t* p_full = s_full + 2;             // [2]: 8 warps
    uint64_t* acc_full = p_full + 2;
    uint64_t* never = acc_full + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(never + 1);
    volatile uint32_t* gone = tmem_slot + 1;
    AttnItem* item = reinterpret_cast<AttnItem*>(tmem_slot + 2);

    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int kvh = (int)blockIdx.x % p.kv_heads;

    if (threadIdx.x == 0) {
        mbar_init(x_full, 1);
        for (int s = 0; s < kGradSlots; ++s) {
            mbar_init(full + s, 1);
            mbar_init(empty + s, 2);
            mbar_init(stat_full + s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(s_full + b, 2);
            mbar_init(p_full + b, 8);
        }
        mbar_init(acc_full, 2);
        mbar_init(never, 1);
        *gone = 0;
        mbar_init_fence();
    }
    if (warp == kGradProducts) tmem_alloc<1>(tmem_slot, 512);
    if (warp == kGradCopies && lane == 0) {
        prefetch_map(&p.x1);
        prefetch_map(&p.x2);
        prefetch_map(&p.z1);
        prefetch_map(&p.z2);
    }
    wait_for_previous_grid();
    if (warp == 0) {
        const AttnItem a = find_item(p.s, (int)blockIdx.x / p.kv_heads, p.items, KEYS ? kAttnRows : p.tile_tokens, KEYS);
        if (lane == 0) *item = a;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = uniform(*tmem_slot);
    const AttnItem a = *item;
    const int row0 = a.index * (KEYS ? kAttnRows : p.tile_tokens);  // first key, or token, of the rows
    const int shift = a.m - a.n;                                    // key j is seen by tokens from j - shift on

    // Steps.  Keys stay: for each run of box_heads heads the tokens from the
    // first that sees a key of the tile.  Queries stay: the keys that the last
    // token sees.
    int per_run = 0, runs = 1, step0 = 0;
    if (a.spares == 0) {
        if (KEYS) {
            const int64_t sees = p.causal ? max((int64_t)0, (int64_t)row0 - shift) : 0;
            if (sees < a.n) {
                step0 = (int)(sees / p.step_tokens);
                per_run = (a.n + p.step_tokens - 1) / p.step_tokens - step0;
            }
            runs = p.group / p.box_heads;
        } else {
            const int last = min(row0 + p.tile_tokens, a.n) - 1;
            const int64_t see = p.causal ? min((int64_t)a.m, (int64_t)last + 1 + shift) : a.m;
            per_run = see > 0 ? (int)((see + kGradCols - 1) / kGradCols) : 0;
        }
    }
    const int steps = uniform(per_run * runs);  // (at most tokens x heads, or keys: checked by the host)
    // A walk over the steps: their first token (or key) and run, without a
    // division a step.
    struct Walk {
        int first, run, begin, end, by;
        __device__ void next()
        {
            first += by;
            if (first >= end) first = begin, ++run;
        }
    };
    const Walk walk{KEYS ? step0 * p.step_tokens : 0, 0, KEYS ? step0 * p.step_tokens : 0, KEYS ? a.n : a.m,
                    KEYS ? p.step_tokens : kGradCols};
    // columns of a step that are the sequence's
    auto cols_of = [&](const Walk& w) {
        return KEYS ? min(p.step_tokens, a.n - w.first) * p.box_heads : min(kGradCols, a.m - w.first);
    };

    if (warp == kGradCopies) {
        if (lane == 0) {
            if (p.force_timeout_ns) role_sleep(never, 0, gone, p.force_timeout_ns, p.status);
            int it = 0;
            const bool rows_sent = steps > 0 && !*gone;
            if (rows_sent) {
                const uint32_t rows = KEYS ? kAttnRows : (uint32_t)(p.tile_tokens * p.group);
                mbar_arrive_expect_tx(x_full, 2 * rows * 128 * DB);
                for (int x = 0; x < 2; ++x)
                    for (int b = 0; b < DB; ++b)
                        tile_g2s_3d(smem_u32(smem + x * kRowTile + b * kAttnBlock), x ? &p.x2 : &p.x1, 64 * b,
                                    KEYS ? kvh : kvh * p.group, (KEYS ? a.k0 : a.q0) + row0, smem_u32(x_full));
            }
            const uint32_t bytes = 2 * DB * 128 * (KEYS ? (uint32_t)(p.step_tokens * p.box_heads) : kGradCols);
            Walk w = walk;
            for (; it < steps && !*gone; ++it, w.next()) {
                const int s = it % kGradSlots;
                if (it >= kGradSlots && !role_sleep(empty + s, (it / kGradSlots - 1) & 1, gone, p.timeout_ns, p.status))
                    break;
                mbar_arrive_expect_tx(full + s, bytes);
                for (int z = 0; z < 2; ++z)
                    for (int b = 0; b < DB; ++b)
                        tile_g2s_3d(smem_u32(ring + s * kSlot + z * kColTile + b * kColBlock), z ? &p.z2 : &p.z1, 64 * b,
                                    KEYS ? kvh * p.group + w.run * p.box_heads : kvh,
                                    (KEYS ? a.q0 : a.k0) + w.first, smem_u32(full + s));
            }
            if (*gone) {  // what is in flight has landed before the memory is let go
                if (rows_sent) mbar_wait_bounded(x_full, 0, p.timeout_ns);
                for (int j = max(it - kGradSlots, 0); j < it; ++j)
                    mbar_wait_bounded(full + j % kGradSlots, (j / kGradSlots) & 1, p.timeout_ns);
            }
        }
    } else if (warp - kGradProducts == 0 || warp - kGradProducts == 1) {
        // g = 0: S = X1 Z1^T and, with P in its place, acc2 += P Z2;
        // g = 1: dP = X2 Z2^T and, with dS in its place, acc1 += dS Z1
        constexpr uint32_t desc_s = mma_desc(kAttnRows, kGradCols, false, false);
        constexpr uint32_t desc_acc = mma_desc(kAttnRows, D, false, true);
        const int g = warp - kGradProducts;
        const uint32_t scores = tmem + (g ? kDp : kScores), acc = tmem + (g ? 0 : kAcc2);
        auto wait = [&](uint64_t* bar, uint32_t parity) {
            const bool ok = role_sleep(bar, parity, gone, p.timeout_ns, p.status);
            return __all_sync(0xffffffffu, ok);
        };
        // the gradient grows by step `it`
        auto grow = [&](int it) {
            if (elect_one()) {
                const int s = it % kGradSlots;
                if (KEYS || g == 1) {
                    const uint64_t db = operand_desc(smem_u32(ring + s * kSlot) + (g ? 0 : kColTile), true);
                    const uint32_t p_at = scores + (it & 1) * 64;
#pragma unroll
                    for (int x = 0; x < kGradCols / 16; ++x)
                        mma_bf16_ts(acc, p_at + x / 2 * 32 + x % 2 * 8, db + x * k_step(true), desc_acc, it > 0 || x > 0);
                }
                mma_commit(smem_u32(empty + s));
            }
            __syncwarp();
        };
        bool ok = steps == 0 || wait(x_full, 0);
        Walk w = walk;
        for (int it = 0; it < steps && ok; ++it, w.next()) {
            const int s = it % kGradSlots, buf = it & 1;
            if (!(ok = wait(full + s, (it / kGradSlots) & 1))) break;
            // columns behind the sequence belong to another, or to nobody: zeros
            // (both warps write them, each before its own reads)
            const int cols = cols_of(w);
            if (cols < kGradCols) {
                for (int x = lane + cols * 8; x < kGradCols * 8; x += 32)
#pragma unroll
                    for (int b = 0; b < 2 * DB; ++b)
                        *reinterpret_cast<uint4*>(ring + s * kSlot + b * kColBlock + x * 16) = make_uint4(0, 0, 0, 0);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            tc_fence_after();
            if (elect_one()) {
                const uint32_t x = smem_u32(smem + g * kRowTile), z = smem_u32(ring + s * kSlot + g * kColTile);
#pragma unroll
                for (int b = 0; b < DB; ++b) {
                    const uint64_t da = operand_desc(x + b * kAttnBlock, false), db = operand_desc(z + b * kColBlock, false);
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        mma_bf16<1>(scores + buf * 64, da + y * k_step(false), db + y * k_step(false), desc_s, b + y > 0);
                }
                mma_commit(smem_u32(s_full + buf));
            }
            __syncwarp();
            if (it > 0) {
                if (!(ok = wait(p_full + (buf ^ 1), ((it - 1) / 2) & 1))) break;
                tc_fence_after();
                grow(it - 1);
            }
        }
        if (steps > 0 && ok && (ok = wait(p_full + ((steps - 1) & 1), ((steps - 1) / 2) & 1))) {
            tc_fence_after();
            grow(steps - 1);
        }
        if (elect_one()) {  // every instruction is done before the memory is let go
            mma_commit(smem_u32(acc_full));
            mbar_wait_bounded(acc_full, 0, p.timeout_ns);
        }
    } else if (warp == kGradStats) {
        if (KEYS) {
            Walk w = walk;
            const int place[2] = {lane / p.box_heads * p.heads + lane % p.box_heads,
                                  (lane + 32) / p.box_heads * p.heads + (lane + 32) % p.box_heads};
            for (int it = 0; it < steps; ++it, w.next()) {
                const int s = it % kGradSlots, cols = cols_of(w);
                const int64_t at = (int64_t)(a.q0 + w.first) * p.heads + kvh * p.group + w.run * p.box_heads;
                float2 st[2];
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int c = lane + 32 * q;  // behind the sequence: p = 0
                    st[q] = c < cols ? p.stats[at + place[q]]
                                     : make_float2(-minus_inf(), 0.0f);
                    st[q] = make_float2(-st[q].x, -st[q].y);  // (as they are added)
                }
                bool ok = it < kGradSlots || role_sleep(empty + s, (it / kGradSlots - 1) & 1, gone, p.timeout_ns, p.status);
                ok = __all_sync(0xffffffffu, ok && !*gone);
                if (!ok) break;
#pragma unroll
                for (int q = 0; q < 2; ++q) col_stats[s * kGradCols + lane + 32 * q] = st[q];
                __syncwarp();
                if (lane == 0) mbar_arrive(stat_full + s);
            }
        }
    } else {
        // turn: of every other step; half: of its columns, whose P and dS lie where
        // this half of S and dP lay
        const int turn = warp >> 3, half = warp >> 2 & 1, r = (warp & 3) * 32 + lane;
        const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        // the row: key row0 + r, or (token, head)
        const int token = row0 + r / p.group, head = kvh * p.group + r % p.group;
        const bool live = a.spares == 0 && (KEYS ? row0 + r < a.m : r < p.tile_tokens * p.group && token < a.n);
        const bool any_live = __any_sync(0xffffffffu, live);
        float2 own = make_float2(minus_inf(), 0.0f);  // both negative
        if (!KEYS && live) {
            own = p.stats[(int64_t)(a.q0 + token) * p.heads + head];
            own = make_float2(-own.x, -own.y);
        }
        // of the sequence's columns, the first that sees the row's key; the last
        // key that the row's token sees
        const int64_t from = KEYS && p.causal ? (int64_t)row0 + r - shift : 0;
        const int64_t upto = p.causal ? min((int64_t)a.m - 1, (int64_t)token + shift) : (int64_t)a.m - 1;
        bool ok = true;
        Walk w = walk;
        if (turn) w.next();
        for (int it = turn; it < steps; it += 2, w.next(), w.next()) {
            const int s = it % kGradSlots;
            ok = role_sleep(s_full + turn, (it / 2) & 1, gone, p.timeout_ns, p.status);
            if (KEYS && ok) ok = role_sleep(stat_full + s, (it / kGradSlots) & 1, gone, p.timeout_ns, p.status);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            if (any_live) {
                const uint32_t s_at = mine + kScores + turn * 64 + half * 32, dp_at = mine + kDp + turn * 64 + half * 32;
                // the columns [lo, hi] of this half that the row sees (or that see it)
                int lo = 0, hi = 31;
                const int f = w.first;
                if (KEYS && p.causal)
                    lo = (int)max((int64_t)0, min((int64_t)32, (from - f) * p.box_heads - half * 32));
                if (!KEYS) hi = (int)max((int64_t)-1, min((int64_t)31, upto - f - half * 32));
                const bool masked = !__all_sync(0xffffffffu, lo == 0 && hi == 31);
                const float2* st = col_stats + s * kGradCols + half * 32;
                const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float sc[16], dp[16];
                    tmem_ld(s_at + 16 * h, sc);
                    tmem_ld(dp_at + 16 * h, dp);
                    tmem_wait_ld(sc);
                    tmem_wait_ld(dp);
                    uint32_t pw[8], dw[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        float2 lse = make_float2(own.x, own.x), delta = make_float2(own.y, own.y);
                        if (KEYS) {
                            const float4 two = *reinterpret_cast<const float4*>(st + 16 * h + 2 * x);
                            lse = make_float2(two.x, two.z);
                            delta = make_float2(two.y, two.w);
                        }
                        float2 e = __ffma2_rn(make_float2(sc[2 * x], sc[2 * x + 1]), scale2, lse);
                        e.x = exp2_fast(e.x);
                        e.y = exp2_fast(e.y);
                        float2 ds = __fmul2_rn(e, __fadd2_rn(make_float2(dp[2 * x], dp[2 * x + 1]), delta));
                        if (masked) {
                            const int c = 16 * h + 2 * x;
                            if (c < lo || c > hi) e.x = 0.0f, ds.x = 0.0f;
                            if (c + 1 < lo || c + 1 > hi) e.y = 0.0f, ds.y = 0.0f;
                        }
                        pw[x] = pack_bf16x2(e.x, e.y);
                        dw[x] = pack_bf16x2(ds.x, ds.y);
                    }
                    // (columns that this thread has read)
                    if (KEYS) tmem_st(s_at + 8 * h, pw);
                    tmem_st(dp_at + 8 * h, dw);
                }
                tmem_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full + turn);
        }
        if (ok && steps > 0) {
            ok = role_sleep(acc_full, 0, gone, p.timeout_ns, p.status) && !*gone;
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
        }
        // dk or dq by warps 0-7, dv by warps 8-15, half of the columns each,
        // through the rows' memory so that a store covers whole rows
        if (ok && any_live && (KEYS || turn == 0)) {
            constexpr int kHalf = D / 2;
            const float scale = turn == 0 ? p.scale : 1.0f;
            uint8_t* stage = smem + turn * kRowTile + (warp & 3) * 32 * D * 2;
#pragma unroll 1
            for (int c = half * kHalf; c < (half + 1) * kHalf; c += 32) {
                float o[32];
                if (steps > 0) {
                    tmem_ld(mine + turn * kAcc2 + c, o);
                    tmem_wait_ld(o);
                } else {
#pragma unroll
                    for (int x = 0; x < 32; ++x) o[x] = 0.0f;
                }
#pragma unroll
                for (int x = 0; x < 32; x += 8)
                    *reinterpret_cast<uint4*>(stage + lane * D * 2 + (((c + x) / 8) ^ (lane & 7)) * 16) =
                        make_uint4(pack_bf16x2(o[x] * scale, o[x + 1] * scale), pack_bf16x2(o[x + 2] * scale, o[x + 3] * scale),
                                   pack_bf16x2(o[x + 4] * scale, o[x + 5] * scale), pack_bf16x2(o[x + 6] * scale, o[x + 7] * scale));
            }
            __syncwarp();
            constexpr int kLanes = kHalf / 8;  // of a row
            __nv_bfloat16* const out = static_cast<__nv_bfloat16*>(turn == 0 ? p.d1 : p.d2);
            const int64_t ld = turn == 0 ? p.ld_d1 : p.ld_d2;
            for (int q = 0; q < 32; q += 32 / kLanes) {
                const int row = q + lane / kLanes, chunk = half * kLanes + lane % kLanes;
                const int rr = (warp & 3) * 32 + row;
                int64_t at;
                bool in = chunk * 8 < p.d;
                if (KEYS) {
                    in = in && row0 + rr < a.m;
                    at = (int64_t)(a.k0 + row0 + rr) * ld + (int64_t)kvh * p.d;
                } else {
                    const int tok = row0 + rr / p.group;
                    in = in && rr < p.tile_tokens * p.group && tok < a.n;
                    at = (int64_t)(a.q0 + tok) * ld + (int64_t)(kvh * p.group + rr % p.group) * p.d;
                }
                if (in)
                    *reinterpret_cast<uint4*>(out + at + chunk * 8) =
                        *reinterpret_cast<const uint4*>(stage + row * D * 2 + (chunk ^ (row & 7)) * 16);
            }
        }
    }
    if (a.spares > 0) {
        if (KEYS) {
            clear_rows(p.d1, p.ld_d1, (int64_t)kvh * p.d, p.d, p.s.key_starts, p.s.n, p.s.keys, a.index, a.spares,
                       threadIdx.x, kGradThreads);
            clear_rows(p.d2, p.ld_d2, (int64_t)kvh * p.d, p.d, p.s.key_starts, p.s.n, p.s.keys, a.index, a.spares,
                       threadIdx.x, kGradThreads);
        } else {
            clear_rows(p.d1, p.ld_d1, (int64_t)kvh * p.group * p.d, p.group * p.d, p.s.starts, p.s.n, p.s.tokens, a.index,
                       a.spares, threadIdx.x, kGradThreads);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kGradProducts) tmem_free<1>(tmem, 512);
}

}  // namespace quasar
