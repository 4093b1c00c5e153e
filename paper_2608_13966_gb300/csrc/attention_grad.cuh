// The gradients of attention.  With p = exp(scale s - lse) made again from q,
// k and the row's log-sum-exp, and D the row's sum of dy y:
//
//   dv = p^T dy,   dp = dy v^T,   ds = p (dp - D)
//   dq = scale ds k,   dk = scale ds^T q
//
// Two kernels of one form, so that every sum has one owner and one order (no
// atomics, no second copy of dq): 128 rows stay in shared memory, the other
// side streams past in steps of 128 columns, and the gradients of the rows grow
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
// The matrix instructions are one thread's, in an order that leaves the rows'
// warps the time of two products for P and as long for dS:
//
//   keys stay:    dv(j), S(j+1), dk(j), dP(j+1)
//   queries stay: S(j+1), dP(j+1), dq(j)          (dP in two places in turn)
//
// (In steps of 64 columns, S and dP of two steps at a time, the tensor cores'
// reading of shared memory took 1.26 as long and the chain of a step was not
// hidden: 4 x 4096 causal, 32 heads of 128 over 8, 1710 us.)
//
// Warps: 0-15 make P and dS, four threads a row; 16 copies, 17 matrix
// instructions, 18 brings the columns' statistics (keys stay).
#pragma once

#include "attention.cuh"

namespace quasar {

constexpr int kGradThreads = 608;
constexpr int kGradRowWarps = 16, kGradCopies = 16, kGradProducts = 17, kGradStats = 18;  // warps
constexpr int kGradSlots1 = 3, kGradSlots2 = 2;  // of the rings of z1 (which waits for the step's end) and z2

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

__host__ __device__ constexpr size_t attention_grad_bytes(int blocks)
{
    return (size_t)(2 + kGradSlots1 + kGradSlots2) * blocks * kAttnBlock + 2 * kGradCols * 8 +
           (1 + 2 * kGradSlots1 + 2 * kGradSlots2 + 2 * 2 + 2 + 2 + 1) * 8 + sizeof(AttnItem) + 8;
}

template <int DB, bool KEYS>
__global__ void __launch_bounds__(kGradThreads, 1) k_attention_grad(const __grid_constant__ AttnGradParams p)
{
    constexpr int D = 64 * DB;
    constexpr uint32_t kTile = DB * kAttnBlock;  // bytes of 128 rows
    // columns of tensor memory: the gradients from 0 (and 128), the scores, dP
    constexpr uint32_t kAcc2 = 128, kScores = KEYS ? 256 : 128;
    auto dp_at = [](int j) { return KEYS ? 384u : 256u + (j & 1) * 128u; };
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring1 = smem + 2 * kTile;
    uint8_t* ring2 = ring1 + kGradSlots1 * kTile;
    float* col_stats = reinterpret_cast<float*>(ring2 + kGradSlots2 * kTile);  // [2][lse, D][128], negative
    uint64_t* x_full = reinterpret_cast<uint64_t*>(col_stats + 4 * kGradCols);
    uint64_t* full1 = x_full + 1;               // [slots1]
    uint64_t* empty1 = full1 + kGradSlots1;
    uint64_t* full2 = empty1 + kGradSlots1;     // [slots2]
    uint64_t* empty2 = full2 + kGradSlots2;
    uint64_t* stat_full = empty2 + kGradSlots2; // [2]
    uint64_t* dp_full = stat_full + 2;          // [2]
    uint64_t* ds_full = dp_full + 2;            // [2]: the rows' warps
    uint64_t* s_full = ds_full + 2;
    uint64_t* p_full = s_full + 1;              // the rows' warps: the scores are read, P is in their place
    uint64_t* acc_full = p_full + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acc_full + 1);
    volatile uint32_t* gone = tmem_slot + 1;
    AttnItem* item = reinterpret_cast<AttnItem*>(tmem_slot + 2);

    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int kvh = (int)blockIdx.x % p.kv_heads;

    uint32_t given;
    asm volatile("mov.u32 %0, %%dynamic_smem_size;" : "=r"(given));
    if (smem + attention_grad_bytes(DB) > smem_raw + given) {  // (it starts at a multiple of 1024, as declared)
        if (threadIdx.x == 0) record_timeout(p.status);
        return;
    }
    if (threadIdx.x == 0) {
        mbar_init(x_full, 1);
        for (int s = 0; s < 2 * kGradSlots1 + 2 * kGradSlots2; ++s) mbar_init(full1 + s, 1);
        for (int b = 0; b < 2; ++b) {
            mbar_init(stat_full + b, 1);
            mbar_init(dp_full + b, 1);
            mbar_init(ds_full + b, kGradRowWarps);
        }
        mbar_init(s_full, 1);
        mbar_init(p_full, kGradRowWarps);
        mbar_init(acc_full, 1);
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

    // Steps.  Keys stay: the tokens from the first that sees a key of the tile.
    // Queries stay: the keys that the last token sees.
    const int by = KEYS ? p.tile_tokens : kGradCols;  // tokens, or keys, of a step
    int begin = 0, end = 0;                           // of the sequence's tokens, or keys
    if (a.spares == 0) {
        if (KEYS) {
            const int64_t sees = p.causal ? max((int64_t)0, (int64_t)row0 - shift) : 0;
            if (sees < a.n) begin = (int)sees / by * by, end = a.n;
        } else {
            const int64_t last = min((int64_t)row0 + p.tile_tokens, (int64_t)a.n) - 1;
            end = (int)max((int64_t)0, p.causal ? min((int64_t)a.m, last + 1 + shift) : (int64_t)a.m);
        }
    }
    const int steps = uniform((end - begin + by - 1) / by);
    const int limit = KEYS ? a.n : a.m;  // columns behind it are not the sequence's
    auto cols_of = [&](int j) { return KEYS ? min(by, limit - begin - j * by) * p.group : min(by, limit - j * by); };
    auto wait = [&](uint64_t* bar, uint32_t parity) {  // the warp's, with one outcome
        const bool ok = role_sleep(bar, parity, gone, p.timeout_ns, p.status);
        return __all_sync(0xffffffffu, ok);
    };

    if (warp == kGradCopies) {
        if (lane == 0) {
            // (no copy asked for: nothing else goes on)
            if (p.force_timeout_ns) role_sleep(acc_full, 0, gone, p.force_timeout_ns, p.status);
            int sent1 = 0, sent2 = 0;
            const bool rows_sent = steps > 0 && !*gone;
            if (rows_sent) {
                const uint32_t rows = KEYS ? kAttnRows : (uint32_t)(p.tile_tokens * p.group);
                mbar_arrive_expect_tx(x_full, 2 * rows * 128 * DB);
                for (int x = 0; x < 2; ++x)
                    for (int b = 0; b < DB; ++b)
                        tile_g2s_3d(smem_u32(smem + x * kTile + b * kAttnBlock), x ? &p.x2 : &p.x1, 64 * b,
                                    KEYS ? kvh : kvh * p.group, (KEYS ? a.k0 : a.q0) + row0, smem_u32(x_full));
            }
            const uint32_t bytes = DB * 128 * (KEYS ? (uint32_t)(p.tile_tokens * p.group) : kGradCols);
            for (int j = 0; j < steps && !*gone; ++j) {
                const int at = (KEYS ? a.q0 : a.k0) + begin + j * by, head = KEYS ? kvh * p.group : kvh;
                const int s1 = j % kGradSlots1, s2 = j % kGradSlots2;
                if (j >= kGradSlots1 && !role_sleep(empty1 + s1, (j / kGradSlots1 - 1) & 1, gone, p.timeout_ns, p.status))
                    break;
                mbar_arrive_expect_tx(full1 + s1, bytes);
                for (int b = 0; b < DB; ++b)
                    tile_g2s_3d(smem_u32(ring1 + s1 * kTile + b * kAttnBlock), &p.z1, 64 * b, head, at, smem_u32(full1 + s1));
                ++sent1;
                if (j >= kGradSlots2 && !role_sleep(empty2 + s2, (j / kGradSlots2 - 1) & 1, gone, p.timeout_ns, p.status))
                    break;
                mbar_arrive_expect_tx(full2 + s2, bytes);
                for (int b = 0; b < DB; ++b)
                    tile_g2s_3d(smem_u32(ring2 + s2 * kTile + b * kAttnBlock), &p.z2, 64 * b, head, at, smem_u32(full2 + s2));
                ++sent2;
            }
            if (*gone) {  // what is in flight has landed before the memory is let go
                if (rows_sent) mbar_wait_bounded(x_full, 0, p.timeout_ns);
                for (int j = max(sent1 - kGradSlots1, 0); j < sent1; ++j)
                    mbar_wait_bounded(full1 + j % kGradSlots1, (j / kGradSlots1) & 1, p.timeout_ns);
                for (int j = max(sent2 - kGradSlots2, 0); j < sent2; ++j)
                    mbar_wait_bounded(full2 + j % kGradSlots2, (j / kGradSlots2) & 1, p.timeout_ns);
            }
        }
    } else if (warp == kGradProducts) {
        constexpr uint32_t desc_s = mma_desc(kAttnRows, kGradCols, false, false);
        constexpr uint32_t desc_acc = mma_desc(kAttnRows, D, false, true);
        // columns behind the sequence belong to another, or to nobody: zeros
        auto blank = [&](uint8_t* z, int j) {
            const int cols = cols_of(j);
            if (cols >= kGradCols) return;
            for (int x = lane + cols * 8; x < kGradCols * 8; x += 32)
#pragma unroll
                for (int b = 0; b < DB; ++b)
                    *reinterpret_cast<uint4*>(z + b * kAttnBlock + x * 16) = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
        };
        // 128 x 128 scores: rows of x by columns of z
        auto scores = [&](uint32_t to, const uint8_t* x, const uint8_t* z, uint64_t* done, uint64_t* free) {
            if (elect_one()) {
                const uint64_t dx = operand_desc(smem_u32(x), false), dz = operand_desc(smem_u32(z), false);
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        mma_bf16<1>(tmem + to, dx + b * (kAttnBlock >> 4) + y * k_step(false),
                                    dz + b * (kAttnBlock >> 4) + y * k_step(false), desc_s, b + y > 0);
                mma_commit(smem_u32(done));
                if (free) mma_commit(smem_u32(free));
            }
            __syncwarp();
        };
        // a gradient grows by the probabilities (or dS) at `from` times z
        auto grow = [&](uint32_t acc, uint32_t from, const uint8_t* z, bool add, uint64_t* free) {
            if (elect_one()) {
                const uint64_t dz = operand_desc_tall(smem_u32(z), kGradCols);
#pragma unroll
                for (int x = 0; x < kGradCols / 16; ++x)
                    mma_bf16_ts(tmem + acc, tmem + from + x / 2 * 32 + x % 2 * 8, dz + x * k_step(true), desc_acc,
                                add || x > 0);
                mma_commit(smem_u32(free));
            }
            __syncwarp();
        };
        // A place of a ring, walked without divisions (a wait and what goes with
        // it is in the way of the tensor cores, instruction by instruction).
        struct Place {
            int slot, phase;
            __device__ void next(int slots)
            {
                if (++slot == slots) slot = 0, phase ^= 1;
            }
        };
        Place z1{0, 0}, z2{0, 0};  // of the next S and dP
        const bool blanks = by * (KEYS ? p.group : 1) < kGradCols;  // (in every step)
        auto come1 = [&](int j) {  // z1 of step j has come
            if (!wait(full1 + z1.slot, z1.phase)) return false;
            if (blanks || j == steps - 1) blank(ring1 + z1.slot * kTile, j);
            return true;
        };
        auto come2 = [&](int j) {
            if (!wait(full2 + z2.slot, z2.phase)) return false;
            if (blanks || j == steps - 1) blank(ring2 + z2.slot * kTile, j);
            return true;
        };
        auto score_s = [&]() {
            scores(kScores, smem, ring1 + z1.slot * kTile, s_full, nullptr);
            z1.next(kGradSlots1);
        };
        auto score_dp = [&](int j) {
            scores(dp_at(j), smem + kTile, ring2 + z2.slot * kTile, dp_full + (j & 1), KEYS ? nullptr : empty2 + z2.slot);
            z2.next(kGradSlots2);
        };
        bool ok = steps == 0 || (wait(x_full, 0) && come1(0) && come2(0));
        if (steps > 0 && ok) {
            tc_fence_after();
            score_s();
            score_dp(0);
        }
        int old1 = 0;
        for (int j = 0; j < steps && ok; ++j) {
            const bool more = j + 1 < steps;
            if (KEYS) {
                // (two products at a time, their operands waited for before them)
                if (more && !(ok = come1(j + 1))) break;
                if (!(ok = wait(p_full, j & 1))) break;
                tc_fence_after();
                grow(kAcc2, kScores, ring2 + (j & 1) * kTile, j > 0, empty2 + (j & 1));
                if (more) score_s();
                if (more && !(ok = come2(j + 1))) break;
            } else {
                if (!(ok = wait(p_full, j & 1))) break;
                if (more && !(ok = come1(j + 1))) break;
                tc_fence_after();
                if (more) score_s();
                if (more && !(ok = come2(j + 1))) break;
                tc_fence_after();
                if (more) score_dp(j + 1);
            }
            if (!(ok = wait(ds_full + (j & 1), (j >> 1) & 1))) break;
            tc_fence_after();
            grow(0, dp_at(j), ring1 + old1 * kTile, j > 0, empty1 + old1);
            if (++old1 == kGradSlots1) old1 = 0;
            if (KEYS && more) score_dp(j + 1);
        }
        static_assert(kGradSlots2 == 2, "z2 of step j is in place j & 1");
        if (elect_one()) {  // every instruction is done before the memory is let go
            mma_commit(smem_u32(acc_full));
            mbar_wait_bounded(acc_full, 0, p.timeout_ns);
        }
        __syncwarp();
    } else if (warp == kGradStats) {
        if (KEYS) {
            int place[4];  // of the columns lane, lane + 32, ... in a row of statistics
#pragma unroll
            for (int q = 0; q < 4; ++q)
                place[q] = (lane + 32 * q) / p.group * p.heads + (lane + 32 * q) % p.group;
            for (int j = 0; j < steps; ++j) {
                const int64_t at = (int64_t)(a.q0 + begin + j * by) * p.heads + kvh * p.group;
                const int cols = cols_of(j);
                float2 st[4];
#pragma unroll
                for (int q = 0; q < 4; ++q)  // (behind the sequence: p = 0)
                    st[q] = lane + 32 * q < cols ? p.stats[at + place[q]] : make_float2(-minus_inf(), 0.0f);
                if (j >= 2 && !wait(ds_full + (j & 1), ((j >> 1) - 1) & 1)) break;
#pragma unroll
                for (int q = 0; q < 4; ++q) {  // (as they are added)
                    float* const to = col_stats + (j & 1) * 2 * kGradCols + lane + 32 * q;
                    to[0] = -st[q].x;
                    to[kGradCols] = -st[q].y;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(stat_full + (j & 1));
            }
        }
    } else {
        // a thread's row, and its quarter of a step's columns, whose P and dS lie
        // where this quarter of S and dP lay
        const int quarter = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_at = mine + kScores + quarter * 32;
        // the row: key row0 + r, or (token, head)
        const int token = row0 + r / p.group, head = kvh * p.group + r % p.group;
        const bool live = a.spares == 0 && (KEYS ? row0 + r < a.m : r < p.tile_tokens * p.group && token < a.n);
        const bool any_live = __any_sync(0xffffffffu, live);
        float2 own = make_float2(minus_inf(), 0.0f);  // both negative
        if (!KEYS && live) {
            own = p.stats[(int64_t)(a.q0 + token) * p.heads + head];
            own = make_float2(-own.x, -own.y);
        }
        // of the sequence's tokens, the first that sees the row's key; the last
        // key that the row's token sees
        const int64_t from = KEYS && p.causal ? (int64_t)row0 + r - shift : 0;
        const int64_t upto = p.causal ? min((int64_t)a.m - 1, (int64_t)token + shift) : (int64_t)a.m - 1;
        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
        bool ok = true;
        for (int j = 0; j < steps; ++j) {
            ok = wait(s_full, j & 1);
            if (KEYS && ok) ok = wait(stat_full + (j & 1), (j >> 1) & 1);
            if (!ok) break;
            tc_fence_after();
            // (four at a time: a load of each took the LSU longer than all else)
            const float4* st = reinterpret_cast<const float4*>(col_stats + (j & 1) * 2 * kGradCols + quarter * 32);
            float2 e[16];
            bool masked = false;
            if (any_live) {
                // the columns [lo, hi] of this quarter that the row sees (or that see it)
                int lo = 0, hi = 31;
                const int64_t f = begin + (int64_t)j * by;
                if (KEYS && p.causal)
                    lo = (int)max((int64_t)0, min((int64_t)32, (from - f) * p.group - quarter * 32));
                if (!KEYS) hi = (int)max((int64_t)-1, min((int64_t)31, upto - f - quarter * 32));
                masked = !__all_sync(0xffffffffu, lo == 0 && hi == 31) || cols_of(j) < kGradCols;
                float s[32];
                tmem_ld(s_at, s);
                tmem_wait_ld(s);
#pragma unroll
                for (int x = 0; x < 16; x += 2) {
                    float4 lse = make_float4(own.x, own.x, own.x, own.x);
                    if (KEYS) lse = st[x / 2];
                    e[x] = __ffma2_rn(make_float2(s[2 * x], s[2 * x + 1]), scale2, make_float2(lse.x, lse.y));
                    e[x + 1] = __ffma2_rn(make_float2(s[2 * x + 2], s[2 * x + 3]), scale2, make_float2(lse.z, lse.w));
                    e[x].x = exp2_fast(e[x].x);
                    e[x].y = exp2_fast(e[x].y);
                    e[x + 1].x = exp2_fast(e[x + 1].x);
                    e[x + 1].y = exp2_fast(e[x + 1].y);
                }
                if (masked) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        if (2 * x < lo || 2 * x > hi) e[x].x = 0.0f;
                        if (2 * x + 1 < lo || 2 * x + 1 > hi) e[x].y = 0.0f;
                    }
                }
                if (KEYS) {
                    uint32_t w[16];
#pragma unroll
                    for (int x = 0; x < 16; ++x) w[x] = pack_bf16x2(e[x].x, e[x].y);
                    tmem_st(s_at, w);
                    tmem_wait_st();
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full);
            ok = wait(dp_full + (j & 1), (j >> 1) & 1);
            if (!ok) break;
            tc_fence_after();
            if (any_live) {
                const uint32_t at = mine + dp_at(j) + quarter * 32;
                float dp[32];
                uint32_t w[16];
                tmem_ld(at, dp);
                tmem_wait_ld(dp);
#pragma unroll
                for (int x = 0; x < 16; x += 2) {
                    float4 delta = make_float4(own.y, own.y, own.y, own.y);
                    if (KEYS) delta = st[kGradCols / 4 + x / 2];
                    float2 ds[2] = {
                        __fmul2_rn(e[x], __fadd2_rn(make_float2(dp[2 * x], dp[2 * x + 1]), make_float2(delta.x, delta.y))),
                        __fmul2_rn(e[x + 1], __fadd2_rn(make_float2(dp[2 * x + 2], dp[2 * x + 3]), make_float2(delta.z, delta.w)))};
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        w[x + y] = pack_bf16x2(ds[y].x, ds[y].y);
                        // (0 times what need not be finite)
                        if (masked) w[x + y] &= (e[x + y].x == 0.0f ? 0u : 0xFFFFu) | (e[x + y].y == 0.0f ? 0u : 0xFFFF0000u);
                    }
                }
                tmem_st(at, w);
                tmem_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_full + (j & 1));
        }
        if (ok && steps > 0) {
            ok = role_sleep(acc_full, 0, gone, p.timeout_ns, p.status) && !*gone;
            ok = __all_sync(0xffffffffu, ok);
            tc_fence_after();
        }
        // dk or dq by warps 0-7, dv by warps 8-15, half of the columns each,
        // through the rows' memory so that a store covers whole rows
        const int turn = warp >> 3, half = warp >> 2 & 1;
        if (ok && any_live && (KEYS || turn == 0)) {
            constexpr int kHalf = D / 2;
            const float scale = turn == 0 ? p.scale : 1.0f;
            uint8_t* stage = smem + turn * kTile + (warp & 3) * 32 * D * 2;
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
