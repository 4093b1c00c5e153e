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
// rounded once for its matrix product (2^-8 of it), sums are fp32.  The tensor core
// cuts off what a product has below 2^-23 of the sum that it is added to, so one sum takes
// 1,024 steps (8,192 products, 2^-10 of it at most); what it has come to is then added to
// the thread's own in local memory (dv of 2^21 rows alike came out 1.6% low in one sum).  Where
// no sequence can have as many steps a kernel without this code runs.
//
// The matrix instructions are one thread's, in an order that leaves the rows'
// warps the time of two products for P and as long for dS:
//
//   keys stay:    dv(j), S(j+1), dk(j), dP(j+1)
//   queries stay: S(j+1), dP(j+1), dq(j)          (dP in two places in turn)
//
// (In steps of 64 columns, S and dP of two steps at a time, 1788 us where steps
// of 128 took 1710: the tensor cores read 1.26 times as much shared memory.)
//
// 4 x 4096 causal, 32 heads of 128 over 8: 1610 us with the statistics, 0.85
// PFLOP/s of the formulas' 5 products, 1.20 of the 7.  What bounds it is the chain
// scores, P, dS, product of a step, of which one CTA's tensor memory holds no
// second one beside the gradients.
//
// Warps: 0-15 make P and dS, four threads a row; 16 copies, 17 matrix
// instructions, 18 brings the columns' statistics (keys stay), 19 looks up the
// items.
#pragma once

#include "attention.cuh"

namespace quasar {

constexpr int kGradThreads = 640;
constexpr int kGradRowWarps = 16, kGradCopies = 16, kGradProducts = 17, kGradStats = 18, kGradItems = 19;  // warps
constexpr int kGradAhead = 3;  // of an item's steps, when the next is asked for
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

// What every role of a CTA knows of an item: its rows, and the steps of the
// other side.  Keys stay: the tokens from the first that sees a key of the tile.
// Queries stay: the keys that the last token sees.
struct GradWork {
    AttnItem a;
    int kvh;
    int row0;   // first key, or token, of the rows
    int begin;  // first token, or key, of the steps
    int steps;
    int end;    // there is no item
};

template <bool KEYS>
__device__ __forceinline__ GradWork grad_work(const AttnGradParams& p, int which)
{
    GradWork w{};
    w.kvh = which % p.kv_heads;
    w.a = find_item(p.s, which / p.kv_heads, p.items, KEYS ? kAttnRows : p.tile_tokens, KEYS);
    if (w.a.spares > 0) return w;
    w.row0 = w.a.index * (KEYS ? kAttnRows : p.tile_tokens);
    const int by = KEYS ? p.tile_tokens : kGradCols, shift = w.a.m - w.a.n;
    int end = 0;
    if (KEYS) {
        const int64_t sees = p.causal ? max((int64_t)0, (int64_t)w.row0 - shift) : 0;
        if (sees < w.a.n) w.begin = (int)sees / by * by, end = w.a.n;
    } else {
        const int64_t last = min((int64_t)w.row0 + p.tile_tokens, (int64_t)w.a.n) - 1;
        end = (int)max((int64_t)0, p.causal ? min((int64_t)w.a.m, last + 1 + shift) : (int64_t)w.a.m);
    }
    w.steps = (end - w.begin + by - 1) / by;
    return w;
}

__host__ __device__ constexpr size_t attention_grad_bytes(int blocks)
{
    return (size_t)(2 + kGradSlots1 + kGradSlots2) * blocks * kAttnBlock + 2 * 2 * kGradCols * 4 +
           (2 + 2 * kGradSlots1 + 2 * kGradSlots2 + 2 * 3 + 2 + 2 + 4 + 8) * 8 + 2 * sizeof(GradWork);
}

// The grid has a CTA for each item, and CTAs that run take those that have not
// been launched: the next one's tiles are on their way, and its first scores are
// made, while the gradients of one are written (with a CTA an item, keys
// and queries of 64 x 256 tokens, 16 heads of 128, took 202 and 191 us against 142
// and 130; of 4 x 4096, 32 heads over 8, 900 and 864 against 877 and 763).
//
// FAR: an item may have more steps than one sum takes.
template <int DB, bool KEYS, bool FAR>
__global__ void __launch_bounds__(kGradThreads, 1) k_attention_grad(const __grid_constant__ AttnGradParams p)
{
    constexpr int D = 64 * DB;
    constexpr uint32_t kTile = DB * kAttnBlock;  // bytes of 128 rows
    // columns of tensor memory: the gradients from 0 (and 128), the scores, dP
    constexpr uint32_t kAcc2 = 128, kScores = KEYS ? 256 : 128;
    auto dp_at = [](int g) { return KEYS ? 384u : 256u + (g & 1) * 128u; };
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring1 = smem + 2 * kTile;
    uint8_t* ring2 = ring1 + kGradSlots1 * kTile;
    float* col_stats = reinterpret_cast<float*>(ring2 + kGradSlots2 * kTile);  // [2][lse, D][128], negative
    uint64_t* x_full = reinterpret_cast<uint64_t*>(col_stats + 4 * kGradCols);
    uint64_t* x_empty = x_full + 1;
    uint64_t* full1 = x_empty + 1;              // [slots1]
    uint64_t* empty1 = full1 + kGradSlots1;
    uint64_t* full2 = empty1 + kGradSlots1;     // [slots2]
    uint64_t* empty2 = full2 + kGradSlots2;
    uint64_t* stat_full = empty2 + kGradSlots2; // [2]
    uint64_t* dp_full = stat_full + 2;          // [2]
    uint64_t* ds_full = dp_full + 2;            // [2]: the rows' warps
    uint64_t* s_full = ds_full + 2;
    uint64_t* p_full = s_full + 1;              // the rows' warps: the scores are read, P is in their place
    uint64_t* acc_full = p_full + 1;
    uint64_t* acc_empty = acc_full + 1;         // the rows' warps
    uint64_t* item_full = acc_empty + 1;        // [2]
    uint64_t* item_empty = item_full + 2;       // [2]: the warps that take items
    uint64_t* drained = item_empty + 2;
    uint64_t* never = drained + 1;
    uint64_t* near = never + 1;                 // an item's end is
    uint64_t* asked = near + 1;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(asked + 1);
    volatile uint32_t* gone = tmem_slot + 1;
    void* answer = asked + 2 + (asked - x_full & 1);  // (x_full is at a 16-byte boundary)
    GradWork* items = reinterpret_cast<GradWork*>(asked + 5);  // [2]

    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    uint32_t given;
    asm volatile("mov.u32 %0, %%dynamic_smem_size;" : "=r"(given));
    if (smem + attention_grad_bytes(DB) > smem_raw + given) {  // (it starts at a multiple of 1024, as declared)
        if (threadIdx.x == 0) record_timeout(p.status);
        return;
    }
    if (threadIdx.x == 0) {
        mbar_init(x_full, 1);
        mbar_init(x_empty, 1);
        for (int s = 0; s < 2 * kGradSlots1 + 2 * kGradSlots2; ++s) mbar_init(full1 + s, 1);
        for (int b = 0; b < 2; ++b) {
            mbar_init(stat_full + b, 1);
            mbar_init(dp_full + b, 1);
            mbar_init(ds_full + b, kGradRowWarps);
            mbar_init(item_full + b, 1);
            mbar_init(item_empty + b, kGradRowWarps + (KEYS ? 3 : 2));
        }
        mbar_init(s_full, 1);
        mbar_init(p_full, kGradRowWarps);
        mbar_init(acc_full, 1);
        mbar_init(acc_empty, kGradRowWarps);
        mbar_init(drained, 1);
        mbar_init(never, 1);
        mbar_init(near, 1);
        mbar_init(asked, 1);
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
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    wait_for_previous_grid();
    const uint32_t tmem = uniform(*tmem_slot);
    const int by = KEYS ? p.tile_tokens : kGradCols;  // tokens, or keys, of a step
    auto wait = [&](uint64_t* bar, uint32_t parity) {  // the warp's, with one outcome
        const bool ok = role_sleep(bar, parity, gone, p.timeout_ns, p.status);
        return __all_sync(0xffffffffu, ok);
    };
    // (an item of many keys may take longer than any one step of it may; the other
    // warps' waits end this one too)
    auto wait_long = [&](uint64_t* bar, uint32_t parity) {
        const bool ok = role_sleep(bar, parity, gone, 64 * p.timeout_ns, p.status);
        return __all_sync(0xffffffffu, ok);
    };
    // item k, once it is known; its place is for k + 2 when all have let it go
    auto take = [&](int k) { return wait(item_full + (k & 1), (k >> 1) & 1); };
    auto release = [&](int k) {
        __syncwarp();
        if (lane == 0) mbar_arrive(item_empty + (k & 1));
    };
    // A place of a ring, walked without divisions (a wait and what goes with it
    // is in the way of the tensor cores, instruction by instruction).
    struct Place {
        int slot, phase;
        __device__ void next(int slots)
        {
            if (++slot == slots) slot = 0, phase ^= 1;
        }
    };
    static_assert(kGradSlots2 == 2, "z2 of a step is in place g & 1");

    if (warp == kGradItems) {
        int which = (int)blockIdx.x;
        for (int k = 0; which >= 0; ++k) {
            if (k >= 2 && !wait_long(item_empty + (k & 1), ((k >> 1) - 1) & 1)) break;
            if (k > 0) {
                if (!wait_long(near, (k - 1) & 1)) break;
                if (lane == 0) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    ask_for_cta(answer, asked);
                }
                __syncwarp();
                if (!wait(asked, (k - 1) & 1)) {  // (nobody leaves before the answer is here)
                    mbar_wait_bounded(asked, (k - 1) & 1, p.timeout_ns);
                    break;
                }
                which = uniform(lane == 0 ? asked_cta(answer) : 0);
            }
            GradWork w{};
            if (which >= 0) w = grad_work<KEYS>(p, which);
            w.end = which < 0;
            if (lane == 0) {
                items[k & 1] = w;
                mbar_arrive(item_full + (k & 1));
            }
            __syncwarp();
        }
    } else if (warp == kGradCopies) {
        bool ok = true;
        if (p.force_timeout_ns) ok = __all_sync(0xffffffffu, role_sleep(never, 0, gone, p.force_timeout_ns, p.status));
        int sets = 0, sent1 = 0, sent2 = 0;  // of rows; steps of z1 and z2
        Place z1{0, 1}, z2{0, 1};            // (the phase of a place's release before)
        const uint32_t x_bytes = 2 * DB * 128 * (KEYS ? kAttnRows : (uint32_t)(p.tile_tokens * p.group));
        const uint32_t z_bytes = DB * 128 * (KEYS ? (uint32_t)(p.tile_tokens * p.group) : kGradCols);
        for (int k = 0, end = 0; ok && !end; ++k) {
            if (!(ok = take(k))) break;
            const GradWork w = items[k & 1];
            release(k);
            end = w.end;
            // the next item is asked for a few steps ahead, no sooner: the CTAs that
            // are through with theirs come first
            const int ask = max(0, w.steps - kGradAhead);
            if (ask == 0 && lane == 0) mbar_arrive(near);
            if (w.steps == 0) continue;
            if (sets > 0 && !(ok = wait(x_empty, (sets - 1) & 1))) break;
            ++sets;
            if (lane == 0) {
                mbar_arrive_expect_tx(x_full, x_bytes);
                for (int x = 0; x < 2; ++x)
                    for (int b = 0; b < DB; ++b)
                        tile_g2s_3d(smem_u32(smem + x * kTile + b * kAttnBlock), x ? &p.x2 : &p.x1, 64 * b,
                                    KEYS ? w.kvh : w.kvh * p.group, (KEYS ? w.a.k0 : w.a.q0) + w.row0, smem_u32(x_full));
            }
            int at = (KEYS ? w.a.q0 : w.a.k0) + w.begin;
            const int head = KEYS ? w.kvh * p.group : w.kvh;
            for (int j = 0; j < w.steps && ok; ++j, at += by) {
                if (j > 0 && j == ask && lane == 0) mbar_arrive(near);
                if (sent1 >= kGradSlots1 && !(ok = wait(empty1 + z1.slot, z1.phase))) break;
                if (lane == 0) {
                    mbar_arrive_expect_tx(full1 + z1.slot, z_bytes);
                    for (int b = 0; b < DB; ++b)
                        tile_g2s_3d(smem_u32(ring1 + z1.slot * kTile + b * kAttnBlock), &p.z1, 64 * b, head, at,
                                    smem_u32(full1 + z1.slot));
                }
                ++sent1;
                z1.next(kGradSlots1);
                if (sent2 >= kGradSlots2 && !(ok = wait(empty2 + z2.slot, z2.phase))) break;
                if (lane == 0) {
                    mbar_arrive_expect_tx(full2 + z2.slot, z_bytes);
                    for (int b = 0; b < DB; ++b)
                        tile_g2s_3d(smem_u32(ring2 + z2.slot * kTile + b * kAttnBlock), &p.z2, 64 * b, head, at,
                                    smem_u32(full2 + z2.slot));
                }
                ++sent2;
                z2.next(kGradSlots2);
            }
        }
        if (*gone && lane == 0) {  // what is in flight has landed before the memory is let go
            if (sets > 0) mbar_wait_bounded(x_full, (sets - 1) & 1, p.timeout_ns);
            for (int j = max(sent1 - kGradSlots1, 0); j < sent1; ++j)
                mbar_wait_bounded(full1 + j % kGradSlots1, (j / kGradSlots1) & 1, p.timeout_ns);
            for (int j = max(sent2 - kGradSlots2, 0); j < sent2; ++j)
                mbar_wait_bounded(full2 + j % kGradSlots2, (j / kGradSlots2) & 1, p.timeout_ns);
        }
        __syncwarp();
    } else if (warp == kGradProducts) {
        constexpr uint32_t desc_s = mma_desc(kAttnRows, kGradCols, false, false);
        constexpr uint32_t desc_acc = mma_desc(kAttnRows, D, false, true);
        // columns behind the sequence belong to another, or to nobody: zeros
        auto blank = [&](uint8_t* z, int cols) {
            if (cols >= kGradCols) return;
            for (int x = lane + cols * 8; x < kGradCols * 8; x += 32)
#pragma unroll
                for (int b = 0; b < DB; ++b)
                    *reinterpret_cast<uint4*>(z + b * kAttnBlock + x * 16) = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
        };
        // 128 x 128 scores: rows of x by columns of z
        auto scores = [&](uint32_t to, const uint8_t* x, const uint8_t* z, uint64_t* done, uint64_t* free,
                          uint64_t* rows_free) {
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
                if (rows_free) mma_commit(smem_u32(rows_free));
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
        Place z1{0, 0}, z2{0, 0};  // of the next S and dP
        int old1 = 0, sets = 0, sums = 0, g = 0;  // z1 of the step that ends; items with steps; sums, steps so far
        bool ok = true;
        for (int k = 0, end = 0; ok && !end; ++k) {
            if (!(ok = take(k))) break;
            const GradWork w = items[k & 1];
            release(k);
            end = uniform(w.end);
            const int steps = uniform(w.steps);
            if (steps == 0) continue;
            // columns of a step that are the sequence's
            const int last = KEYS ? (w.a.n - w.begin - (steps - 1) * by) * p.group : w.a.m - (steps - 1) * by;
            const int full = KEYS ? by * p.group : by;
            auto come1 = [&](int j) {  // z1 of step j has come
                if (!wait(full1 + z1.slot, z1.phase)) return false;
                if (full < kGradCols || j == steps - 1) blank(ring1 + z1.slot * kTile, j == steps - 1 ? last : full);
                return true;
            };
            auto come2 = [&](int j) {
                if (!wait(full2 + z2.slot, z2.phase)) return false;
                if (full < kGradCols || j == steps - 1) blank(ring2 + z2.slot * kTile, j == steps - 1 ? last : full);
                return true;
            };
            auto score_s = [&]() {
                scores(kScores, smem, ring1 + z1.slot * kTile, s_full, nullptr, nullptr);
                z1.next(kGradSlots1);
            };
            auto score_dp = [&](int j) {
                scores(dp_at(g + j), smem + kTile, ring2 + z2.slot * kTile, dp_full + (g + j & 1),
                       KEYS ? nullptr : empty2 + z2.slot, j == steps - 1 ? x_empty : nullptr);
                z2.next(kGradSlots2);
            };
            if (!(ok = wait(x_full, sets & 1) && come1(0) && come2(0))) break;
            tc_fence_after();
            score_s();
            score_dp(0);
            for (int j = 0; j < steps; ++j) {
                const bool more = j + 1 < steps;
                const int gj = g + j;
                // the gradients of the item before, or of the sum before, have been read
                const bool first = FAR ? j % kGradFold == 0 : j == 0;
                if (first && sums > 0 && !(ok = wait(acc_empty, (sums - 1) & 1))) break;
                if (KEYS) {
                    // (two products at a time, their operands waited for before them)
                    if (more && !(ok = come1(j + 1))) break;
                    if (!(ok = wait(p_full, gj & 1))) break;
                    tc_fence_after();
                    grow(kAcc2, kScores, ring2 + (gj & 1) * kTile, !first, empty2 + (gj & 1));
                    if (more) score_s();
                    if (more && !(ok = come2(j + 1))) break;
                } else {
                    if (!(ok = wait(p_full, gj & 1))) break;
                    if (more && !(ok = come1(j + 1))) break;
                    tc_fence_after();
                    if (more) score_s();
                    if (more && !(ok = come2(j + 1))) break;
                    tc_fence_after();
                    if (more) score_dp(j + 1);
                }
                if (!(ok = wait(ds_full + (gj & 1), (gj >> 1) & 1))) break;
                tc_fence_after();
                grow(0, dp_at(gj), ring1 + old1 * kTile, !first, empty1 + old1);
                if (++old1 == kGradSlots1) old1 = 0;
                if (FAR && more && (j + 1) % kGradFold == 0) {  // a sum is full
                    if (elect_one()) mma_commit(smem_u32(acc_full));
                    __syncwarp();
                    ++sums;
                }
                if (KEYS && more) score_dp(j + 1);
            }
            if (!ok) break;
            if (elect_one()) mma_commit(smem_u32(acc_full));
            __syncwarp();
            ++sets;
            ++sums;
            g += steps;
        }
        if (elect_one()) {  // every instruction is done before the memory is let go
            mma_commit(smem_u32(drained));
            mbar_wait_bounded(drained, 0, p.timeout_ns);
        }
        __syncwarp();
    } else if (warp == kGradStats) {
        if (KEYS) {
            int place[4];  // of the columns lane, lane + 32, ... in a row of statistics
#pragma unroll
            for (int q = 0; q < 4; ++q)
                place[q] = (lane + 32 * q) / p.group * p.heads + (lane + 32 * q) % p.group;
            bool ok = true;
            int g = 0;
            for (int k = 0, end = 0; ok && !end; ++k) {
                if (!(ok = take(k))) break;
                const GradWork w = items[k & 1];
                release(k);
                end = w.end;
                for (int j = 0; j < w.steps; ++j, ++g) {
                    const int64_t at = (int64_t)(w.a.q0 + w.begin + j * by) * p.heads + w.kvh * p.group;
                    const int cols = min(by, w.a.n - w.begin - j * by) * p.group;
                    float2 st[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q)  // (behind the sequence: p = 0)
                        st[q] = lane + 32 * q < cols ? p.stats[at + place[q]] : make_float2(-minus_inf(), 0.0f);
                    if (g >= 2 && !(ok = wait(ds_full + (g & 1), ((g >> 1) - 1) & 1))) break;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {  // (as they are added)
                        float* const to = col_stats + (g & 1) * 2 * kGradCols + lane + 32 * q;
                        to[0] = -st[q].x;
                        to[kGradCols] = -st[q].y;
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(stat_full + (g & 1));
                }
            }
        }
    } else {
        // a thread's row, and its quarter of a step's columns, whose P and dS lie
        // where this quarter of S and dP lay
        const int quarter = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t mine = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_at = mine + kScores + quarter * 32;
        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2);
        // keys stay: dk by warps 0-7, dv by warps 8-15, half of the columns each;
        // queries stay: a quarter of the columns of dq each
        constexpr int kSpan = KEYS ? D / 2 : D / 4;
        const bool second = KEYS && warp >= 8;
        const int c0 = KEYS ? (quarter & 1) * kSpan : quarter * kSpan;
        const uint32_t acc_at = mine + (second ? kAcc2 : 0) + c0;
        bool ok = true;
        int sums = 0, g = 0;
        for (int k = 0; ok; ++k) {
            if (!(ok = take(k))) break;
            const GradWork& w = items[k & 1];
            if (w.end) break;
            if (w.a.spares > 0) {
                constexpr int kMany = kGradRowWarps * 32;
                if (KEYS) {
                    clear_rows(p.d1, p.ld_d1, (int64_t)w.kvh * p.d, p.d, p.s.key_starts, p.s.n, p.s.keys, w.a.index,
                               w.a.spares, threadIdx.x, kMany);
                    clear_rows(p.d2, p.ld_d2, (int64_t)w.kvh * p.d, p.d, p.s.key_starts, p.s.n, p.s.keys, w.a.index,
                               w.a.spares, threadIdx.x, kMany);
                } else {
                    clear_rows(p.d1, p.ld_d1, (int64_t)w.kvh * p.group * p.d, p.group * p.d, p.s.starts, p.s.n,
                               p.s.tokens, w.a.index, w.a.spares, threadIdx.x, kMany);
                }
                release(k);
                continue;
            }
            // the row: key row0 + r, or (token, head)
            const int steps = w.steps, shift = w.a.m - w.a.n;  // key j is seen by tokens from j - shift on
            const int token = w.row0 + r / p.group, head = w.kvh * p.group + r % p.group;
            const bool live = KEYS ? w.row0 + r < w.a.m : r < p.tile_tokens * p.group && token < w.a.n;
            const bool any_live = __any_sync(0xffffffffu, live);
            float2 own = make_float2(minus_inf(), 0.0f);  // both negative
            if (!KEYS && live) {
                own = p.stats[(int64_t)(w.a.q0 + token) * p.heads + head];
                own = make_float2(-own.x, -own.y);
            }
            // of the sequence's tokens, the first that sees the row's key; the last
            // key that the row's token sees
            // (-2^30: it sees none; a sequence's places are below 2^31)
            const int from = KEYS && p.causal ? (int)max((int64_t)0, (int64_t)w.row0 + r - shift) : 0;
            const int64_t last = (int64_t)w.a.m - 1;
            const int upto = (int)max((int64_t)-(1 << 30), p.causal ? min(last, (int64_t)token + shift) : last);
            const int begin = w.begin;
            [[maybe_unused]] float before[FAR ? kSpan : 1];  // the gradients of the sums before (in local memory)
            for (int j = 0; j < steps; ++j, ++g) {
                ok = wait(s_full, g & 1);
                if (KEYS && ok) ok = wait(stat_full + (g & 1), (g >> 1) & 1);
                if (!ok) break;
                tc_fence_after();
                // (four at a time: a load of each took the LSU longer than all else)
                const float4* st = reinterpret_cast<const float4*>(col_stats + (g & 1) * 2 * kGradCols + quarter * 32);
                float2 e[16];
                bool masked = false;
                if (any_live) {
                    // the columns [lo, hi] of this quarter that the row sees (or that see it)
                    int lo = 0, hi = 31;
                    const int f = begin + j * by;
                    if (KEYS && p.causal) lo = max(0, min(32, min(max(from - f, 0), kGradCols) * p.group - quarter * 32));
                    if (!KEYS) hi = max(-1, min(31, upto - f - quarter * 32));
                    masked = !__all_sync(0xffffffffu, lo == 0 && hi == 31) || (KEYS && j == steps - 1) ||
                             (KEYS && by * p.group < kGradCols);
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
                        uint32_t words[16];
#pragma unroll
                        for (int x = 0; x < 16; ++x) words[x] = pack_bf16x2(e[x].x, e[x].y);
                        tmem_st(s_at, words);
                        tmem_wait_st();
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full);
                ok = wait(dp_full + (g & 1), (g >> 1) & 1);
                if (!ok) break;
                tc_fence_after();
                if (any_live) {
                    const uint32_t at = mine + dp_at(g) + quarter * 32;
#pragma unroll
                    for (int h = 0; h < 16; h += 8) {  // (16 columns at a time: registers)
                        float dp[16];
                        uint32_t words[8];
                        tmem_ld(at + 2 * h, dp);
                        tmem_wait_ld(dp);
#pragma unroll
                        for (int x = 0; x < 8; x += 2) {
                            float4 delta = make_float4(own.y, own.y, own.y, own.y);
                            if (KEYS) delta = st[kGradCols / 4 + (h + x) / 2];
                            float2 ds[2] = {__fadd2_rn(make_float2(dp[2 * x], dp[2 * x + 1]), make_float2(delta.x, delta.y)),
                                            __fadd2_rn(make_float2(dp[2 * x + 2], dp[2 * x + 3]),
                                                       make_float2(delta.z, delta.w))};
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                ds[y] = __fmul2_rn(e[h + x + y], ds[y]);
                                words[x + y] = pack_bf16x2(ds[y].x, ds[y].y);
                                // (0 times what need not be finite)
                                if (masked)
                                    words[x + y] &= (e[h + x + y].x == 0.0f ? 0u : 0xFFFFu) |
                                                    (e[h + x + y].y == 0.0f ? 0u : 0xFFFF0000u);
                            }
                        }
                        tmem_st(at + h, words);
                    }
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(ds_full + (g & 1));
                if (FAR && (j + 1) % kGradFold == 0 && j + 1 < steps) {  // a sum is full
                    if (!(ok = wait(acc_full, sums & 1))) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < kSpan; c += 16) {
                        float o[16];
                        tmem_ld16(acc_at + c, o);
#pragma unroll
                        for (int x = 0; x < 16; ++x) before[c + x] = j < kGradFold ? o[x] : before[c + x] + o[x];
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(acc_empty);
                    ++sums;
                }
            }
            if (!ok) break;
            if (steps > 0) {
                if (!(ok = wait(acc_full, sums & 1))) break;
                tc_fence_after();
            }
            const float scale = second ? 1.0f : p.scale;
            uint32_t out[kSpan / 2];
#pragma unroll
            for (int c = 0; c < kSpan; c += 16) {
                float o[16];
                if (steps > 0) {
                    tmem_ld(acc_at + c, o);
                    tmem_wait_ld(o);
                } else {
#pragma unroll
                    for (int x = 0; x < 16; ++x) o[x] = 0.0f;
                }
                if (FAR && steps > kGradFold) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) o[x] += before[c + x];
                }
#pragma unroll
                for (int x = 0; x < 16; x += 2) out[(c + x) / 2] = pack_bf16x2(o[x] * scale, o[x + 1] * scale);
            }
            if (!KEYS && upto < 0) {  // it sees no key: 0, and not 0 times keys that need not be finite
#pragma unroll
                for (int x = 0; x < kSpan / 2; ++x) out[x] = 0;
            }
            if (steps > 0) {  // read: the next item's may grow
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(acc_empty);
                ++sums;
            }
            if (live) {
                __nv_bfloat16* const to =
                    static_cast<__nv_bfloat16*>(second ? p.d2 : p.d1) +
                    (KEYS ? (int64_t)(w.a.k0 + w.row0 + r) * (second ? p.ld_d2 : p.ld_d1) + (int64_t)w.kvh * p.d
                          : (int64_t)(w.a.q0 + token) * p.ld_d1 + (int64_t)head * p.d) + c0;
#pragma unroll
                for (int c = 0; c < kSpan; c += 8)
                    if (c0 + c < p.d)
                        *reinterpret_cast<uint4*>(to + c) =
                            make_uint4(out[c / 2], out[c / 2 + 1], out[c / 2 + 2], out[c / 2 + 3]);
            }
            release(k);
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kGradProducts) tmem_free<1>(tmem, 512);
}

}  // namespace quasar
