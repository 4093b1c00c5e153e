// Attention over packed sequences: y = softmax(scale q k^T) v, with the row's
// log-sum-exp.
//
// A CTA takes two tiles of 128 rows.  A row is a (token, head) pair: the heads
// that share keys lie side by side in a tile, so that few tokens with many
// heads still fill it and keys are read once for all of them.  The tiles take
// turns on the tensor cores: while one's probabilities are made, the other's
// products run.  For each key tile j and row tile i
//
//   S_i = Q_i K_j^T          in tensor memory, 128 x 128 fp32
//   m, l, P                  P in bf16 takes S's place, each half in its half
//   O_i += P V_j             P from tensor memory, V as it lies in memory
//
// in one pass over the keys with the running maximum m and sum l of the
// softmax.  O and l follow the maximum only when it has grown by more than
// 2^8 (so P stays below 2^8, and the rounding of P to bf16 is relative): the
// quotient O / l does not depend on which maximum was subtracted.
//
// P is rounded to bf16 for the matrix product (2^-8 of it at most); l is the sum
// before the rounding.
//
// The tensor core cuts off what a product has below 2^-23 of the sum that it is added
// to, of many keys alike a little each time: in one sum values of 1.99 over 2^20 keys came
// out 0.8% low, over 2^22 3.9%.  So O grows by 1,024 key tiles at a time (8,192
// products, 2^-10 of a sum at most), each with a maximum and an l of its own, and what they
// leave is joined in fp32 in the thread's local memory.  Where k has no more rows than
// that (131,072) a kernel without this code runs (256 single tokens over 2,048 keys
// each: 357 us without, 361 with it).
//
// Where rows are few, a cluster of CTAs shares a row's keys, and where there are
// rows for one tile alone, the tiles are twins: the same rows, every other key
// tile each.  Twins are joined in tensor memory, the parts of a cluster's CTAs
// through distributed shared memory, always in the same order.
//
// Warps: 0-7 and 8-15 the rows of tiles 0 and 1, two threads a row, 64 keys of a
// key tile each, that exchange their maxima (with one thread a row the tensor
// cores waited for a tile's 4 warps: 565 us); 16 copies, 17 matrix instructions,
// 18 looks up the items.
//
// 4 x 4096 causal, 32 heads of 128 over 8: 452 us, 1.22 PFLOP/s of the products at
// and below the diagonal, 0.72 of the sustained rate.  What bounds it is the
// chain from a tile's scores through P to its next product, which the other tile
// hides in part, and the product thread's waits (some hundred cycles each, and
// the tensor cores hold few instructions); masked halves of diagonal tiles are
// computed too, 1.03 of the work.  One query for each of 61 sequences of up to
// 2,048 keys, 32 heads over 8: 73 us, 4.5 TB/s, bound by the last of 3.2 items an SM
// (256 sequences of 2,048 keys 354 us, 6.1 TB/s).  For each of 8 sequences of up to 16,384
// keys: 77 us, 4.6 TB/s: 64 items are fewer than the SMs, so clusters of four CTAs have one
// each, 256 CTAs for 152 SMs, whose second round starts when the first has ended.
#pragma once

#include "attention.h"
#include "cluster.cuh"
#include "tensor_core.cuh"

namespace quasar {

constexpr int kAttnThreads = 608;
constexpr int kAttnRowWarps = 16, kAttnCopies = 16, kAttnProducts = 17, kAttnItems = 18;  // warps
// Places of the ring, each a tile of values and one of keys: 128 KB (heads of 64 with
// two: 128 queries of 2,048 keys, 32 heads over 8, 125 us against 104).
template <int DB>
constexpr int kAttnSlots = DB == 1 ? 4 : 2;
constexpr int kAttnAhead = 3;             // of an item's entries, when the next is asked for
constexpr float kAttnSlack = 8.0f;        // log2 of how far m may fall behind
constexpr uint32_t kAttnBlock = kAttnRows * 128;  // bytes of 128 rows x 64 bf16

__device__ __forceinline__ float minus_inf() { return __int_as_float(0xFF800000); }

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The rows of sequence i.  Whatever the offsets hold, no row outside the
// tensor is named.
__device__ __forceinline__ void sequence_rows(const int* starts, int i, int rows, int& from, int& n)
{
    if (!starts) {
        from = 0, n = rows;
        return;
    }
    from = min(max(starts[i], 0), rows);
    n = min(max(starts[i + 1], from), rows) - from;
}

struct AttnItem {
    int q0, n;   // rows of q
    int k0, m;   // rows of k and v
    int index;   // of the item in the sequence, or of a spare item
    int spares;  // > 0: no sequence has this item; how many such there are
};

// The sequence that item `want` falls into, where a sequence of n rows has
// ceil(n / span) items (rows of q, or of the keys).  Whole-warp call; 128
// sequences are read at a time.
__device__ __forceinline__ AttnItem find_item(const AttnSequences& s, int want, int items, int span, bool of_keys = false)
{
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int base = 0; base < s.n; base += 128) {
        int mine[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            int from = 0, n = 0;
            if (base + 32 * q + lane < s.n)
                sequence_rows(of_keys ? s.key_starts : s.starts, base + 32 * q + lane, of_keys ? s.keys : s.tokens, from, n);
            mine[q] = (int)(((int64_t)n + span - 1) / span);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            int upto = mine[q];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, upto, o);
                if (lane >= o) upto += x;
            }
            const unsigned hit = __ballot_sync(0xffffffffu, before + upto > want);
            if (hit) {
                const int l = __ffs(hit) - 1;
                AttnItem a{};
                sequence_rows(s.starts, base + 32 * q + l, s.tokens, a.q0, a.n);
                sequence_rows(s.key_starts, base + 32 * q + l, s.keys, a.k0, a.m);
                const int count = __shfl_sync(0xffffffffu, mine[q], l);
                // the longest first, under a causal mask: the last tokens, the first keys
                a.index = want - before - __shfl_sync(0xffffffffu, upto - mine[q], l);
                if (!of_keys) a.index = count - 1 - a.index;
                return a;
            }
            before += __shfl_sync(0xffffffffu, upto, 31);
        }
    }
    return AttnItem{0, 0, 0, 0, want - before, items - before};
}

// Zeros in the columns [c0, c0 + width) of the rows that no sequence has, the
// spare items taking turns.  (bf16, 16-byte aligned)
__device__ __forceinline__ void clear_rows(void* out, int64_t ld, int64_t c0, int width, const int* starts, int n_seq,
                                           int rows, int index, int spares, int thread, int threads)
{
    if (!out) return;
    const int first = starts ? min(max(starts[0], 0), rows) : 0;
    const int last = starts ? max(first, min(max(starts[n_seq], 0), rows)) : rows;
    const int vecs = width / 8;
    for (int64_t r = index; r < (int64_t)first + (rows - last); r += spares) {
        const int64_t row = r < first ? r : r - first + last;
        uint4* p = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(out) + row * ld + c0);
        for (int v = thread; v < vecs; v += threads) p[v] = make_uint4(0, 0, 0, 0);
    }
}

__device__ __forceinline__ void clear_lse(float* lse, int heads, int h0, int group, const int* starts, int n_seq,
                                          int rows, int index, int spares, int thread, int threads)
{
    if (!lse) return;
    const int first = starts ? min(max(starts[0], 0), rows) : 0;
    const int last = starts ? max(first, min(max(starts[n_seq], 0), rows)) : rows;
    for (int64_t r = index; r < (int64_t)first + (rows - last); r += spares) {
        const int64_t row = r < first ? r : r - first + last;
        for (int h = thread; h < group; h += threads) lse[row * heads + h0 + h] = minus_inf();
    }
}

// Key tiles that a row tile of tokens [t0, t1) of the sequence sees.
__device__ __forceinline__ int key_tiles(const AttnItem& a, int t0, int t1, bool causal)
{
    const int last = min(t1, a.n) - 1;
    if (last < t0) return 0;
    const int64_t see = causal ? min((int64_t)a.m, (int64_t)last + 1 + a.m - a.n) : a.m;
    return see > 0 ? (int)((see + kAttnKeys - 1) / kAttnKeys) : 0;
}

// What every role of a CTA knows of an item: its rows, and its key tiles:
// `count` from `first` on, of which tile i takes n_i (twins: every other one).
// They come as entries of the ring, a key tile with the values of the one `lag`
// before it.
struct AttnWork {
    AttnItem a;
    int kvh;
    int t0;  // first token of tile 0
    int first, count, n[2];
    int twins, lag, entries;
    int end;  // 1: the CTA's last item, 2: there is none
};

__device__ __forceinline__ AttnWork attention_work(const AttnParams& p, int which, int rank)
{
    AttnWork w{};
    w.kvh = which % p.kv_heads;
    w.a = find_item(p.s, which / p.kv_heads, p.items, 2 * p.tile_tokens);
    w.t0 = w.a.index * 2 * p.tile_tokens;
    w.lag = 1;
    if (w.a.spares > 0) return w;
    w.n[0] = key_tiles(w.a, w.t0, w.t0 + p.tile_tokens, p.causal);
    w.n[1] = key_tiles(w.a, w.t0 + p.tile_tokens, w.t0 + 2 * p.tile_tokens, p.causal);
    w.twins = w.a.n - w.t0 <= p.tile_tokens && w.n[0] > 1;
    const int most = max(w.n[0], w.n[1]);
    w.first = (int)((int64_t)most * rank / p.split);
    w.count = (int)((int64_t)most * (rank + 1) / p.split) - w.first;
    if (w.twins) {
        w.lag = 2;
        w.n[0] = (w.count + 1) / 2;
        w.n[1] = w.count / 2;
    } else {
        w.n[0] = max(min(w.n[0] - w.first, w.count), 0);
        w.n[1] = max(min(w.n[1] - w.first, w.count), 0);
    }
    w.entries = max(w.n[0], w.n[1]) > 0 ? w.count + w.lag : 0;
    return w;
}

// What a row has summed of some key tiles (O's columns, l and its maximum) joined to
// what it has of those before; O, l and m then start again or, behind the last tiles,
// hold it all.
template <int COLUMNS>
__device__ __forceinline__ float2 join_tiles(float* before, uint32_t o_at, float m, float l, bool first, bool last)
{
    const float top = first ? m : fmaxf(m, before[COLUMNS + 1]), shift = top == minus_inf() ? 0.0f : top;
    const float old = first ? 0.0f : exp2_fast(before[COLUMNS + 1] - shift), now = exp2_fast(m - shift);
#pragma unroll 1
    for (int c = 0; c < COLUMNS; c += 16) {
        float o[16];
        tmem_ld16(o_at + c, o);
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            const float sum = first ? o[x] : fmaf(o[x], now, before[c + x] * old);
            before[c + x] = sum;
            o[x] = last ? sum : 0.0f;
        }
        tmem_st16(o_at + c, o);
    }
    tmem_wait_st();
    l = first ? l : fmaf(l, now, before[COLUMNS] * old);
    before[COLUMNS] = l;
    before[COLUMNS + 1] = top;
    return last ? make_float2(top, l) : make_float2(minus_inf(), 0.0f);
}

// D = 64 DB columns; a head of d columns is completed with zeros.
//
// A CTA takes items until there are none (or, where few are, has one): while one's
// last products run and its rows are written, the next one's tiles are on their
// way and its first products follow at once.  The grid has a CTA for each item,
// and CTAs that run take those that have not been launched (replayed side by side,
// 4 x 4096 440 us; with items dealt out beforehand 454, though one sequence of 2,048 40
// as now; with a CTA an item 512; 256 queries of 2,048 keys 346, with a CTA an item
// 460, without twins 378).
//
// FAR: a sequence may have more key tiles than one sum takes.
template <int DB, bool FAR>
__global__ void __launch_bounds__(kAttnThreads, 1) k_attention(const __grid_constant__ AttnParams p)
{
    constexpr int D = 64 * DB;
    constexpr uint32_t kTile = DB * kAttnBlock;  // bytes of a tile of q, k or v
    constexpr int kSlots = kAttnSlots<DB>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ring = smem + 2 * kTile;
    uint64_t* q_full = reinterpret_cast<uint64_t*>(ring + kSlots * 2 * kTile);
    uint64_t* q_empty = q_full + 1;
    uint64_t* full = q_empty + 1;          // [slots]
    uint64_t* empty = full + kSlots;       // [slots]
    uint64_t* s_full = empty + kSlots;     // [2]
    uint64_t* p_full = s_full + 2;         // [2]: 8 warps
    uint64_t* o_full = p_full + 2;         // [2]
    uint64_t* o_empty = o_full + 2;        // [2]: 8 warps
    uint64_t* item_full = o_empty + 2;     // [2]
    uint64_t* item_empty = item_full + 2;  // [2]: the other warps
    uint64_t* drained = item_empty + 2;
    uint64_t* never = drained + 1;
    uint64_t* near = never + 1;  // an item's end is
    uint64_t* join = near + 1;   // [4]: twin 1 of 32 rows is done
    uint64_t* asked = join + 4;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(asked + 1);
    volatile uint32_t* gone = tmem_slot + 1;
    void* answer = asked + 3;                                 // (at a 16-byte boundary, and what follows)
    float2* stat = reinterpret_cast<float2*>(asked + 5);      // [2][128]: m and l, where rows have parts
    float2* swap = stat + 256;                                // [2 turns][2 tiles][2 halves][128]
    uint8_t* stages = reinterpret_cast<uint8_t*>(swap + 1024);   // 1 KB a warp of rows
    AttnWork* items = reinterpret_cast<AttnWork*>(stages + kAttnRowWarps * 1024);  // [2]

    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int rank = p.split > 1 ? (int)cluster_rank() : 0;
    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(full + s, 1);
            mbar_init(empty + s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(s_full + i, 1);
            mbar_init(p_full + i, 8);
            mbar_init(o_full + i, 1);
            mbar_init(o_empty + i, 8);
            mbar_init(item_full + i, 1);
            mbar_init(item_empty + i, kAttnRowWarps + 2);
        }
        mbar_init(drained, 1);
        mbar_init(never, 1);
        mbar_init(near, 1);
        mbar_init(asked, 1);
        for (int i = 0; i < 4; ++i) mbar_init(join + i, 1);
        *gone = 0;
        mbar_init_fence();
    }
    if (warp == kAttnProducts) tmem_alloc<1>(tmem_slot, 512);
    if (warp == kAttnCopies && lane == 0) {
        prefetch_map(&p.q);
        prefetch_map(&p.k);
        prefetch_map(&p.v);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    wait_for_previous_grid();
    const uint32_t tmem = uniform(*tmem_slot);
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

    if (warp == kAttnItems) {
        int which = (int)blockIdx.x / p.split;
        for (int k = 0, end = 0; end == 0; ++k) {
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
            AttnWork w{};
            if (which >= 0) w = attention_work(p, which, rank);
            w.end = end = which < 0 ? 2 : !p.persistent;
            if (lane == 0) {
                items[k & 1] = w;
                mbar_arrive(item_full + (k & 1));
            }
            __syncwarp();
        }
    } else if (warp == kAttnCopies) {
        bool ok = true;
        if (p.force_timeout_ns) ok = __all_sync(0xffffffffu, role_sleep(never, 0, gone, p.force_timeout_ns, p.status));
        int it = 0, queries = 0;  // entries of the ring and sets of queries so far
        for (int k = 0, end = 0; ok && end == 0; ++k) {
            if (!(ok = take(k))) break;
            const AttnWork w = items[k & 1];
            release(k);
            end = w.end;
            // the next item is asked for a few key tiles ahead, no sooner: the CTAs
            // that are through with theirs come first (at once, 2,048 tokens of one
            // sequence took 54 us against 41)
            const int ask = max(0, w.entries - kAttnAhead);
            if (ask == 0 && lane == 0) mbar_arrive(near);
            if (w.entries == 0) continue;
            if (queries > 0 && !(ok = wait(q_empty, (queries - 1) & 1))) break;
            if (lane == 0) {
                const uint32_t bytes = (uint32_t)(p.tile_tokens * p.group) * 128 * DB;
                const bool both = w.n[1] > 0 && !w.twins;
                mbar_arrive_expect_tx(q_full, (w.n[0] > 0 ? bytes : 0) + (both ? bytes : 0));
                for (int i = 0; i < 2; ++i)
                    if (i ? both : w.n[0] > 0)
                        for (int b = 0; b < DB; ++b)
                            tile_g2s_3d(smem_u32(smem + i * kTile + b * kAttnBlock), &p.q, 64 * b, w.kvh * p.group,
                                        w.a.q0 + w.t0 + i * p.tile_tokens, smem_u32(q_full));
            }
            ++queries;
            for (int e = 0; e < w.entries; ++e, ++it) {
                const int s = it % kSlots;
                if (e > 0 && e == ask && lane == 0) mbar_arrive(near);
                if (it >= kSlots && !(ok = wait(empty + s, (it / kSlots - 1) & 1))) break;
                if (lane == 0) {
                    const bool values = e >= w.lag, keys = e < w.count;
                    mbar_arrive_expect_tx(full + s, (values ? kTile : 0) + (keys ? kTile : 0));
                    const uint32_t to = smem_u32(ring + s * 2 * kTile);
                    const int key = w.a.k0 + (w.first + e) * kAttnKeys;
                    for (int b = 0; b < DB; ++b) {
                        if (values)
                            tile_g2s_3d(to + b * kAttnBlock, &p.v, 64 * b, w.kvh, key - w.lag * kAttnKeys,
                                        smem_u32(full + s));
                        if (keys) tile_g2s_3d(to + kTile + b * kAttnBlock, &p.k, 64 * b, w.kvh, key, smem_u32(full + s));
                    }
                }
                __syncwarp();
            }
        }
        if (*gone && lane == 0) {  // what is in flight has landed before the memory is let go
            if (queries > 0) mbar_wait_bounded(q_full, (queries - 1) & 1, p.timeout_ns);
            for (int j = max(it - kSlots, 0); j < it; ++j)
                mbar_wait_bounded(full + j % kSlots, (j / kSlots) & 1, p.timeout_ns);
        }
    } else if (warp == kAttnProducts) {
        // One thread for both tiles, first come first served: with a warp each
        // their products share the tensor cores instruction by instruction,
        // both end late, and 4 x 4096 took 550 us where one thread's took 492.
        constexpr uint32_t desc_s = mma_desc(kAttnRows, kAttnKeys, false, false);
        constexpr uint32_t desc_o = mma_desc(kAttnRows, D, false, true);
        int it = 0, queries = 0, done[2] = {0, 0}, outs[2] = {0, 0};  // steps and rows of outputs of a tile
        bool ok = true;
        for (int k = 0, end = 0; ok && end == 0; ++k) {
            if (!(ok = take(k))) break;
            const AttnWork w = items[k & 1];
            release(k);
            end = uniform(w.end);
            const int entries = uniform(w.entries), count = uniform(w.count), lag = uniform(w.lag);
            const int n[2] = {uniform(w.n[0]), uniform(w.n[1])};
            const bool twins = uniform(w.twins) != 0;
            if (entries == 0) continue;
            if (!(ok = wait(q_full, queries & 1))) break;
            ++queries;
            for (int e = 0; e < entries && ok; ++e, ++it) {
                const int s = it % kSlots;
                if (!(ok = wait(full + s, (it / kSlots) & 1))) break;
                uint8_t* const values = ring + s * 2 * kTile;
                // rows of V behind the sequence belong to another, or to nobody:
                // their probabilities are 0, but 0 times what lies there need not be
                const int left = w.a.m - (w.first + e - lag) * kAttnKeys;
                if (e >= lag && left < kAttnKeys) {
                    for (int x = lane + left * 8; x < kAttnKeys * 8; x += 32)
#pragma unroll
                        for (int b = 0; b < DB; ++b)
                            *reinterpret_cast<uint4*>(values + b * kAttnBlock + x * 16) = make_uint4(0, 0, 0, 0);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                const uint64_t dv = operand_desc_tall(smem_u32(values), kAttnKeys);
                const uint64_t dk = operand_desc(smem_u32(values + kTile), false);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (twins && i != (e & 1)) continue;
                    const int j = (twins ? e >> 1 : e) - 1;  // of the values, in the tile's own steps
                    const bool grow = j >= 0 && j < n[i], score = j + 1 < n[i];
                    if (grow) {
                        if (!(ok = wait(p_full + i, (done[i] + j) & 1))) break;
                        // the rows of the item before have been read
                        if (j == 0 && outs[i] > 0 && !(ok = wait(o_empty + i, (outs[i] - 1) & 1))) break;
                    }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t s_at = tmem + i * 128, o_at = tmem + 256 + i * 128;
                        if (grow) {
#pragma unroll
                            for (int x = 0; x < kAttnKeys / 16; ++x)
                                mma_bf16_ts(o_at, s_at + x / 4 * 64 + x % 4 * 8, dv + x * k_step(true), desc_o,
                                            j > 0 || x > 0);
                            mma_commit(smem_u32(o_full + i));
                        }
                        if (score) {  // S = Q K^T
                            const uint64_t dq = operand_desc(smem_u32(smem + (twins ? 0 : i) * kTile), false);
#pragma unroll
                            for (int b = 0; b < DB; ++b)
#pragma unroll
                                for (int x = 0; x < 4; ++x)
                                    mma_bf16<1>(s_at, dq + b * (kAttnBlock >> 4) + x * k_step(false),
                                                dk + b * (kAttnBlock >> 4) + x * k_step(false), desc_s, b + x > 0);
                            mma_commit(smem_u32(s_full + i));
                        }
                        if (i == 1 || twins) {
                            mma_commit(smem_u32(empty + s));
                            if (e == count - 1) mma_commit(smem_u32(q_empty));
                        }
                    }
                    __syncwarp();
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                done[i] += n[i];
                outs[i] += n[i] > 0;
            }
        }
        if (elect_one()) {
            mma_commit(smem_u32(drained));
            mbar_wait_bounded(drained, 0, p.timeout_ns);
        }
        __syncwarp();
    } else {
        // a thread's row: r of tile i; its half of the row's keys, and of its columns
        constexpr int kHalf = D / 2;
        const int i = warp >> 3 & 1, half = warp >> 2 & 1, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_at = lanes + i * 128 + half * 64, o_at = lanes + 256 + i * 128 + half * kHalf;
        int done = 0, swaps = 0, joins = 0;  // steps, exchanges and joined twins so far
        uint32_t agreed = 0;
        bool ok = true;
        // Both warps of a row come to this barrier at the same places, whatever
        // their waits gave, and leave together.
        auto exchange = [&](float x, float& other) {
            float2* at = swap + ((swaps & 1) * 2 + i) * 256 + r;
            ++swaps;
            at[half * 128] = make_float2(x, ok ? 1.0f : 0.0f);
            asm volatile("bar.sync %0, 64;" ::"r"(1 + i * 4 + (warp & 3)) : "memory");
            const float2 theirs = at[(half ^ 1) * 128];
            other = theirs.x;
            return ok && theirs.y != 0.0f;
        };
        bool synced = false;
        for (int k = 0, end = 0; end == 0; ++k) {
            // (an item that one of them did not get, or did not finish, ends it for
            // both warps of a row, and for all where they will meet)
            ok = ok && take(k);
            if (p.persistent) {
                float nothing;
                ok = exchange(0.0f, nothing);
            } else {
                asm volatile(
                    "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
                    "bar.red.and.pred q, 9, 512, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                    : "=r"(agreed)
                    : "r"((uint32_t)ok)
                    : "memory");
                ok = agreed != 0;
            }
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            const AttnWork& w = items[k & 1];
            const AttnItem& a = w.a;
            end = w.end;
            if (end == 2) break;
            if (a.spares > 0) {
                if (rank == 0) {
                    clear_rows(p.y, p.ld_y, (int64_t)w.kvh * p.group * p.d, p.group * p.d, p.s.starts, p.s.n, p.s.tokens,
                               a.index, a.spares, threadIdx.x, kAttnRowWarps * 32);
                    clear_lse(p.lse, p.heads, w.kvh * p.group, p.group, p.s.starts, p.s.n, p.s.tokens, a.index, a.spares,
                              threadIdx.x, kAttnRowWarps * 32);
                }
                release(k);
                continue;
            }
            const int token = w.t0 + (w.twins ? 0 : i) * p.tile_tokens + r / p.group, head = w.kvh * p.group + r % p.group;
            const bool live = r < p.tile_tokens * p.group && token < a.n;
            const bool any_live = __any_sync(0xffffffffu, live);
            const int n = w.n[i];
            float m = minus_inf(), l = 0.0f;
            [[maybe_unused]] float before[FAR ? kHalf + 2 : 1];  // (indexed: in local memory)
            if (n > 0) {
                // the last key that the row sees (rows of nobody mask nothing)
                const int64_t last = (int64_t)a.m - 1;
                const int64_t see = !live      ? (int64_t)1 << 40
                                    : p.causal ? min(last, (int64_t)token + a.m - a.n)
                                               : last;
                bool together = true;
                [[maybe_unused]] auto join = [&](int upto) {  // the tiles before `upto`, whose products are done
                    if constexpr (FAR) {
                        if (!ok || !any_live) return;
                        tc_fence_after();
                        const float2 ml = join_tiles<kHalf>(before, o_at, m, l, upto == kAttnFold, upto == n);
                        m = ml.x, l = ml.y;
                        tc_fence_before();
                    }
                };
                for (int j = 0; j < n; ++j) {
                    ok = ok && wait(s_full + i, (done + j) & 1);
                    tc_fence_after();
                    float larger = m, other;
                    const int64_t key0 = (int64_t)(w.first + (w.twins ? 2 * j + i : j)) * kAttnKeys + 64 * half;
                    const bool masked = !__all_sync(0xffffffffu, see >= key0 + 63);
                    const int upto = (int)max((int64_t)-1, min(see - key0, (int64_t)64));
                    auto scores = [&](int c, float (&s)[32]) {  // 32 of this half's, where the row sees them
                        tmem_ld(s_at + 32 * c, s);
                        tmem_wait_ld(s);
                        if (masked) {
#pragma unroll
                            for (int x = 0; x < 32; ++x)
                                if (32 * c + x > upto) s[x] = minus_inf();
                        }
                    };
                    if (any_live && ok) {
                        float top[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float s[32];
                            scores(c, s);
                            float t[4];
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
                                t[q] = fmaxf(s[8 * q], s[8 * q + 1]);
#pragma unroll
                                for (int x = 2; x < 8; x += 2) t[q] = fmax3(t[q], s[8 * q + x], s[8 * q + x + 1]);
                            }
                            top[c] = fmaxf(fmax3(t[0], t[1], t[2]), t[3]);
                        }
                        larger = fmaxf(m, fmaxf(top[0], top[1]) * p.scale_log2);
                    }
                    together = exchange(larger, other);
                    if (!together) break;
                    if (any_live) {
                        larger = fmaxf(larger, other);
                        if (__any_sync(0xffffffffu, live && larger > m + kAttnSlack)) {
                            const float f = larger == m ? 1.0f : exp2_fast(m - larger);
                            l *= f;
                            m = larger;
                            if (j > 0) {
                                ok = wait(o_full + i, (done + j - 1) & 1);
                                if (!ok) continue;
                                tc_fence_after();
#pragma unroll 1
                                for (int c = 0; c < kHalf; c += 16) {
                                    float o[16];
                                    tmem_ld16(o_at + c, o);
#pragma unroll
                                    for (int x = 0; x < 16; ++x) o[x] *= f;
                                    tmem_st16(o_at + c, o);
                                }
                            }
                        }
                        const float shift = m == minus_inf() ? 0.0f : -m;
                        const float2 scale2 = make_float2(p.scale_log2, p.scale_log2), shift2 = make_float2(shift, shift);
                        float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            // (read again: kept from the maximum on, 64 scores leave
                            // too few registers for what follows)
                            float s[32];
                            scores(c, s);
                            uint32_t x16[16];
#pragma unroll
                            for (int x = 0; x < 16; ++x) {
                                float2 e = __ffma2_rn(make_float2(s[2 * x], s[2 * x + 1]), scale2, shift2);
                                e.x = exp2_fast(e.x);
                                e.y = exp2_fast(e.y);
                                sum[x & 1] = __fadd2_rn(sum[x & 1], e);
                                x16[x] = pack_bf16x2(e.x, e.y);
                            }
                            tmem_st(s_at + 16 * c, x16);
                        }
                        tmem_wait_st();
                        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(p_full + i);
                    if (FAR && (j + 1) % kAttnFold == 0 && j + 1 < n) {
                        ok = ok && wait(o_full + i, (done + j) & 1);
                        join(j + 1);
                    }
                }
                if (together) {
                    ok = ok && wait(o_full + i, (done + n - 1) & 1);
                    if (FAR && n > kAttnFold) join(n);
                    float other;
                    ok = exchange(l, other);
                    l = half ? other + l : l + other;
                    tc_fence_after();
                } else {
                    ok = false;
                }
                done += n;
            }
            const bool whole = p.split == 1;  // the row has no parts in other CTAs
            const bool joined = whole && w.twins;
            if (joined) {  // twin 1 leaves its sums to twin 0, where they lie
                if (i == 1) {
                    if (half == 0) {
                        stat[128 + r] = make_float2(m, l);
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0 && ok) mbar_arrive(join + (warp & 3));
                    }
                } else {
                    ok = ok && wait(join + (warp & 3), joins & 1);
                    tc_fence_after();
                    if (ok && any_live) {
                        const float2 twin = stat[128 + r];
                        const float top = fmaxf(m, twin.x), shift = top == minus_inf() ? 0.0f : top;
                        const float mine = exp2_fast(m - shift), theirs = exp2_fast(twin.x - shift);
                        const bool none = l == 0.0f, no_twin = twin.y == 0.0f;  // (what is not seen left nothing)
#pragma unroll 1
                        for (int c = 0; c < kHalf; c += 16) {
                            float o[16], z[16];
                            tmem_ld16(o_at + c, o);
                            tmem_ld16(o_at + 128 + c, z);
#pragma unroll
                            for (int x = 0; x < 16; ++x)
                                o[x] = fmaf(theirs, no_twin ? 0.0f : z[x], mine * (none ? 0.0f : o[x]));
                            tmem_st16(o_at + c, o);
                        }
                        tmem_wait_st();
                        l = fmaf(mine, l, theirs * twin.y);
                        m = top;
                    }
                }
                ++joins;
            }
            if (whole && ok && any_live && !(joined && i == 1)) {
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                uint32_t out[kHalf / 2];
#pragma unroll
                for (int c = 0; c < kHalf; c += 32) {
                    float o[32];
                    if (n > 0) {
                        tmem_ld(o_at + c, o);
                        tmem_wait_ld(o);
                    } else {
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] = 0.0f;
                    }
#pragma unroll
                    for (int x = 0; x < 32; x += 2) out[(c + x) / 2] = pack_bf16x2(o[x] * inv, o[x + 1] * inv);
                }
                if (l == 0.0f) {  // (0 times values that need not be finite)
#pragma unroll
                    for (int x = 0; x < kHalf / 2; ++x) out[x] = 0;
                }
                // 1 KB of rows at a time through shared memory, so that a store
                // covers whole lines (of a row a thread each store touched 32)
                constexpr int kVecs = kHalf / 8, kRows = 64 / kVecs;  // 16-byte vectors of a row; rows at a time
                uint8_t* const stage = stages + warp * 1024;
#pragma unroll 1
                for (int q = 0; q < 32; q += kRows) {
                    __syncwarp();
                    if (lane >= q && lane < q + kRows) {
#pragma unroll
                        for (int c = 0; c < kVecs; ++c)
                            *reinterpret_cast<uint4*>(stage + ((lane - q) * kVecs + (c ^ (lane & (kVecs - 1)))) * 16) =
                                make_uint4(out[4 * c], out[4 * c + 1], out[4 * c + 2], out[4 * c + 3]);
                    }
                    __syncwarp();
#pragma unroll
                    for (int z = lane; z < 64; z += 32) {
                        const int row = q + z / kVecs, c = z % kVecs;
                        const int rr = (warp & 3) * 32 + row, tok = w.t0 + i * p.tile_tokens + rr / p.group;
                        if (rr < p.tile_tokens * p.group && tok < a.n && half * kHalf + 8 * c < p.d)
                            *reinterpret_cast<uint4*>(
                                static_cast<__nv_bfloat16*>(p.y) + (int64_t)(a.q0 + tok) * p.ld_y +
                                (int64_t)(w.kvh * p.group + rr % p.group) * p.d + half * kHalf + 8 * c) =
                                *reinterpret_cast<const uint4*>(stage + (z - c + (c ^ (row & (kVecs - 1)))) * 16);
                    }
                }
                if (p.lse && live && half == 0)
                    p.lse[(int64_t)(a.q0 + token) * p.heads + head] = l == 0.0f ? minus_inf() : 0.69314718f * (m + log2f(l));
            }
            if (n > 0) {  // the outputs are read: the next item's may grow
                tc_fence_before();
                __syncwarp();
                if (lane == 0 && !(joined && i == 1)) {
                    mbar_arrive(o_empty + i);
                    if (joined) mbar_arrive(o_empty + 1);
                }
            }
            if (!whole) {
                // (one item, then: every product of this CTA is done, and the
                // ring's memory takes O)
                asm volatile("bar.sync 9, 512;" ::: "memory");
                float* part = reinterpret_cast<float*>(ring);  // [2][128][D], vectors of 4 swizzled by row
                if (half == 0) stat[i * 128 + r] = make_float2(m, ok ? l : 0.0f);
                if (n > 0 && ok) {
#pragma unroll 1
                    for (int c = 0; c < kHalf; c += 32) {
                        float o[32];
                        tmem_ld(o_at + c, o);
                        tmem_wait_ld(o);
#pragma unroll
                        for (int x = 0; x < 32; x += 4)
                            *reinterpret_cast<float4*>(part + (size_t)(i * 128 + r) * D +
                                                       (((half * kHalf + c + x) / 4) ^ (r & 7)) * 4) =
                                make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
                    }
                }
                cluster_sync();
                synced = true;
                constexpr int kVecs = D / 4, kMany = kAttnRowWarps * 32;
                const int rows = p.tile_tokens * p.group;
                auto peer = [&](const void* x, int q) { return peer_addr(smem_u32(x), (uint32_t)q); };
                for (int x = rank * kMany + (int)threadIdx.x; x < (w.twins ? 1 : 2) * rows * kVecs; x += p.split * kMany) {
                    const int tile = x / (rows * kVecs), row = x / kVecs % rows, c = x % kVecs;
                    const int tok = w.t0 + tile * p.tile_tokens + row / p.group;
                    if (tok >= a.n || 4 * c >= p.d) continue;
                    float top = minus_inf(), total_l = 0.0f;
                    float2 st[kAttnMostSplit][2];
#pragma unroll
                    for (int q = 0; q < kAttnMostSplit; ++q)
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            st[q][z] = make_float2(minus_inf(), 0.0f);
                            if (q >= p.split || (z == 1 && !w.twins)) continue;
                            asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];"
                                         : "=f"(st[q][z].x), "=f"(st[q][z].y)
                                         : "r"(peer(stat + (tile + z) * 128 + row, q))
                                         : "memory");
                            top = fmaxf(top, st[q][z].x);
                        }
                    const float shift = top == minus_inf() ? 0.0f : top;
                    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                    for (int q = 0; q < kAttnMostSplit; ++q)
#pragma unroll
                        for (int z = 0; z < 2; ++z)
                            if (st[q][z].y != 0.0f) {  // (a part without keys left nothing)
                                const float f = exp2_fast(st[q][z].x - shift);
                                const float4 v =
                                    ld_peer4(peer(part + (size_t)((tile + z) * 128 + row) * D + (c ^ (row & 7)) * 4, q));
                                total_l = fmaf(f, st[q][z].y, total_l);
                                o.x = fmaf(f, v.x, o.x), o.y = fmaf(f, v.y, o.y);
                                o.z = fmaf(f, v.z, o.z), o.w = fmaf(f, v.w, o.w);
                            }
                    const float inv = total_l == 0.0f ? 0.0f : 1.0f / total_l;
                    const int64_t to = (int64_t)(a.q0 + tok);
                    const int h = w.kvh * p.group + row % p.group;
                    *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p.y) + to * p.ld_y + (int64_t)h * p.d + 4 * c) =
                        make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
                    if (p.lse && c == 0)
                        p.lse[to * p.heads + h] = total_l == 0.0f ? minus_inf() : 0.69314718f * (shift + log2f(total_l));
                }
            }
            release(k);
        }
        __syncwarp();
        if (p.split > 1 && !synced) cluster_sync();
    }
    __syncwarp();
    if (p.split > 1 && warp >= kAttnRowWarps) cluster_sync();  // (the one that the rows' warps have had)
    tc_fence_before();
    __syncthreads();
    if (p.split > 1) cluster_sync();  // nobody leaves while its memory is read
    if (warp == kAttnProducts) tmem_free<1>(tmem, 512);
}

}  // namespace quasar
