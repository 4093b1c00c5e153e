// Embedding: rows of a table by token, and the table's gradient.
//
//   y[t] = scale table[id_t] + residual[t]
//   dtable[v] = scale sum over the t with id_t = v of dy[t]
//
// The gradient's sums have one order, whatever the timing: the tokens are
// sorted by id (stable, so a row's tokens stay in their order), every whole
// chunk of 32 sorted tokens that share an id is summed first (a frequent
// token's rows are then spread over the device), and each row of the table
// adds up its tokens' rows and chunks.  A table's row without tokens is
// written with zeros by the CTA that it belongs to: no pass clears the table
// first.
#pragma once

#include "cluster.cuh"
#include "layers.h"
#include "row_access.cuh"

namespace quasar {

// Token t's row of the table, or -1.
__device__ __forceinline__ int64_t id_at(const void* ids, int wide, int64_t t, int64_t vocab)
{
    const int64_t id = wide ? static_cast<const long long*>(ids)[t] : static_cast<const int*>(ids)[t];
    return id >= 0 && id < vocab ? id : -1;
}

// 4 tokens and 2,048 columns a CTA, so that four rows are on their way at once:
// 16384 tokens of 4096 bf16 38 us, 7.0 TB/s (frequent rows come from L2), 0.97 of
// the copy rate's 37 (a row a CTA 49 us).
template <bool VECTORS, bool WIDE>
__global__ void __launch_bounds__(kEmbedThreads) k_embedding(const __grid_constant__ EmbedParams p)
{
    wait_for_previous_grid();
    const int64_t t0 = (int64_t)blockIdx.x * kEmbedTokens;
    const int64_t c0 = (int64_t)blockIdx.y * kEmbedCols;
    const int cols = (int)(p.width - c0 < kEmbedCols ? p.width - c0 : kEmbedCols);
    Raw8<WIDE> raw[kEmbedTokens], res[kEmbedTokens];
#pragma unroll
    for (int q = 0; q < kEmbedTokens; ++q) {
        const int64_t id = t0 + q < p.tokens ? id_at(p.ids, p.ids_64, t0 + q, p.vocab) : -1;
        load_raw<kEmbedThreads, VECTORS>(
            raw[q],
            static_cast<const uint8_t*>(row_of(p.table, p.table_f32, id < 0 ? 0 : id, p.ld_table)) +
                c0 * (p.table_f32 ? 4 : 2),
            p.table_f32, threadIdx.x, 0, id < 0 ? 0 : cols);
        if (p.residual)
            load_raw<kEmbedThreads, VECTORS>(
                res[q], static_cast<const uint8_t*>(row_of(p.residual, p.y_f32, t0 + q, p.ld_res)) + c0 * (p.y_f32 ? 4 : 2),
                p.y_f32, threadIdx.x, 0, t0 + q < p.tokens ? cols : 0);
    }
#pragma unroll
    for (int q = 0; q < kEmbedTokens; ++q) {
        if (t0 + q >= p.tokens) break;
        float v[8], r[8];
        unpack_raw(raw[q], p.table_f32, v);
        if (p.residual) {
            unpack_raw(res[q], p.y_f32, r);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(p.scale, v[i], r[i]);
        store_row<kEmbedThreads, VECTORS>(
            static_cast<uint8_t*>(row_of(p.y, p.y_f32, t0 + q, p.ld_y)) + c0 * (p.y_f32 ? 4 : 2), p.y_f32,
            threadIdx.x, 0, cols, v);
    }
}

// -- the tokens' order -------------------------------------------------------------

// Stable sort of (id, place) by id, 9 bits a pass from the lowest, by one
// cluster in one launch.  A warp keeps a contiguous share of the list; the
// rank of an entry is what lies before its bin, before its CTA, before its
// warp and before it in its warp.  (n is small beside the rows it sorts: a
// token's row of 4096 is 8 KB, its entry 8 bytes a pass: 16384 ids of 131072 22 us
// of the gradient's 240, 11 a pass.)
__global__ void __launch_bounds__(kSortThreads) k_sort_ids(const __grid_constant__ SortParams p)
{
    constexpr int kBins = 1 << kSortBits, kWarps = kSortThreads / 32;
    extern __shared__ uint8_t smem_raw[];
    uint32_t* count = reinterpret_cast<uint32_t*>(smem_raw);  // [warps][bins]
    uint32_t* total = count + kWarps * kBins;                 // [bins], read by the cluster
    uint32_t* scan = total + kBins;                           // [kBins / 32]
    uint32_t* halves = scan + kBins / 32;                     // [bins]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = p.ctas > 1 ? (int)cluster_rank() : 0;
    const int64_t gw = rank * kWarps + warp, all = (int64_t)p.ctas * kWarps;
    const int from = (int)(p.n * gw / all), to = (int)(p.n * (gw + 1) / all);
    const bool held = to - from <= 128;  // 4 entries a lane, kept between a pass's two walks
    uint32_t* mine = count + warp * kBins;
    // a bin's column of counts, half of the warps each
    const int bin = threadIdx.x % kBins, part = threadIdx.x / kBins;
    static_assert(kSortThreads == 2 * kBins, "two threads a bin");
    uint32_t* column = count + part * (kWarps / 2) * kBins + bin;
    wait_for_previous_grid();

    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = pass * kSortBits;
        const int in = (p.passes - pass) & 1, out = in ^ 1;  // (the last pass writes to 0)
        uint32_t key[4], place[4];
        auto load = [&](int i0) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = i0 + 32 * q + lane;
                key[q] = 0, place[q] = (uint32_t)i;
                if (i >= to) continue;
                if (pass == 0) {
                    const int64_t id = id_at(p.ids, p.ids_64, i, p.vocab);
                    key[q] = (uint32_t)(id < 0 ? p.vocab : id);
                } else {
                    key[q] = __ldcg(p.keys[in] + i);
                    place[q] = __ldcg(p.places[in] + i);
                }
            }
        };
        for (int b = threadIdx.x; b < kWarps * kBins / 4; b += kSortThreads)
            reinterpret_cast<uint4*>(count)[b] = make_uint4(0, 0, 0, 0);
        load(from);
        __syncthreads();
        for (int i0 = from; i0 < to; i0 += 128) {
            if (i0 > from) load(i0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (i0 + 32 * q >= to) break;
                const bool live = i0 + 32 * q + lane < to;
                const uint32_t digit = live ? key[q] >> shift & (kBins - 1) : kBins;
                const uint32_t same = __match_any_sync(0xffffffffu, digit);
                if (live && (same & ((1u << lane) - 1)) == 0) mine[digit] += __popc(same);
                __syncwarp();
            }
        }
        __syncthreads();
        // a bin's counts become what its warps before have
        uint32_t sum = 0;
#pragma unroll
        for (int w = 0; w < kWarps / 2; ++w) {
            const uint32_t c = column[w * kBins];
            column[w * kBins] = sum;
            sum += c;
        }
        if (part == 0) halves[bin] = sum;
        __syncthreads();
        if (part == 1) total[bin] = halves[bin] + sum;
        __syncthreads();
        if (p.ctas > 1) cluster_sync();
        uint32_t whole = 0, before = 0;  // this bin's entries: all, and in the CTAs before
        if (p.ctas > 1) {
            uint32_t n[kSortCtas];
#pragma unroll
            for (int c = 0; c < kSortCtas; ++c) {
                n[c] = 0;
                if (c < p.ctas)
                    asm volatile("ld.shared::cluster.u32 %0, [%1];"
                                 : "=r"(n[c])
                                 : "r"(peer_addr(smem_u32(total + bin), (uint32_t)c))
                                 : "memory");
            }
#pragma unroll
            for (int c = 0; c < kSortCtas; ++c) {
                whole += n[c];
                if (c < rank) before += n[c];
            }
        } else {
            whole = total[bin];
        }
        uint32_t upto = whole;  // inclusive sum over the bins
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        if (part == 0 && lane == 31) scan[warp] = upto;
        __syncthreads();
        uint32_t base = upto - whole + before + (part ? halves[bin] : 0);
        for (int w = 0; w < bin / 32; ++w) base += scan[w];
#pragma unroll
        for (int w = 0; w < kWarps / 2; ++w) column[w * kBins] += base;
        __syncthreads();
        for (int i0 = from; i0 < to; i0 += 128) {
            if (!held) load(i0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (i0 + 32 * q >= to) break;
                const bool live = i0 + 32 * q + lane < to;
                const uint32_t digit = live ? key[q] >> shift & (kBins - 1) : kBins;
                const uint32_t same = __match_any_sync(0xffffffffu, digit);
                const uint32_t earlier = __popc(same & ((1u << lane) - 1));
                const uint32_t at = live ? mine[digit] + earlier : 0;
                __syncwarp();
                if (live) {
                    if (earlier == 0) mine[digit] += __popc(same);
                    p.keys[out][at] = key[q];
                    p.places[out][at] = place[q];
                }
                __syncwarp();
            }
        }
        // the next pass reads what the other CTAs wrote (from L2)
        __threadfence();
        __syncthreads();
        if (p.ctas > 1) cluster_sync();
    }
}

// -- the gradient ------------------------------------------------------------------

// sum += the rows of the tokens places[i] .. places[end - 1], N on their way at
// once.
template <int N, bool VECTORS, bool WIDE>
__device__ __forceinline__ void add_rows(float (&sum)[8], const EmbedGradParams& p, const uint32_t* places, int i, int end,
                                         int64_t c0, int cols)
{
    const uint8_t* dy = static_cast<const uint8_t*>(p.dy) + c0 * (p.dy_f32 ? 4 : 2);
    for (; i < end; i += N) {
        Raw8<WIDE> raw[N];
#pragma unroll
        for (int q = 0; q < N; ++q)
            load_raw<kEmbedThreads, VECTORS>(raw[q],
                                             row_of(static_cast<const void*>(dy), p.dy_f32,
                                                    places[min(i + q, end - 1)], p.ld_dy),
                                             p.dy_f32, threadIdx.x, 0, i + q < end ? cols : 0);
#pragma unroll
        for (int q = 0; q < N; ++q) {
            float v[8];
            unpack_raw(raw[q], p.dy_f32, v);
#pragma unroll
            for (int x = 0; x < 8; ++x) sum[x] += v[x];
        }
    }
}

// Sums of whole chunks of sorted tokens that share an id: 13 us for 16384 tokens
// of 4096 (in chunks of 128, a batch of rows after the other, 52 us).
template <bool VECTORS, bool WIDE>
__global__ void __launch_bounds__(kEmbedThreads) k_embedding_chunks(const __grid_constant__ EmbedGradParams p)
{
    __shared__ uint32_t places[kRunChunk];
    wait_for_previous_grid();
    const int i0 = (int)blockIdx.x * kRunChunk;
    const uint32_t id = p.keys[i0];
    if (threadIdx.x < kRunChunk) places[threadIdx.x] = p.places[i0 + threadIdx.x];
    if (id >= p.vocab || id != p.keys[i0 + kRunChunk - 1]) return;
    __syncthreads();
    const int64_t c0 = (int64_t)blockIdx.y * kEmbedCols;
    const int cols = (int)(p.width - c0 < kEmbedCols ? p.width - c0 : kEmbedCols);
    float sum[8] = {};
    add_rows<WIDE ? 8 : 16, VECTORS, WIDE>(sum, p, places, 0, kRunChunk, c0, cols);
    float* to = p.sums + (int64_t)blockIdx.x * p.width + c0;
    store_row<kEmbedThreads, VECTORS>(to, true, threadIdx.x, 0, cols, sum);
}

// First of the sorted keys in [from, to) that is not below `key`.
__device__ __forceinline__ int lower_bound(const uint32_t* keys, int from, int to, uint32_t key)
{
    while (from < to) {
        const int mid = from + (to - from) / 2;
        if (keys[mid] < key)
            from = mid + 1;
        else
            to = mid;
    }
    return from;
}

// kEmbedRows rows of the table by 2,048 columns a CTA.  Where most of a large
// table's rows have no token, bound by writing the gradient (131072 x 4096 bf16,
// 16384 tokens: 214 us, 5.2 TB/s of DRAM).  Rows that have tokens come one after the
// other, each a wait for its places and then for its rows of dy: 16384 tokens over
// every row of 4096 x 4096 140 us with the sort, 150 over 192 x 256 (3 CTAs) 103 us.
// 8003 x 1003 fp32 has 126 CTAs, fewer than the SMs, and stores single elements: 33 us
// with the sort, where its bytes take 5.
template <bool VECTORS, bool WIDE>
__global__ void __launch_bounds__(kEmbedThreads) k_embedding_grad(const __grid_constant__ EmbedGradParams p)
{
    __shared__ int ends[kEmbedRows + 1];  // where each row's tokens start
    wait_for_previous_grid();
    const int64_t v0 = (int64_t)blockIdx.x * kEmbedRows;
    const int rows = (int)(p.vocab - v0 < kEmbedRows ? p.vocab - v0 : kEmbedRows);
    const int64_t c0 = (int64_t)blockIdx.y * kEmbedCols;
    const int cols = (int)(p.width - c0 < kEmbedCols ? p.width - c0 : kEmbedCols);
    if (threadIdx.x <= rows) ends[threadIdx.x] = lower_bound(p.keys, 0, p.n, (uint32_t)(v0 + threadIdx.x));
    __syncthreads();
    if (p.add && ends[0] == ends[rows]) return;
    uint8_t* const first = static_cast<uint8_t*>(row_of(p.dtable, p.f32, v0, p.ld)) + c0 * (p.f32 ? 4 : 2);
    const int64_t pitch = p.ld * (p.f32 ? 4 : 2);
    if (!p.add) {  // the rows without tokens
        uint8_t* row = first;
        if (VECTORS && (int)threadIdx.x * 8 + 8 <= cols) {
            row += threadIdx.x * (p.f32 ? 32 : 16);
            const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll 4
            for (int r = 0; r < rows; ++r, row += pitch)
                if (ends[r] == ends[r + 1]) {
                    __stcs(reinterpret_cast<uint4*>(row), zero);
                    if (p.f32) __stcs(reinterpret_cast<uint4*>(row) + 1, zero);
                }
        } else {
            const float zeros[8] = {};
            for (int r = 0; r < rows; ++r, row += pitch)
                if (ends[r] == ends[r + 1]) store_row<kEmbedThreads, VECTORS>(row, p.f32, threadIdx.x, 0, cols, zeros);
        }
    }
    int i = ends[0];
#pragma unroll 1
    for (int r = 0; r < rows; ++r) {
        const int end = ends[r + 1];
        if (i == end) continue;
        uint8_t* const row = first + r * pitch;
        float sum[8] = {};
        // up to the first whole chunk, the chunks, and from the last on
        const int head = min(end, (i + kRunChunk - 1) / kRunChunk * kRunChunk);
        add_rows<8, VECTORS, WIDE>(sum, p, p.places, i, head, c0, cols);
        const int tail = max(head, end / kRunChunk * kRunChunk);
#pragma unroll 4
        for (int q = head / kRunChunk; q < tail / kRunChunk; ++q) {
            float v[8];
            load_floats<kEmbedThreads, VECTORS>(v, p.sums + (int64_t)q * p.width + c0, threadIdx.x, 0, cols, 0.0f);
#pragma unroll
            for (int x = 0; x < 8; ++x) sum[x] += v[x];
        }
        add_rows<8, VECTORS, WIDE>(sum, p, p.places, tail, end, c0, cols);
        i = end;
#pragma unroll
        for (int x = 0; x < 8; ++x) sum[x] *= p.scale;
        if (p.add) {
            Raw8<WIDE> raw;
            float v[8];
            load_raw<kEmbedThreads, VECTORS>(raw, row, p.f32, threadIdx.x, 0, cols);
            unpack_raw(raw, p.f32, v);
#pragma unroll
            for (int x = 0; x < 8; ++x) sum[x] += v[x];
        }
        store_row<kEmbedThreads, VECTORS>(row, p.f32, threadIdx.x, 0, cols, sum);
    }
}

}  // namespace quasar
