// C ABI of attention.  Argument validation, launch plans and launches;
// declarations and contracts are in include/quasar.h.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "attention.h"
#include "host_launch.h"
#include "quasar.h"

namespace quasar {
const void* attention_kernel(int d, bool far);
int attention_threads();
size_t attention_smem(int d);
const void* attention_stats_kernel(int d);
const void* attention_grad_kernel(int d, bool keys, bool far);
int attention_grad_threads();
size_t attention_grad_smem(int d);
}  // namespace quasar

namespace {

using namespace quasar;

constexpr float kLog2e = 1.44269504f;

// [rows, heads, d] bf16 as it lies in columns of a matrix: tiles of 64 columns
// of a head, `box_heads` heads and `box_rows` rows.
quasar_status head_map(const void* p, int64_t rows, int64_t heads, int64_t d, int64_t ld, int box_heads, int box_rows,
                       CUtensorMap* map)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return QUASAR_ERR_UNSUPPORTED;
    const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)rows};
    const cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)ld * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows};
    const cuuint32_t step[3] = {1, 1, 1};
    const CUresult r =
        encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(p), dims, strides, box, step,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? QUASAR_OK : QUASAR_ERR_INVALID_ARG;
}

bool valid_heads(int64_t heads, int64_t kv_heads, int64_t d)
{
    return heads >= 1 && kv_heads >= 1 && heads % kv_heads == 0 && d >= 8 && d % 8 == 0 &&
           heads <= (int64_t(1) << 31) / d;
}

bool valid_sequences(const int32_t* starts, const int32_t* key_starts, int64_t n)
{
    if (n < 0 || n > (int64_t(1) << 24) || !aligned(starts, 4) || !aligned(key_starts, 4)) return false;
    return n == 1 || (starts && key_starts);
}

}  // namespace

extern "C" {

quasar_status quasar_attention(const void* q, int64_t ld_q, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                               int64_t tokens, int64_t keys, int64_t heads, int64_t kv_heads, int64_t head_dim,
                               const int32_t* starts, const int32_t* key_starts, int64_t sequences, int causal,
                               float scale, void* y, int64_t ld_y, float* lse, quasar_stream_t stream)
{
    if (!valid_heads(heads, kv_heads, head_dim) || !valid_sequences(starts, key_starts, sequences))
        return QUASAR_ERR_INVALID_ARG;
    if (!valid_operand(q, tokens, heads * head_dim, ld_q) || !valid_operand(k, keys, kv_heads * head_dim, ld_k) ||
        !valid_operand(v, keys, kv_heads * head_dim, ld_v) || !valid_operand(y, tokens, heads * head_dim, ld_y))
        return QUASAR_ERR_INVALID_ARG;
    if (!(scale > 0.0f) || !std::isfinite(scale * kLog2e) || (causal != 0 && causal != 1) || !aligned(lse, 4))
        return QUASAR_ERR_INVALID_ARG;
    if (head_dim > 128 || heads / kv_heads > kAttnRows) return QUASAR_ERR_UNSUPPORTED;
    if (tokens == 0) return QUASAR_OK;
    const Bytes b_q(q, tokens, heads * head_dim, ld_q, 2), b_k(k, keys, kv_heads * head_dim, ld_k, 2);
    const Bytes b_v(v, keys, kv_heads * head_dim, ld_v, 2), b_y(y, tokens, heads * head_dim, ld_y, 2);
    const Bytes b_lse(lse, tokens * heads, 4), b_s(starts, sequences + 1, 4), b_ks(key_starts, sequences + 1, 4);
    for (const Bytes* in : {&b_q, &b_k, &b_v, &b_s, &b_ks})
        if (overlaps(b_y, *in) || overlaps(b_lse, *in)) return QUASAR_ERR_INVALID_ARG;
    if (overlaps(b_y, b_lse)) return QUASAR_ERR_INVALID_ARG;
    AttnParams p{};
    int n_sm = 0;
    quasar_status st = host_device(&n_sm, &p.status);
    if (st != QUASAR_OK) return st;
    p.s = AttnSequences{starts, key_starts, (int)sequences, (int)tokens, (int)keys};
    p.heads = (int)heads;
    p.kv_heads = (int)kv_heads;
    p.group = (int)(heads / kv_heads);
    p.d = (int)head_dim;
    p.tile_tokens = kAttnRows / p.group;
    p.causal = causal;
    p.scale_log2 = scale * kLog2e;
    p.y = y;
    p.ld_y = ld_y;
    p.lse = lse;
    p.timeout_ns = host_timeout_ns();
    p.force_timeout_ns = host_forced_timeout_ns();
    // sequences of n_i tokens have ceil(n_i / span) items, and one more clears
    // the rows of none
    const int64_t items = tokens / (2 * p.tile_tokens) + sequences + 1;
    if (items * kv_heads * kAttnMostSplit > (int64_t(1) << 31) - 1) return QUASAR_ERR_UNSUPPORTED;
    p.items = (int)items;
    const int64_t work = std::max<int64_t>(1, items - 1) * kv_heads;  // (the one more aside)
    const int64_t tiles = keys / std::max<int64_t>(1, sequences) / kAttnKeys;
    p.split = 1;
    const void* fn = attention_kernel(p.d, keys > (int64_t)kAttnFold * kAttnKeys);  // (no sequence has more)
    const size_t smem = attention_smem(p.d);
    // more items than SMs: their CTAs take them from one another (not so, 16 x 512
    // tokens 107 us against 78, 512 queries of 512 keys 472 against 229).  Fewer:
    // as many CTAs share one's keys as fill the device, four key tiles each (two:
    // two queries of 1,024 keys 22.7 us against 12.3; eight: 13.9)
    p.persistent = work > n_sm;
    while (p.split < kAttnMostSplit && work * p.split < n_sm && tiles >= 4 * p.split) p.split *= 2;
    const int64_t ctas = items * kv_heads * p.split;
    if ((st = head_map(q, tokens, heads, head_dim, ld_q, p.group, p.tile_tokens, &p.q)) != QUASAR_OK) return st;
    // (without keys no copy is made: any valid map will do)
    const bool none = keys == 0;
    if ((st = head_map(none ? q : k, none ? tokens : keys, none ? heads : kv_heads, head_dim, none ? ld_q : ld_k, 1,
                       kAttnKeys, &p.k)) != QUASAR_OK)
        return st;
    if ((st = head_map(none ? q : v, none ? tokens : keys, none ? heads : kv_heads, head_dim, none ? ld_q : ld_v, 1,
                       kAttnKeys, &p.v)) != QUASAR_OK)
        return st;
    return launch(fn, &p, dim3((unsigned)ctas), attention_threads(), p.split, smem, stream);
}

quasar_status quasar_attention_backward_workspace(int64_t tokens, int64_t heads, int64_t* bytes)
{
    if (!bytes || !valid_shape(tokens, heads, heads)) return QUASAR_ERR_INVALID_ARG;
    *bytes = 8 * tokens * heads;
    return QUASAR_OK;
}

quasar_status quasar_attention_backward(const void* dy, int64_t ld_dy, const void* q, int64_t ld_q, const void* k,
                                        int64_t ld_k, const void* v, int64_t ld_v, const void* y, int64_t ld_y,
                                        const float* lse, int64_t tokens, int64_t keys, int64_t heads, int64_t kv_heads,
                                        int64_t head_dim, const int32_t* starts, const int32_t* key_starts,
                                        int64_t sequences, int causal, float scale, void* dq, int64_t ld_dq, void* dk,
                                        int64_t ld_dk, void* dv, int64_t ld_dv, void* workspace,
                                        int64_t workspace_bytes, quasar_stream_t stream)
{
    if (!valid_heads(heads, kv_heads, head_dim) || !valid_sequences(starts, key_starts, sequences))
        return QUASAR_ERR_INVALID_ARG;
    const int64_t cols = heads * head_dim, kv_cols = kv_heads * head_dim;
    if (!valid_operand(dy, tokens, cols, ld_dy) || !valid_operand(q, tokens, cols, ld_q) ||
        !valid_operand(y, tokens, cols, ld_y) || !valid_operand(k, keys, kv_cols, ld_k) ||
        !valid_operand(v, keys, kv_cols, ld_v))
        return QUASAR_ERR_INVALID_ARG;
    if ((dk == nullptr) != (dv == nullptr)) return QUASAR_ERR_INVALID_ARG;
    if ((dq && !valid_operand(dq, tokens, cols, ld_dq)) ||
        (dk && (!valid_operand(dk, keys, kv_cols, ld_dk) || !valid_operand(dv, keys, kv_cols, ld_dv))))
        return QUASAR_ERR_INVALID_ARG;
    if (!(scale > 0.0f) || !std::isfinite(scale * kLog2e) || (causal != 0 && causal != 1)) return QUASAR_ERR_INVALID_ARG;
    if (!aligned(lse, 4) || (tokens > 0 && !lse)) return QUASAR_ERR_INVALID_ARG;
    if (head_dim > 128 || heads / kv_heads > kAttnRows) return QUASAR_ERR_UNSUPPORTED;
    const int64_t need = 8 * tokens * heads;
    if (workspace_bytes < need || (need > 0 && (!workspace || !aligned(workspace, 16)))) return QUASAR_ERR_INVALID_ARG;
    const Bytes outs[] = {Bytes(dq, tokens, cols, ld_dq, 2), Bytes(dk, keys, kv_cols, ld_dk, 2),
                          Bytes(dv, keys, kv_cols, ld_dv, 2), Bytes(workspace, need, 1)};
    const Bytes ins[] = {Bytes(dy, tokens, cols, ld_dy, 2),   Bytes(q, tokens, cols, ld_q, 2),
                         Bytes(k, keys, kv_cols, ld_k, 2),    Bytes(v, keys, kv_cols, ld_v, 2),
                         Bytes(y, tokens, cols, ld_y, 2),     Bytes(lse, tokens * heads, 4),
                         Bytes(starts, sequences + 1, 4),     Bytes(key_starts, sequences + 1, 4)};
    for (int i = 0; i < 4; ++i) {
        for (const Bytes& in : ins)
            if (overlaps(outs[i], in)) return QUASAR_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (overlaps(outs[i], outs[j])) return QUASAR_ERR_INVALID_ARG;
    }
    const bool want_q = dq && tokens > 0, want_k = dk && keys > 0;
    if (!want_q && !want_k) return QUASAR_OK;
    AttnGradParams p{};
    int n_sm = 0;
    quasar_status st = host_device(&n_sm, &p.status);
    if (st != QUASAR_OK) return st;
    p.s = AttnSequences{starts, key_starts, (int)sequences, (int)tokens, (int)keys};
    p.heads = (int)heads;
    p.kv_heads = (int)kv_heads;
    p.group = (int)(heads / kv_heads);
    p.d = (int)head_dim;
    p.tile_tokens = kAttnRows / p.group;
    p.causal = causal;
    p.scale = scale;
    p.scale_log2 = scale * kLog2e;
    p.stats = static_cast<const float2*>(workspace);
    p.timeout_ns = host_timeout_ns();
    p.force_timeout_ns = host_forced_timeout_ns();
    const int64_t key_items = keys / kAttnRows + sequences + 1, query_items = tokens / p.tile_tokens + sequences + 1;
    constexpr int64_t kMost = (int64_t(1) << 31) - 1;
    const int lanes = p.d <= 64 ? 8 : 16;
    if (key_items * kv_heads > kMost || query_items * kv_heads > kMost ||
        tokens * heads > kMost * 256 / lanes)
        return QUASAR_ERR_UNSUPPORTED;
    const size_t smem = attention_grad_smem(p.d);
    if (tokens > 0) {
        AttnStatsParams s{dy, ld_dy, y, ld_y, lse, tokens, p.heads, p.d, static_cast<float2*>(workspace)};
        if ((st = launch(attention_stats_kernel(p.d), &s, dim3((unsigned)((tokens * heads * lanes + 255) / 256)), 256, 1,
                         0, stream)) != QUASAR_OK)
            return st;
    }
    // (a side without rows is not copied: any valid map will do)
    auto map = [&](bool of_keys, const void* ptr, int64_t ld, int box_heads, int box_rows, CUtensorMap* to) {
        if (of_keys ? keys == 0 : tokens == 0)
            return of_keys ? head_map(q, tokens, heads, head_dim, ld_q, 1, 1, to)
                           : head_map(k, keys, kv_heads, head_dim, ld_k, 1, 1, to);
        return head_map(ptr, of_keys ? keys : tokens, of_keys ? kv_heads : heads, head_dim, ld, box_heads, box_rows, to);
    };
    if (want_k) {
        p.items = (int)key_items;
        p.d1 = dk, p.ld_d1 = ld_dk, p.d2 = dv, p.ld_d2 = ld_dv;
        if ((st = map(true, k, ld_k, 1, kAttnRows, &p.x1)) != QUASAR_OK ||
            (st = map(true, v, ld_v, 1, kAttnRows, &p.x2)) != QUASAR_OK ||
            (st = map(false, q, ld_q, p.group, p.tile_tokens, &p.z1)) != QUASAR_OK ||
            (st = map(false, dy, ld_dy, p.group, p.tile_tokens, &p.z2)) != QUASAR_OK ||
            (st = launch(attention_grad_kernel(p.d, true, tokens > (int64_t)kGradFold * p.tile_tokens), &p, dim3((unsigned)(key_items * kv_heads)),
                         attention_grad_threads(), 1, smem, stream)) != QUASAR_OK)
            return st;
    }
    if (want_q) {
        p.items = (int)query_items;
        p.d1 = dq, p.ld_d1 = ld_dq, p.d2 = nullptr, p.ld_d2 = 0;
        if ((st = map(false, q, ld_q, p.group, p.tile_tokens, &p.x1)) != QUASAR_OK ||
            (st = map(false, dy, ld_dy, p.group, p.tile_tokens, &p.x2)) != QUASAR_OK ||
            (st = map(true, k, ld_k, 1, kGradCols, &p.z1)) != QUASAR_OK ||
            (st = map(true, v, ld_v, 1, kGradCols, &p.z2)) != QUASAR_OK ||
            (st = launch(attention_grad_kernel(p.d, false, keys > (int64_t)kGradFold * kGradCols), &p, dim3((unsigned)(query_items * kv_heads)),
                         attention_grad_threads(), 1, smem, stream)) != QUASAR_OK)
            return st;
    }
    return QUASAR_OK;
}

}  // extern "C"
