// C ABI of the layers between the products: embedding and layer norm with
// their gradients.  Argument validation, launch plans and launches;
// declarations and contracts are in include/quasar.h.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "host_launch.h"
#include "layers.h"
#include "quasar.h"

namespace quasar {
const void* layer_norm_kernel(int64_t cols, bool vectors, bool grad, bool wide, int* threads, int* rows, int* per_sm);
const void* layer_norm_ring_kernel(int64_t cols, bool grad, bool wide, int* threads, int* per_sm);
int layer_norm_slots(uint32_t slot_bytes, int threads, int per_sm, size_t* smem);
const void* layer_norm_long_kernel();
const void* layer_norm_grad_long_kernel();
const void* layer_norm_grad_columns_kernel();
const void* part_sum_kernel();
const void* embedding_kernel(bool vectors, bool wide);
const void* sort_ids_kernel();
size_t sort_ids_smem();
const void* embedding_chunks_kernel(bool vectors, bool wide);
const void* embedding_grad_kernel(bool vectors, bool wide);
}  // namespace quasar

namespace {

using namespace quasar;

// Whether a matrix's rows start at 16-byte boundaries (NULL: yes).
bool vector_rows(const void* p, int64_t rows, int64_t ld, quasar_dtype dtype)
{
    return aligned(p, 16) && (!p || rows <= 1 || ld * dtype_size(dtype) % 16 == 0);
}

bool valid_matrix(const void* p, int64_t rows, int64_t cols, int64_t ld, quasar_dtype dtype)
{
    return valid_dtype(dtype) && valid_shape(rows, cols, ld) &&
           (rows == 0 || cols == 0 || (p && aligned(p, (uintptr_t)dtype_size(dtype))));
}

// -- layer norm ------------------------------------------------------------------

constexpr int64_t kColumnParts = 64;  // shares of the rows, where a row is too long for registers

// CTAs of the gradient's kernel: each leaves a partial sum of dw and db.
quasar_status norm_parts(int64_t rows, int64_t cols, int64_t* parts)
{
    int n_sm = 0, threads = 0, at_once = 1, per_sm = 1;
    unsigned int* status = nullptr;
    const quasar_status st = host_device(&n_sm, &status);
    if (st != QUASAR_OK) return st;
    if (layer_norm_ring_kernel(cols, true, false, &threads, &per_sm))  // (whichever kernel it will be)
        *parts = std::min<int64_t>(rows, (int64_t)n_sm * per_sm);
    else if (layer_norm_kernel(cols, true, true, false, &threads, &at_once, &per_sm))
        *parts = std::min<int64_t>((rows + at_once - 1) / at_once, (int64_t)n_sm * per_sm);
    else
        *parts = std::min(rows, kColumnParts);
    return QUASAR_OK;
}

// One part is the sum itself.
int64_t norm_workspace(int64_t parts, int64_t cols) { return parts <= 1 ? 0 : 2 * parts * cols * 4; }

// -- embedding -------------------------------------------------------------------

int64_t up16(int64_t n) { return (n + 15) & ~(int64_t)15; }

// Two lists of (id, place), and the chunks' sums.
int64_t embedding_workspace(int64_t tokens, int64_t width)
{
    return 4 * up16(4 * tokens) + 4 * (tokens / kRunChunk) * width;
}

bool valid_ids(const void* ids, quasar_index_type type, int64_t tokens)
{
    if (type != QUASAR_I32 && type != QUASAR_I64) return false;
    return tokens == 0 || (ids && aligned(ids, type == QUASAR_I64 ? 8 : 4));
}

}  // namespace

extern "C" {

quasar_status quasar_layer_norm(const void* x, quasar_dtype x_dtype, int64_t ld_x, const float* weight,
                                const float* bias, int64_t rows, int64_t cols, int center, float eps, void* y,
                                quasar_dtype y_dtype, int64_t ld_y, float* stats, quasar_stream_t stream)
{
    if (!valid_matrix(x, rows, cols, ld_x, x_dtype) || !valid_matrix(y, rows, cols, ld_y, y_dtype))
        return QUASAR_ERR_INVALID_ARG;
    if (!(eps >= 0.0f) || !std::isfinite(eps) || (center != 0 && center != 1)) return QUASAR_ERR_INVALID_ARG;
    if (!aligned(weight, 4) || !aligned(bias, 4) || !aligned(stats, 4)) return QUASAR_ERR_INVALID_ARG;
    if (cols == 0 && rows > 0) return QUASAR_ERR_INVALID_ARG;  // (a mean of nothing)
    if (rows == 0) return QUASAR_OK;
    const Bytes b_x(x, rows, cols, ld_x, dtype_size(x_dtype)), b_y(y, rows, cols, ld_y, dtype_size(y_dtype));
    const Bytes b_w(weight, cols, 4), b_b(bias, cols, 4), b_s(stats, 2 * rows, 4);
    // y may take x's place, in exactly its place
    if ((!(b_x == b_y) && overlaps(b_x, b_y)) || overlaps(b_y, b_w) || overlaps(b_y, b_b) || overlaps(b_y, b_s) ||
        overlaps(b_s, b_x) || overlaps(b_s, b_w) || overlaps(b_s, b_b))
        return QUASAR_ERR_INVALID_ARG;
    int n_sm = 0;
    unsigned int* status = nullptr;
    const quasar_status st = host_device(&n_sm, &status);
    if (st != QUASAR_OK) return st;
    NormParams p{x, ld_x, x_dtype == QUASAR_F32, weight, bias, rows, cols, center, eps,
                 y, ld_y, y_dtype == QUASAR_F32, stats, 0, host_timeout_ns(), host_forced_timeout_ns(), status};
    const bool vectors = vector_rows(x, rows, ld_x, x_dtype) && vector_rows(y, rows, ld_y, y_dtype) &&
                         aligned(weight, 16) && aligned(bias, 16);
    int threads = 0, at_once = 0, per_sm = 0;
    const bool wide = x_dtype == QUASAR_F32;
    if (vectors) {
        if (const void* ring = layer_norm_ring_kernel(cols, false, wide, &threads, &per_sm)) {
            size_t smem = 0;
            p.slots = layer_norm_slots((uint32_t)(cols * dtype_size(x_dtype)), threads, per_sm, &smem);
            return launch(ring, &p, dim3((unsigned)std::min<int64_t>(rows, (int64_t)n_sm * per_sm)), threads, 1, smem,
                          stream);
        }
    }
    const void* fn = layer_norm_kernel(cols, vectors, false, wide, &threads, &at_once, &per_sm);
    if (!fn)
        return launch(layer_norm_long_kernel(), &p, dim3((unsigned)std::min<int64_t>(rows, (int64_t)n_sm * 4)), 512, 1,
                      0, stream);
    return launch(fn, &p, dim3((unsigned)((rows + at_once - 1) / at_once)), threads, 1, 0, stream);
}

quasar_status quasar_layer_norm_backward_workspace(int64_t rows, int64_t cols, int64_t* bytes)
{
    if (!bytes || !valid_shape(rows, cols, cols)) return QUASAR_ERR_INVALID_ARG;
    int64_t parts = 0;
    const quasar_status st = norm_parts(rows, cols, &parts);
    if (st == QUASAR_OK) *bytes = norm_workspace(parts, cols);
    return st;
}

quasar_status quasar_layer_norm_backward(const void* dy, quasar_dtype dy_dtype, int64_t ld_dy, const void* x,
                                         quasar_dtype x_dtype, int64_t ld_x, const float* weight, const float* stats,
                                         int64_t rows, int64_t cols, int center, const void* residual,
                                         int64_t ld_residual, void* dx, quasar_dtype dx_dtype, int64_t ld_dx,
                                         float* dweight, float* dbias, void* workspace, int64_t workspace_bytes,
                                         quasar_stream_t stream)
{
    if (!valid_matrix(dy, rows, cols, ld_dy, dy_dtype) || !valid_matrix(x, rows, cols, ld_x, x_dtype))
        return QUASAR_ERR_INVALID_ARG;
    if (!valid_dtype(dx_dtype) || (center != 0 && center != 1)) return QUASAR_ERR_INVALID_ARG;
    if (dx && !valid_matrix(dx, rows, cols, ld_dx, dx_dtype)) return QUASAR_ERR_INVALID_ARG;
    if (residual && (!dx || !valid_matrix(residual, rows, cols, ld_residual, dx_dtype))) return QUASAR_ERR_INVALID_ARG;
    if (!aligned(weight, 4) || !aligned(stats, 4) || !aligned(dweight, 4) || !aligned(dbias, 4))
        return QUASAR_ERR_INVALID_ARG;
    if (cols == 0 && rows > 0) return QUASAR_ERR_INVALID_ARG;
    if (rows > 0 && !stats) return QUASAR_ERR_INVALID_ARG;
    if (cols == 0 || (!dx && !dweight && !dbias)) return QUASAR_OK;
    const Bytes ins[] = {Bytes(dy, rows, cols, ld_dy, dtype_size(dy_dtype)),
                         Bytes(x, rows, cols, ld_x, dtype_size(x_dtype)),
                         Bytes(residual, rows, cols, ld_residual, dtype_size(dx_dtype)), Bytes(weight, cols, 4),
                         Bytes(stats, 2 * rows, 4)};
    const Bytes outs[] = {Bytes(dx, rows, cols, ld_dx, dtype_size(dx_dtype)), Bytes(dweight, cols, 4),
                          Bytes(dbias, cols, 4)};
    for (int i = 0; i < 3; ++i) {
        // dx may take dy's, x's or the residual's place, in exactly its place
        for (int j = 0; j < 5; ++j)
            if (!(i == 0 && j < 3 && outs[0] == ins[j]) && overlaps(outs[i], ins[j]))
                return QUASAR_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (overlaps(outs[i], outs[j])) return QUASAR_ERR_INVALID_ARG;
    }
    int64_t parts = 0;
    quasar_status st = norm_parts(rows, cols, &parts);
    if (st != QUASAR_OK) return st;
    const int64_t need = dweight || dbias ? norm_workspace(parts, cols) : 0;
    if (workspace_bytes < need || (need > 0 && (!workspace || !aligned(workspace, 16)))) return QUASAR_ERR_INVALID_ARG;
    const Bytes b_ws(need > 0 ? workspace : nullptr, need, 1);
    for (const Bytes& b : ins)
        if (overlaps(b_ws, b)) return QUASAR_ERR_INVALID_ARG;
    for (const Bytes& b : outs)
        if (overlaps(b_ws, b)) return QUASAR_ERR_INVALID_ARG;
    NormGradParams p{dy,   ld_dy,  dy_dtype == QUASAR_F32, x,        ld_x,        x_dtype == QUASAR_F32,
                     weight, stats, rows, cols, center, residual, ld_residual, dx, ld_dx, dx_dtype == QUASAR_F32,
                     nullptr, nullptr, 0, host_timeout_ns(), host_forced_timeout_ns(), nullptr};
    int n_sm = 0;
    if ((st = host_device(&n_sm, &p.status)) != QUASAR_OK) return st;
    float* const partial = static_cast<float*>(workspace);
    if (dweight) p.part_w = parts <= 1 ? dweight : partial;
    if (dbias) p.part_b = parts <= 1 ? dbias : partial + parts * cols;
    PartSumParams sums{{p.part_w, p.part_b}, {dweight, dbias}, (int)parts, cols};
    if (rows > 0) {
        const bool vectors = vector_rows(dy, rows, ld_dy, dy_dtype) && vector_rows(x, rows, ld_x, x_dtype) &&
                             vector_rows(residual, rows, ld_residual, dx_dtype) && vector_rows(dx, rows, ld_dx, dx_dtype) &&
                             aligned(weight, 16);
        int threads = 0, at_once = 0, per_sm = 0;
        const bool wide = x_dtype == QUASAR_F32 || dy_dtype == QUASAR_F32 || (residual && dx_dtype == QUASAR_F32);
        const void* ring = vectors ? layer_norm_ring_kernel(cols, true, wide, &threads, &per_sm) : nullptr;
        const void* fn = ring ? nullptr : layer_norm_kernel(cols, vectors, true, wide, &threads, &at_once, &per_sm);
        if (ring) {
            size_t smem = 0;
            const int64_t bytes =
                cols * (dtype_size(x_dtype) + dtype_size(dy_dtype) + (residual ? dtype_size(dx_dtype) : 0));
            p.slots = layer_norm_slots((uint32_t)bytes, threads, per_sm, &smem);
            if ((st = launch(ring, &p, dim3((unsigned)parts), threads, 1, smem, stream)) != QUASAR_OK) return st;
        } else if (fn) {
            if ((st = launch(fn, &p, dim3((unsigned)parts), threads, 1, 0, stream)) != QUASAR_OK) return st;
        } else {
            // (the columns' sums first: dx may take dy's or x's place)
            if ((dweight || dbias) &&
                (st = launch(layer_norm_grad_columns_kernel(), &p, dim3((unsigned)((cols + 255) / 256), (unsigned)parts),
                             256, 1, 0, stream)) != QUASAR_OK)
                return st;
            if (dx && (st = launch(layer_norm_grad_long_kernel(), &p,
                                   dim3((unsigned)std::min<int64_t>(rows, (int64_t)1 << 16)), 512, 1, 0, stream)) !=
                          QUASAR_OK)
                return st;
        }
    }
    if (parts == 1 || (!dweight && !dbias)) return QUASAR_OK;
    if (!dweight) sums.part[0] = sums.part[1], sums.out[0] = sums.out[1];
    return launch(part_sum_kernel(), &sums, dim3((unsigned)((cols + 31) / 32), dweight && dbias ? 2 : 1), 1024, 1, 0,
                  stream);
}

quasar_status quasar_embedding(const void* ids, quasar_index_type ids_type, int64_t tokens, const void* table,
                               quasar_dtype table_dtype, int64_t ld_table, int64_t vocab, int64_t width, float scale,
                               const void* residual, int64_t ld_residual, void* y, quasar_dtype y_dtype, int64_t ld_y,
                               quasar_stream_t stream)
{
    if (!valid_ids(ids, ids_type, tokens) || !valid_matrix(table, vocab, width, ld_table, table_dtype) ||
        !valid_matrix(y, tokens, width, ld_y, y_dtype))
        return QUASAR_ERR_INVALID_ARG;
    if (residual && !valid_matrix(residual, tokens, width, ld_residual, y_dtype)) return QUASAR_ERR_INVALID_ARG;
    if (tokens == 0 || width == 0) return QUASAR_OK;
    const Bytes b_y(y, tokens, width, ld_y, dtype_size(y_dtype));
    const Bytes b_res(residual, tokens, width, ld_residual, dtype_size(y_dtype));
    // y may take the residual's place, in exactly its place
    if (overlaps(b_y, Bytes(table, vocab, width, ld_table, dtype_size(table_dtype))) ||
        overlaps(b_y, Bytes(ids, tokens, ids_type == QUASAR_I64 ? 8 : 4)) || (!(b_res == b_y) && overlaps(b_y, b_res)))
        return QUASAR_ERR_INVALID_ARG;
    const int64_t chunks = (width + kEmbedCols - 1) / kEmbedCols;
    if (chunks > 65535) return QUASAR_ERR_UNSUPPORTED;
    EmbedParams p{ids, ids_type == QUASAR_I64, tokens, table, ld_table, table_dtype == QUASAR_F32, vocab, width, scale,
                  residual, ld_residual, y, ld_y, y_dtype == QUASAR_F32};
    const bool vectors = vector_rows(table, vocab, ld_table, table_dtype) && vector_rows(y, tokens, ld_y, y_dtype) &&
                         vector_rows(residual, tokens, ld_residual, y_dtype);
    const bool wide = table_dtype == QUASAR_F32 || (residual && y_dtype == QUASAR_F32);
    return launch(embedding_kernel(vectors, wide), &p,
                  dim3((unsigned)((tokens + kEmbedTokens - 1) / kEmbedTokens), (unsigned)chunks), kEmbedThreads, 1, 0,
                  stream);
}

quasar_status quasar_embedding_backward_workspace(int64_t tokens, int64_t width, int64_t* bytes)
{
    if (!bytes || !valid_shape(tokens, width, width)) return QUASAR_ERR_INVALID_ARG;
    *bytes = embedding_workspace(tokens, width);
    return QUASAR_OK;
}

quasar_status quasar_embedding_backward(const void* dy, quasar_dtype dy_dtype, int64_t ld_dy, const void* ids,
                                        quasar_index_type ids_type, int64_t tokens, int64_t vocab, int64_t width,
                                        float scale, void* dtable, quasar_dtype dtable_dtype, int64_t ld_dtable,
                                        int accumulate, void* workspace, int64_t workspace_bytes,
                                        quasar_stream_t stream)
{
    if (!valid_ids(ids, ids_type, tokens) || !valid_matrix(dy, tokens, width, ld_dy, dy_dtype) ||
        !valid_matrix(dtable, vocab, width, ld_dtable, dtable_dtype) || (accumulate != 0 && accumulate != 1))
        return QUASAR_ERR_INVALID_ARG;
    if (vocab == 0 || width == 0 || (tokens == 0 && accumulate)) return QUASAR_OK;
    const int64_t need = embedding_workspace(tokens, width);
    if (workspace_bytes < need || (need > 0 && (!workspace || !aligned(workspace, 16)))) return QUASAR_ERR_INVALID_ARG;
    const Bytes b_out(dtable, vocab, width, ld_dtable, dtype_size(dtable_dtype)), b_ws(workspace, need, 1);
    const Bytes b_dy(dy, tokens, width, ld_dy, dtype_size(dy_dtype));
    const Bytes b_ids(ids, tokens, ids_type == QUASAR_I64 ? 8 : 4);
    if (overlaps(b_out, b_dy) || overlaps(b_out, b_ids) || overlaps(b_out, b_ws) || overlaps(b_ws, b_dy) ||
        overlaps(b_ws, b_ids))
        return QUASAR_ERR_INVALID_ARG;
    const int64_t chunks = (width + kEmbedCols - 1) / kEmbedCols;
    if (chunks > 65535) return QUASAR_ERR_UNSUPPORTED;
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    const int64_t list = up16(4 * tokens);
    SortParams s{};
    EmbedGradParams p{};
    s.ids = ids;
    s.ids_64 = ids_type == QUASAR_I64;
    s.n = (int)tokens;
    s.vocab = vocab;
    for (int i = 0; i < 2; ++i) {
        s.keys[i] = reinterpret_cast<uint32_t*>(ws + 2 * i * list);
        s.places[i] = reinterpret_cast<uint32_t*>(ws + (2 * i + 1) * list);
    }
    for (int64_t v = vocab; v > 0; v >>= kSortBits) ++s.passes;
    // a CTA of the sort keeps up with some 2,048 tokens in the time that a
    // cluster's exchange takes
    s.ctas = 1;
    while (s.ctas < kSortCtas && tokens > 2048 * (int64_t)s.ctas) s.ctas *= 2;
    quasar_status st;
    if (tokens > 0 && (st = launch(sort_ids_kernel(), &s, dim3((unsigned)s.ctas), kSortThreads, s.ctas, sort_ids_smem(),
                                   stream)) != QUASAR_OK)
        return st;
    p.dy = dy;
    p.ld_dy = ld_dy;
    p.dy_f32 = dy_dtype == QUASAR_F32;
    p.keys = s.keys[0];
    p.places = s.places[0];
    p.n = (int)tokens;
    p.sums = reinterpret_cast<float*>(ws + 4 * list);
    p.vocab = vocab;
    p.width = width;
    p.scale = scale;
    p.dtable = dtable;
    p.ld = ld_dtable;
    p.f32 = dtable_dtype == QUASAR_F32;
    p.add = accumulate;
    const bool vectors = vector_rows(dy, tokens, ld_dy, dy_dtype) && vector_rows(dtable, vocab, ld_dtable, dtable_dtype) &&
                         width % 4 == 0;  // (the chunks' sums)
    const bool wide = dy_dtype == QUASAR_F32 || (accumulate && dtable_dtype == QUASAR_F32);
    if (tokens >= kRunChunk && (st = launch(embedding_chunks_kernel(vectors, wide), &p,
                                            dim3((unsigned)(tokens / kRunChunk), (unsigned)chunks), kEmbedThreads, 1, 0,
                                            stream)) != QUASAR_OK)
        return st;
    return launch(embedding_grad_kernel(vectors, wide), &p,
                  dim3((unsigned)((vocab + kEmbedRows - 1) / kEmbedRows), (unsigned)chunks), kEmbedThreads, 1, 0, stream);
}

}  // extern "C"
