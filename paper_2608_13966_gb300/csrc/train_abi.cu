// C ABI of the operators around the reconstruction: matrix products with the
// reconstructed weights, a teacher's top logits, and distillation from them.
// Argument validation, launch plans and launches; declarations and contracts
// are in include/quasar.h.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "host.h"
#include "linear.h"
#include "linear_plan.h"
#include "logits.h"
#include "quasar.h"

namespace quasar {
const void* product_tile_kernel(int bn, bool a_mn, bool b_mn, bool promote);
const void* product_pair_kernel(bool a_mn, bool b_mn, bool promote);
int product_pair_threads();
size_t product_pair_smem();
const void* linear_one_kernel();
const void* outer_kernel(int64_t tokens, bool f32, int* padded);
const void* column_sum_kernel();
const void* activation_grad_kernel();
const void* distill_kernel(bool f32, int threads, bool backward);
const void* top_logits_kernel(bool f32, int threads);
size_t distill_smem(int vecs, int threads);
size_t top_logits_smem(int threads, int ctas, int k);
}  // namespace quasar

namespace {

using namespace quasar;

bool valid_dtype(quasar_dtype d) { return d == QUASAR_F32 || d == QUASAR_BF16; }
int64_t dtype_size(quasar_dtype d) { return d == QUASAR_BF16 ? 2 : 4; }
bool valid_act(quasar_activation a) { return a >= QUASAR_ACT_NONE && a <= QUASAR_ACT_GELU; }
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// The bytes of a strided matrix: `width` of them in each of `rows` rows that
// are `pitch` apart.
struct Bytes {
    uintptr_t at;
    size_t rows, width, pitch;

    Bytes(const void* p, int64_t rows_, int64_t cols, int64_t ld, int64_t size)
        : at(reinterpret_cast<uintptr_t>(p)), rows(p ? (size_t)rows_ : 0), width((size_t)(cols * size)),
          pitch((size_t)(ld * size))
    {
    }
    Bytes(const void* p, int64_t n, int64_t size) : Bytes(p, 1, n, n, size) {}
    size_t span() const { return rows == 0 || width == 0 ? 0 : (rows - 1) * pitch + width; }
    bool operator==(const Bytes& o) const
    {
        return at == o.at && rows == o.rows && width == o.width && (rows <= 1 || pitch == o.pitch);
    }
};

// Whether two matrices share a byte.  Columns of one buffer (the same pitch)
// lie between each other's without: decided by where they lie in its rows.
bool overlaps(const Bytes& a, const Bytes& b)
{
    const size_t na = a.span(), nb = b.span();
    if (na == 0 || nb == 0 || a.at >= b.at + nb || b.at >= a.at + na) return false;
    const size_t pitch = a.rows > 1 ? a.pitch : b.pitch;
    if ((b.rows > 1 && b.pitch != pitch) || a.width > pitch || b.width > pitch) return true;
    const size_t from = b.at >= a.at ? (b.at - a.at) % pitch : (pitch - (a.at - b.at) % pitch) % pitch;
    return from < a.width || from + b.width > pitch;
}

// Sizes a 2-D view may have: coordinates are 32-bit on the device, offsets 64.
bool valid_shape(int64_t rows, int64_t cols, int64_t ld)
{
    constexpr int64_t kMax = (int64_t(1) << 31) - 256;
    return rows >= 0 && cols >= 0 && rows <= kMax && cols <= kMax && ld >= cols &&
           ld <= (int64_t(1) << 36) && (rows == 0 || ld <= (int64_t(1) << 58) / rows);
}

// -- launches ------------------------------------------------------------------

// A programmatic dependent launch: every kernel of this file waits for the
// grid before it in the stream before it touches global memory, and only its
// prologue (barriers, tensor memory, tensor maps) runs earlier.
quasar_status launch(const void* fn, void* params, dim3 grid, int threads, int cluster, size_t smem,
                     quasar_stream_t stream)
{
    const quasar_status st = host_allow_smem(fn, smem);
    if (st != QUASAR_OK) return st;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = reinterpret_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    void* args[] = {params};
    return cudaLaunchKernelExC(&cfg, fn, args) == cudaSuccess ? QUASAR_OK : QUASAR_ERR_CUDA;
}

// -- matrix products -------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                 CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) !=
                cudaSuccess ||
            q != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

// An operand as it lies in memory: bf16 [outer, inner], 64 x box_outer tiles.
struct Operand {
    const void* p;
    int64_t ld;
    int64_t outer, inner;
    bool mn_major;  // inner is the coordinate of D's rows (or columns), not the reduction
};

quasar_status tile_map(const Operand& o, int box_outer, CUtensorMap* map)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return QUASAR_ERR_UNSUPPORTED;
    const cuuint64_t dims[2] = {(cuuint64_t)o.inner, (cuuint64_t)o.outer};
    const cuuint64_t strides[1] = {(cuuint64_t)o.ld * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_outer};
    const cuuint32_t step[2] = {1, 1};
    const CUresult r =
        encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(o.p), dims, strides, box, step,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? QUASAR_OK : QUASAR_ERR_INVALID_ARG;
}

// An operand's rows start at 16-byte boundaries (the rule of tiled copies).
bool valid_operand(const void* p, int64_t rows, int64_t cols, int64_t ld)
{
    return valid_shape(rows, cols, ld) && (rows == 0 || cols == 0 || (p && aligned(p, 16) && ld % 8 == 0));
}

// Stages of k_product_tile for bn columns: what two CTAs an SM leave each.
int tile_stages(int bn, size_t* smem)
{
    const size_t stage = 128 * 128 + (size_t)bn * 128;
    const int stages = (int)std::min<size_t>(8, (size_t)100 * 1024 / stage);
    // exchange of partial tiles through the stages' memory
    *smem = 1024 + stages * stage + (2 * stages + 6) * 8 + 16;
    return stages;
}

// D (rows x cols, rows contiguous) = A B^T over `depth`, then the epilogue.
quasar_status product(const Operand& a, const Operand& b, int64_t rows, int64_t cols, int64_t depth,
                      const Epilogue& e, quasar_stream_t stream)
{
    if (rows == 0 || cols == 0) return QUASAR_OK;
    ProductParams p{};
    int n_sm = 0;
    quasar_status st = host_device(&n_sm, &p.status);
    if (st != QUASAR_OK) return st;
    p.e = e;
    p.rows = rows;
    p.cols = cols;
    p.k_blocks = (int)((depth + 63) / 64);
    p.timeout_ns = host_timeout_ns();
    p.force_timeout_ns = host_forced_timeout_ns();

    // Paired 256 x 256 tiles or one 128-row tile a cluster, by what they take
    // (measured, 512 to 14336 a side): a pair works through a block of 64 of
    // the reduction in 315 ns, 76 pairs side by side; the smaller tiles are
    // bound by L2, 2.1 ns a tile and block in all, and start 3 us dearer.
    const int64_t pair_tiles = ((rows + 255) / 256) * ((cols + 255) / 256);
    const int64_t small_tiles = ((rows + 127) / 128) * ((cols + 127) / 128);
    const double pair_ns = (double)((pair_tiles + n_sm / 2 - 1) / (n_sm / 2)) * p.k_blocks * 315.0;
    if (depth > 0 && cols > 64 && rows > 128 && pair_ns < 3000.0 + 2.1 * (double)small_tiles * p.k_blocks) {
        p.tiles_row = (int)((rows + 255) / 256);
        p.tiles_col = (int)((cols + 255) / 256);
        if ((st = tile_map(a, a.mn_major ? 64 : 128, &p.a)) != QUASAR_OK) return st;
        if ((st = tile_map(b, b.mn_major ? 64 : 128, &p.b)) != QUASAR_OK) return st;
        const void* fn = product_pair_kernel(a.mn_major, b.mn_major, e.out_f32 && p.k_blocks > 8);
        if (!fn) return QUASAR_ERR_UNSUPPORTED;
        int pairs = 0;
        if ((st = host_max_clusters(fn, 2, product_pair_threads(), product_pair_smem(), &pairs)) != QUASAR_OK) return st;
        pairs = (int)std::min<int64_t>(pair_tiles, pairs);
        return launch(fn, &p, dim3((unsigned)pairs * 2), product_pair_threads(), 2, product_pair_smem(),
                      stream);
    }
    int bn = cols <= 16 ? 16 : (cols <= 32 ? 32 : (cols <= 64 ? 64 : 128));
    if (b.mn_major) bn = std::max(bn, 64);
    p.tiles_row = (int)((rows + 127) / 128);
    p.tiles_col = (int)((cols + bn - 1) / bn);
    const int64_t tiles = (int64_t)p.tiles_row * p.tiles_col;
    size_t smem = 0;
    // (the answer holds for every variant: one kernel is asked for all)
    tile_stages(128, &smem);
    const void* asked = product_tile_kernel(128, false, false, false);
    auto max_clusters = [&](int size, int* n) { return host_max_clusters(asked, size, 192, smem, n); };
    if ((st = tile_split(tiles, p.k_blocks, n_sm, max_clusters, &p.split)) != QUASAR_OK) return st;
    p.stages = tile_stages(bn, &smem);
    if (tiles * p.split > (int64_t(1) << 31) - 1) return QUASAR_ERR_UNSUPPORTED;
    // parts are only worth promoting where there are several
    const bool promote = e.out_f32 && (p.k_blocks + p.split - 1) / p.split > 8;
    if (depth > 0) {
        if ((st = tile_map(a, a.mn_major ? 64 : 128, &p.a)) != QUASAR_OK) return st;
        if ((st = tile_map(b, b.mn_major ? 64 : bn, &p.b)) != QUASAR_OK) return st;
    }
    const void* fn = product_tile_kernel(bn, a.mn_major, b.mn_major, promote);
    if (!fn) return QUASAR_ERR_UNSUPPORTED;
    return launch(fn, &p, dim3((unsigned)(tiles * p.split)), 192, p.split, smem, stream);
}

// -- rows of logits ----------------------------------------------------------------

// How a row is spread: one CTA, or more (a power of two, one cluster) while
// the rows alone leave SMs idle and a share keeps at least 1,024 vectors (16
// KB: below that the exchange costs more than the reading), or while a share
// is longer than the distillation's shared memory can describe.
quasar_status plan_rows(const void* logits, quasar_dtype dtype, int64_t ld, int64_t rows, int64_t vocab,
                        RowParams* row, int* threads)
{
    int n_sm = 0;
    quasar_status st = host_device(&n_sm, &row->status);
    if (st != QUASAR_OK) return st;
    row->logits = logits;
    row->ld = ld;
    row->vocab = vocab;
    row->force_timeout_ns = host_forced_timeout_ns();
    const int64_t per = 16 / dtype_size(dtype);
    const int64_t vecs = (vocab + per - 1 + per - 1) / per;  // for any start within 16 bytes
    int c = 1;
    while (c < kRowCtas && ((rows * c < n_sm && vecs / (2 * c) >= 1024) || vecs / c > kMostVectors)) c *= 2;
    if (vecs / c > kMostVectors) return QUASAR_ERR_UNSUPPORTED;
    row->ctas = c;
    row->vecs = (int)((vecs + c - 1) / c);
    *threads = row->vecs <= kFewVectors ? kFewThreads : kRowThreads;
    if (rows * c > (int64_t(1) << 31) - 1) return QUASAR_ERR_UNSUPPORTED;
    return QUASAR_OK;
}

quasar_status check_rows(const void* logits, quasar_dtype dtype, int64_t ld, int64_t rows, int64_t vocab,
                         int k, float temperature)
{
    if (!valid_dtype(dtype) || !valid_shape(rows, vocab, ld)) return QUASAR_ERR_INVALID_ARG;
    if (!(temperature >= 1e-6f && temperature <= 1e6f)) return QUASAR_ERR_INVALID_ARG;
    if (vocab < 1 || k < 1 || k > vocab) return QUASAR_ERR_INVALID_ARG;
    if (k > kMaxTop) return QUASAR_ERR_UNSUPPORTED;
    if (rows > 0 && (!logits || !aligned(logits, (uintptr_t)dtype_size(dtype)))) return QUASAR_ERR_INVALID_ARG;
    return QUASAR_OK;
}

quasar_status run_distill(const void* logits, quasar_dtype dtype, int64_t ld, int64_t rows, int64_t vocab,
                          const int32_t* indices, const float* values, int k, const float* teacher_lse,
                          const float* row_weight, float temperature, float* loss, float* stats, void* grad,
                          int64_t ld_grad, bool backward, quasar_stream_t stream)
{
    quasar_status st = check_rows(logits, dtype, ld, rows, vocab, k, temperature);
    if (st != QUASAR_OK) return st;
    if (grad && !valid_shape(rows, vocab, ld_grad)) return QUASAR_ERR_INVALID_ARG;
    if (rows == 0) return QUASAR_OK;
    if (!indices || !values || !aligned(indices, 4) || !aligned(values, 4)) return QUASAR_ERR_INVALID_ARG;
    if (!aligned(teacher_lse, 4) || !aligned(row_weight, 4) || !aligned(loss, 4) || !aligned(stats, 4))
        return QUASAR_ERR_INVALID_ARG;
    if (backward ? (!stats || !grad) : !loss) return QUASAR_ERR_INVALID_ARG;
    if (!aligned(grad, (uintptr_t)dtype_size(dtype))) return QUASAR_ERR_INVALID_ARG;
    const Bytes b_logits(logits, rows, vocab, ld, dtype_size(dtype));
    const Bytes b_grad(grad, rows, vocab, ld_grad, dtype_size(dtype));
    // the gradient may replace the logits, in exactly their place
    if (!(b_grad == b_logits) && overlaps(b_grad, b_logits)) return QUASAR_ERR_INVALID_ARG;
    const Bytes outs[] = {b_grad, Bytes(backward ? nullptr : loss, rows, 4),
                          Bytes(backward ? nullptr : stats, 2 * rows, 4)};
    const Bytes ins[] = {Bytes(indices, rows * k, 4), Bytes(values, rows * k, 4), Bytes(teacher_lse, rows, 4),
                         Bytes(row_weight, rows, 4), Bytes(backward ? stats : nullptr, 2 * rows, 4)};
    for (int i = 0; i < 3; ++i) {
        for (const Bytes& in : ins)
            if (overlaps(outs[i], in)) return QUASAR_ERR_INVALID_ARG;
        if (i > 0 && overlaps(outs[i], b_logits)) return QUASAR_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (overlaps(outs[i], outs[j])) return QUASAR_ERR_INVALID_ARG;
    }
    DistillParams p{};
    int threads = 0;
    if ((st = plan_rows(logits, dtype, ld, rows, vocab, &p.row, &threads)) != QUASAR_OK) return st;
    if (backward && threads == kRowThreads) threads = kBackThreads;
    p.k = k;
    p.indices = indices;
    p.values = values;
    p.teacher_lse = teacher_lse;
    p.row_weight = row_weight;
    p.temperature = temperature;
    p.loss = loss;
    p.stats = stats;
    p.grad = grad;
    p.ld_grad = ld_grad;
    return launch(distill_kernel(dtype == QUASAR_F32, threads, backward), &p, dim3((unsigned)(rows * p.row.ctas)),
                  threads, backward ? 1 : p.row.ctas, distill_smem(p.row.vecs, threads), stream);
}

}  // namespace

extern "C" {

quasar_status quasar_linear(const void* x, int64_t ld_x, const void* r, int64_t ld_r, const float* bias,
                            quasar_activation activation, const void* residual, int64_t ld_residual,
                            int64_t tokens, int64_t features, int64_t inputs, void* y, quasar_dtype y_dtype,
                            int64_t ld_y, void* pre, int64_t ld_pre, quasar_stream_t stream)
{
    if (!valid_act(activation) || !valid_dtype(y_dtype)) return QUASAR_ERR_INVALID_ARG;
    if (!valid_operand(x, tokens, inputs, ld_x) || !valid_operand(r, features, inputs, ld_r))
        return QUASAR_ERR_INVALID_ARG;
    if (!valid_shape(tokens, features, ld_y)) return QUASAR_ERR_INVALID_ARG;
    if (residual && !valid_shape(tokens, features, ld_residual)) return QUASAR_ERR_INVALID_ARG;
    if (pre && !valid_shape(tokens, features, ld_pre)) return QUASAR_ERR_INVALID_ARG;
    if (tokens == 0 || features == 0) return QUASAR_OK;
    const int64_t size = dtype_size(y_dtype);
    if (!y || !aligned(y, size) || !aligned(residual, size) || !aligned(bias, 4) || !aligned(pre, 2))
        return QUASAR_ERR_INVALID_ARG;
    const Bytes b_y(y, tokens, features, ld_y, size), b_pre(pre, tokens, features, ld_pre, 2);
    const Bytes b_res(residual, tokens, features, ld_residual, size), b_bias(bias, features, 4);
    const Bytes b_x(x, tokens, inputs, ld_x, 2), b_r(r, features, inputs, ld_r, 2);
    // y may replace the residual, in exactly its place
    if (overlaps(b_y, b_x) || overlaps(b_y, b_r) || overlaps(b_y, b_bias) ||
        (!(b_res == b_y) && overlaps(b_y, b_res)) || overlaps(b_pre, b_x) || overlaps(b_pre, b_r) ||
        overlaps(b_pre, b_bias) || overlaps(b_pre, b_res) || overlaps(b_pre, b_y))
        return QUASAR_ERR_INVALID_ARG;
    const Epilogue e{bias, pre, ld_pre, nullptr, 0, residual, ld_residual, y, ld_y, activation,
                     y_dtype == QUASAR_F32};
    // one token: 2.7 us through 1024 x 4096, 5.8 through 4096 x 4096 and 20.4
    // through 4096 x 14336, by the tensor cores' kernel 7.2, 8.2 and 22.0 (22.6 by
    // both through 14336 x 4096); two tokens already take 29 there against 22
    if (tokens == 1 && inputs > 0) {
        OneParams f{x, r, ld_r, features, inputs, e};
        return launch(linear_one_kernel(), &f, dim3((unsigned)((features + 3) / 4)), 256, 1,
                      8 * 4 * 4, stream);
    }
    return product(Operand{r, ld_r, features, inputs, false}, Operand{x, ld_x, tokens, inputs, false}, features,
                   tokens, inputs, e, stream);
}

quasar_status quasar_linear_grad_input(const void* dz, int64_t ld_dz, const void* r, int64_t ld_r,
                                       const void* pre_in, int64_t ld_pre_in, quasar_activation activation_in,
                                       const void* residual, int64_t ld_residual, int64_t tokens,
                                       int64_t features, int64_t inputs, void* dx, quasar_dtype dx_dtype,
                                       int64_t ld_dx, quasar_stream_t stream)
{
    if (!valid_act(activation_in) || !valid_dtype(dx_dtype)) return QUASAR_ERR_INVALID_ARG;
    if (!valid_operand(dz, tokens, features, ld_dz) || !valid_operand(r, features, inputs, ld_r))
        return QUASAR_ERR_INVALID_ARG;
    if (!valid_shape(tokens, inputs, ld_dx)) return QUASAR_ERR_INVALID_ARG;
    if (residual && !valid_shape(tokens, inputs, ld_residual)) return QUASAR_ERR_INVALID_ARG;
    const bool slope = activation_in != QUASAR_ACT_NONE;
    if (pre_in && !valid_shape(tokens, inputs, ld_pre_in)) return QUASAR_ERR_INVALID_ARG;
    if (tokens == 0 || inputs == 0) return QUASAR_OK;
    const int64_t size = dtype_size(dx_dtype);
    if (!dx || !aligned(dx, size) || !aligned(residual, size) || !aligned(pre_in, 2)) return QUASAR_ERR_INVALID_ARG;
    if (slope && !pre_in) return QUASAR_ERR_INVALID_ARG;
    const Bytes b_dx(dx, tokens, inputs, ld_dx, size), b_pre(pre_in, tokens, inputs, ld_pre_in, 2);
    const Bytes b_res(residual, tokens, inputs, ld_residual, size);
    // dx may replace the residual or a bf16 pre_in, in exactly their place
    if (overlaps(b_dx, Bytes(dz, tokens, features, ld_dz, 2)) ||
        overlaps(b_dx, Bytes(r, features, inputs, ld_r, 2)) || (!(b_pre == b_dx) && overlaps(b_dx, b_pre)) ||
        (!(b_res == b_dx) && overlaps(b_dx, b_res)))
        return QUASAR_ERR_INVALID_ARG;
    const Epilogue e{nullptr, nullptr, 0, slope ? pre_in : nullptr, ld_pre_in, residual, ld_residual, dx, ld_dx,
                     activation_in, dx_dtype == QUASAR_F32};
    return product(Operand{r, ld_r, features, inputs, true}, Operand{dz, ld_dz, tokens, features, false}, inputs,
                   tokens, features, e, stream);
}

quasar_status quasar_linear_grad_weight(const void* dz, int64_t ld_dz, const void* x, int64_t ld_x,
                                        int64_t tokens, int64_t features, int64_t inputs, void* dr,
                                        quasar_dtype dr_dtype, int64_t ld_dr, float* dbias,
                                        quasar_stream_t stream)
{
    if (!valid_dtype(dr_dtype) || !valid_operand(dz, tokens, features, ld_dz)) return QUASAR_ERR_INVALID_ARG;
    if (dr && (!valid_operand(x, tokens, inputs, ld_x) || !valid_shape(features, inputs, ld_dr)))
        return QUASAR_ERR_INVALID_ARG;
    if (features == 0) return QUASAR_OK;
    if ((dr && !aligned(dr, dtype_size(dr_dtype))) || !aligned(dbias, 4)) return QUASAR_ERR_INVALID_ARG;
    const Bytes b_dz(dz, tokens, features, ld_dz, 2), b_x(dr ? x : nullptr, tokens, inputs, ld_x, 2);
    const Bytes b_dr(dr, features, inputs, ld_dr, dtype_size(dr_dtype)), b_dbias(dbias, features, 4);
    if (overlaps(b_dr, b_dz) || overlaps(b_dr, b_x) || overlaps(b_dbias, b_dz) || overlaps(b_dbias, b_x) ||
        overlaps(b_dbias, b_dr))
        return QUASAR_ERR_INVALID_ARG;
    if ((!dr || inputs == 0) && !dbias) return QUASAR_OK;
    // a few tokens: writing dr is what it takes, 20 us against the tensor cores'
    // 36 for 4 tokens and 14336 x 4096, 24 for 8 (12 would take 43)
    const int64_t outer_blocks = (features + 31) / 32;
    if (tokens <= 8 && outer_blocks <= 65535) {
        OuterParams o{dz, ld_dz, x, ld_x, (int)tokens, features, dr ? inputs : 0, dr, ld_dr, dbias};
        int padded = 0;
        const void* fn = outer_kernel(tokens, dr_dtype == QUASAR_F32, &padded);
        return launch(fn, &o, dim3((unsigned)std::max<int64_t>(1, (o.inputs + 2047) / 2048), (unsigned)outer_blocks),
                      256, 1, (size_t)32 * padded * 4, stream);
    }
    if (dbias) {
        ColumnSumParams c{dz, ld_dz, tokens, features, dbias};
        const int64_t blocks = (features + 63) / 64;
        const quasar_status st =
            launch(column_sum_kernel(), &c, dim3((unsigned)(blocks * 8)), 256, 8, (256 + 256) * 8, stream);
        if (st != QUASAR_OK) return st;
    }
    if (!dr) return QUASAR_OK;
    const Epilogue e{nullptr, nullptr, 0, nullptr, 0, nullptr, 0, dr, ld_dr, QUASAR_ACT_NONE,
                     dr_dtype == QUASAR_F32};
    return product(Operand{x, ld_x, tokens, inputs, true}, Operand{dz, ld_dz, tokens, features, true}, inputs,
                   features, tokens, e, stream);
}

quasar_status quasar_activation_grad(const void* dy, int64_t ld_dy, const void* pre, int64_t ld_pre,
                                     quasar_activation activation, int64_t rows, int64_t cols, void* dz,
                                     int64_t ld_dz, quasar_stream_t stream)
{
    const bool slope = activation != QUASAR_ACT_NONE;
    if (!valid_act(activation) || !valid_shape(rows, cols, ld_dy) || !valid_shape(rows, cols, ld_dz))
        return QUASAR_ERR_INVALID_ARG;
    if (slope && !valid_shape(rows, cols, ld_pre)) return QUASAR_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return QUASAR_OK;
    if (!dy || !dz || (slope && !pre) || !aligned(dy, 2) || !aligned(dz, 2) || !aligned(pre, 2))
        return QUASAR_ERR_INVALID_ARG;
    const Bytes b_dz(dz, rows, cols, ld_dz, 2), b_dy(dy, rows, cols, ld_dy, 2);
    const Bytes b_pre(slope ? pre : nullptr, rows, cols, ld_pre, 2);
    if ((!(b_dz == b_dy) && overlaps(b_dz, b_dy)) || (!(b_dz == b_pre) && overlaps(b_dz, b_pre)))
        return QUASAR_ERR_INVALID_ARG;
    ActGradParams p{dy, ld_dy, slope ? pre : nullptr, ld_pre, dz, ld_dz, rows, cols, activation};
    return launch(activation_grad_kernel(), &p,
                  dim3((unsigned)((cols + 255) / 256), (unsigned)std::min<int64_t>(rows, 65535)), 256, 1, 0, stream);
}

quasar_status quasar_top_logits(const void* logits, quasar_dtype dtype, int64_t ld, int64_t rows, int64_t vocab,
                                int k, float temperature, float* values, int32_t* indices, float* lse,
                                quasar_stream_t stream)
{
    quasar_status st = check_rows(logits, dtype, ld, rows, vocab, k, temperature);
    if (st != QUASAR_OK) return st;
    if (rows == 0) return QUASAR_OK;
    if (!values || !indices || !aligned(values, 4) || !aligned(indices, 4) || !aligned(lse, 4))
        return QUASAR_ERR_INVALID_ARG;
    const Bytes b_logits(logits, rows, vocab, ld, dtype_size(dtype)), b_lse(lse, rows, 4);
    const Bytes b_values(values, rows * k, 4), b_indices(indices, rows * k, 4);
    if (overlaps(b_values, b_logits) || overlaps(b_indices, b_logits) || overlaps(b_lse, b_logits) ||
        overlaps(b_values, b_indices) || overlaps(b_lse, b_values) || overlaps(b_lse, b_indices))
        return QUASAR_ERR_INVALID_ARG;
    TopParams p{};
    int threads = 0;
    if ((st = plan_rows(logits, dtype, ld, rows, vocab, &p.row, &threads)) != QUASAR_OK) return st;
    // the bound is the k-th largest of the threads' maxima: it takes k of them
    if (k > kFewThreads) threads = kRowThreads;
    p.k = k;
    p.temperature = temperature;
    p.values = values;
    p.indices = indices;
    p.lse = lse;
    return launch(top_logits_kernel(dtype == QUASAR_F32, threads), &p, dim3((unsigned)(rows * p.row.ctas)), threads,
                  p.row.ctas, top_logits_smem(threads, p.row.ctas, k), stream);
}

quasar_status quasar_distill_top(const void* logits, quasar_dtype dtype, int64_t ld, int64_t rows, int64_t vocab,
                                 const int32_t* indices, const float* values, int k, const float* teacher_lse,
                                 const float* row_weight, float temperature, float* loss, float* stats,
                                 void* grad, int64_t ld_grad, quasar_stream_t stream)
{
    return run_distill(logits, dtype, ld, rows, vocab, indices, values, k, teacher_lse, row_weight, temperature,
                       loss, stats, grad, ld_grad, false, stream);
}

quasar_status quasar_distill_top_backward(const void* logits, quasar_dtype dtype, int64_t ld, int64_t rows,
                                          int64_t vocab, const int32_t* indices, const float* values, int k,
                                          const float* teacher_lse, const float* stats, const float* row_weight,
                                          float temperature, void* grad, int64_t ld_grad,
                                          quasar_stream_t stream)
{
    return run_distill(logits, dtype, ld, rows, vocab, indices, values, k, teacher_lse, row_weight, temperature,
                       nullptr, const_cast<float*>(stats), grad, ld_grad, true, stream);
}

}  // extern "C"
