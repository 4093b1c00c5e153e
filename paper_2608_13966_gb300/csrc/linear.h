// Launch parameters of the matrix-product kernels (shared by host and device).
#pragma once

#include <cstdint>
#include <cuda.h>

namespace quasar {

// What follows the accumulators of a product D (rows x cols, D[i][j] kept at
// memory row j, column i: i is contiguous).
struct Epilogue {
    const float* bias;      // [i], added to the product, or NULL
    void* pre;              // bf16 copy of product + bias, or NULL
    int64_t ld_pre;
    const void* scale_pre;  // bf16 z: the product is multiplied by act'(z), or NULL
    int64_t ld_scale;
    const void* residual;   // added last, of the output's type, or NULL
    int64_t ld_res;
    void* out;
    int64_t ld_out;
    int act;                // quasar_activation: of the product, or of scale_pre's derivative
    int out_f32;
};

struct ProductParams {
    CUtensorMap a;  // operand of D's rows
    CUtensorMap b;  // operand of D's columns
    Epilogue e;
    int64_t rows;   // of D: contiguous in memory
    int64_t cols;
    int k_blocks;   // blocks of 64 along the reduction (0: the product is zero)
    int tiles_row;
    int tiles_col;
    int split;      // CTAs of a cluster that share a tile's reduction
    int stages;
    uint64_t timeout_ns;
    uint64_t force_timeout_ns;
    unsigned int* status;
};

struct OneParams {
    const void* x;
    const void* r;
    int64_t ld_r;
    int64_t features;
    int64_t inputs;
    Epilogue e;
};

struct OuterParams {
    const void* dz;  // bf16 [tokens, features]
    int64_t ld_dz;
    const void* x;   // bf16 [tokens, inputs]
    int64_t ld_x;
    int tokens;
    int64_t features;
    int64_t inputs;
    void* dr;
    int64_t ld_dr;
    float* dbias;    // or NULL
};

struct ColumnSumParams {
    const void* in;  // bf16 [rows, cols]
    int64_t ld;
    int64_t rows;
    int64_t cols;
    float* out;
};

struct ActGradParams {
    const void* dy;   // bf16
    int64_t ld_dy;
    const void* pre;  // bf16, or NULL (copy)
    int64_t ld_pre;
    void* dz;         // bf16
    int64_t ld_dz;
    int64_t rows;
    int64_t cols;
    int act;
};

}  // namespace quasar
