// Launch parameters of the kernels of the layers between the products (shared
// by host and device).
#pragma once

#include <cstdint>

namespace quasar {

// -- layer norm ----------------------------------------------------------------

constexpr int kNormMostCols = 16384;  // of a row kept in registers

struct NormParams {
    const void* x;
    int64_t ld_x;
    int x_f32;
    const float* weight;  // or NULL: 1
    const float* bias;    // or NULL
    int64_t rows;
    int64_t cols;
    int center;
    float eps;
    void* y;
    int64_t ld_y;
    int y_f32;
    float* stats;         // [rows, 2]: mean, 1 / deviation; or NULL
    int slots;            // of the ring, where rows come through shared memory
    uint64_t timeout_ns;
    uint64_t force_timeout_ns;
    unsigned int* status;
};

struct NormGradParams {
    const void* dy;
    int64_t ld_dy;
    int dy_f32;
    const void* x;
    int64_t ld_x;
    int x_f32;
    const float* weight;  // or NULL: 1
    const float* stats;
    int64_t rows;
    int64_t cols;
    int center;
    const void* residual;  // of dx's type, or NULL
    int64_t ld_res;
    void* dx;              // or NULL
    int64_t ld_dx;
    int dx_f32;
    float* part_w;         // [CTAs of rows, cols] partial sums, or NULL
    float* part_b;
    int slots;
    uint64_t timeout_ns;
    uint64_t force_timeout_ns;
    unsigned int* status;
};

struct PartSumParams {
    const float* part[2];  // [parts, cols], or NULL
    float* out[2];
    int parts;
    int64_t cols;
};

// -- embedding -----------------------------------------------------------------

constexpr int kSortBits = 9;        // of a pass
constexpr int kSortThreads = 1024;
constexpr int kSortCtas = 8;        // most of a cluster
constexpr int kRunChunk = 32;       // sorted tokens summed ahead where they share an id
constexpr int kEmbedThreads = 256;
constexpr int kEmbedCols = kEmbedThreads * 8;  // of a CTA
constexpr int kEmbedTokens = 4;     // of a CTA of the lookup
constexpr int kEmbedRows = 64;      // of the table, a CTA of the gradient

struct EmbedParams {
    const void* ids;
    int ids_64;
    int64_t tokens;
    const void* table;
    int64_t ld_table;
    int table_f32;
    int64_t vocab;
    int64_t width;
    float scale;
    const void* residual;  // of y's type, or NULL
    int64_t ld_res;
    void* y;
    int64_t ld_y;
    int y_f32;
};

struct SortParams {
    const void* ids;
    int ids_64;
    int n;
    int64_t vocab;      // an id outside [0, vocab) is sorted as vocab
    uint32_t* keys[2];  // the last pass writes keys[0] and places[0]
    uint32_t* places[2];
    int passes;
    int ctas;
};

struct EmbedGradParams {
    const void* dy;
    int64_t ld_dy;
    int dy_f32;
    const uint32_t* keys;    // sorted
    const uint32_t* places;
    int n;
    float* sums;             // [n / kRunChunk, width]
    int64_t vocab;
    int64_t width;
    float scale;
    void* dtable;
    int64_t ld;
    int f32;
    int add;                 // to what dtable holds
};

}  // namespace quasar
