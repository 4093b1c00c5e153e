// Launch parameters of the attention kernels (shared by host and device).
#pragma once

#include <cstdint>
#include <cuda.h>

namespace quasar {

constexpr int kAttnRows = 128;     // of a tile: (token, head) pairs, the lanes of tensor memory
constexpr int kAttnKeys = 128;     // of a key tile
constexpr int kAttnMostSplit = 8;  // CTAs of a cluster that share a row's keys
constexpr int kAttnFold = 1024;    // key tiles of one sum of a row

// Sequences packed along the rows of q, and of k and v: sequence i has the rows
// starts[i] .. starts[i + 1] (NULL: one sequence of all rows).
struct AttnSequences {
    const int* starts;
    const int* key_starts;
    int n;
    int tokens;  // rows of q
    int keys;    // rows of k, v
};

struct AttnParams {
    CUtensorMap q;  // [tokens, heads, d]: boxes of 64 x group x tile_tokens
    CUtensorMap k;  // [keys, kv_heads, d]: boxes of 64 x 1 x 128
    CUtensorMap v;
    AttnSequences s;
    int heads;
    int kv_heads;
    int group;        // heads that share keys
    int d;
    int tile_tokens;  // kAttnRows / group
    int causal;
    int items;        // pairs of tiles there may be, and one (per kv head)
    int split;
    int persistent;   // CTAs take items (and a row has one part)
    float scale_log2;
    void* y;
    int64_t ld_y;
    float* lse;       // [tokens, heads], or NULL
    uint64_t timeout_ns;
    uint64_t force_timeout_ns;
    unsigned int* status;
};

constexpr int kGradCols = 128;   // of a step of the backward kernels
constexpr int kGradFold = 1024;  // steps of one sum

// One of the two backward kernels: 128 rows stay, the other side streams past
// in steps of 128 columns.
struct AttnGradParams {
    CUtensorMap x1, x2;  // of the rows:  k, v (keys stay) or q, dy (queries stay)
    CUtensorMap z1, z2;  // of the steps: q, dy            or k, v
    AttnSequences s;
    int heads;
    int kv_heads;
    int group;
    int d;
    int tile_tokens;     // of 128 rows, or columns, of queries
    int causal;
    int items;
    float scale_log2;
    float scale;
    const float2* stats;  // [tokens, heads]: lse in bits, sum of dy y
    void* d1;             // dk or dq
    int64_t ld_d1;
    void* d2;             // dv
    int64_t ld_d2;
    uint64_t timeout_ns;
    uint64_t force_timeout_ns;
    unsigned int* status;
};

struct AttnStatsParams {
    const void* dy;
    int64_t ld_dy;
    const void* y;
    int64_t ld_y;
    const float* lse;
    int64_t tokens;
    int heads;
    int d;
    float2* stats;
};

}  // namespace quasar
