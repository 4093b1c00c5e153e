// Launch parameters of the kernels over rows of logits (shared by host and
// device).
#pragma once

#include <cstdint>

namespace quasar {

constexpr int kMaxTop = 256;          // most entries of a row's top list
constexpr int kRowCtas = 8;           // most CTAs (one cluster) a row is spread over
constexpr int kRowThreads = 512;      // of a CTA
constexpr int kBackThreads = 256;     // ... of a backward call, whose rows pass only once
constexpr int kFewThreads = 128;      // ... whose share is no more than kFewVectors (top lists: k no more than 128)
constexpr int kFewVectors = 1024;
constexpr int kMostVectors = 200000;  // of a share (a byte of shared memory each)

// A row is shared out to `ctas` CTAs, `vecs` 16-byte vectors each.
struct RowParams {
    const void* logits;
    int64_t ld;
    int64_t vocab;
    int ctas;       // of a cluster
    int vecs;       // of a CTA's share
    uint64_t force_timeout_ns;
    unsigned int* status;
};

struct TopParams {
    RowParams row;
    int k;
    float temperature;
    float* values;
    int32_t* indices;
    float* lse;     // or NULL
};

struct DistillParams {
    RowParams row;
    int k;
    const int32_t* indices;
    const float* values;
    const float* teacher_lse;  // or NULL: renormalise over the k
    const float* row_weight;   // or NULL: 1
    float temperature;
    float* loss;               // forward
    float* stats;              // forward: written if given; backward: read
    void* grad;                // or NULL
    int64_t ld_grad;
};

}  // namespace quasar
