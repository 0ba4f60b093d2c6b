// Arguments of the kernels of token_logprobs.hip (internal header).
#pragma once

#include "common.h"

namespace pcm {

struct Logits {
    const void* z;
    int64_t ld;
    const uint8_t* allowed;      // or null
    int64_t allowed_ld;          // 0: the same tokens for every row
    const void* tokens;
    int token_type;
    int64_t rows;
    int V;
    float t, inv_t;              // the temperature
};

// What has been seen of a row: s = sum 2^a and t = sum 2^a a with a = (z - r) (log2 e) / temperature relative to a logit r (the lowest value: none yet).  The
// difference comes first: it is zero for z = r, where a difference of products would be off by the rounding of one of them, which has no bound.
struct RowSums {
    float r, s, t;
};
struct LogprobsOut {
    float *logp, *lse, *entropy;     // entropy: or null
    int top;
    int32_t* top_ids;
    float* top_logp;
};
// What a part of a row leaves for the launch that joins them.
struct RowParts {
    RowSums* sums;                      // [rows, parts]
    uint64_t* keys;                  // [rows, parts, top]
    int parts;
};

struct LogprobsGradient {
    const float *lse, *dlogp, *entropy, *dentropy;       // the last two: both or none
    void* dz;
    int64_t dz_ld;
};

}  // namespace pcm
