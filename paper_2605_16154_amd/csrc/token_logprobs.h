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
    float inv_t;
};

// What has been seen of a row: s = sum 2^a and t = sum 2^a a with a = z c - R.  r is the logit that R = r c was made from (-inf:
// none yet); R is rounded, which takes nothing from the sums, as it is the same in all of them.  Logits beyond 1e38, where r c could
// overflow, have R = 0 and a = (z - r) c.
struct RowSums {
    float r, R, s, t;
    __device__ bool far() const { return fabsf(r) > 1e38f && r != -__builtin_huge_valf(); }
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
