// Arguments of the kernels of adamw_many.hip (internal header).
#pragma once

#include "adamw.h"

namespace pcm {

constexpr int kManyBlock = PCM_ADAMW_BLOCK;      // elements that share an exponent
constexpr int kManyChunk = 2048;                 // elements of a chunk: what a workgroup takes at a time, eight a lane

// A piece of one tensor: the plan is a list of these.
struct AdamwChunk {
    const void* grad;
    float* weight;
    uint16_t* lowp;          // bf16 copy, or null
    int64_t at;              // its first element among the states, a multiple of kManyChunk or the tensor's first
    int32_t count;
    int32_t grad_bf16;
};

struct ManyStep {
    const AdamwChunk* chunks;
    int64_t n;
    char* state;
    int64_t elements;
    const double* partial;   // of the sum of squares; parts = 0: gradients are taken as they are
    int parts;
    double max_norm;
    float* norm_out;         // or null
    AdamConst c;
    uint32_t step[2], seed[2];
};

}  // namespace pcm
