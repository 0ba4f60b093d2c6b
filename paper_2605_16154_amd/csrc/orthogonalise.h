// Arguments of the kernels of orthogonalise.hip that are not products (internal header).
#pragma once

#include "pairs.h"

namespace pcm {

constexpr int kOrthGroup = 8;        // matrices of a launch

struct UpdateMatrix {
    const void* in;              // [rows, cols] of `bf16` or fp32
    float* momentum;             // or null: the iteration is on `in`
    int64_t ld;
    int rows, cols, bf16, tall;  // tall: more rows than columns, X is the transpose
    float mu;
    int nesterov;
    double* partial;
    int parts, first_part;       // of the launch of the squares
    int tiles_c, tiles, first_tile;
    f16 *X, *Xt;                 // [m, n] and [n, m] with m <= n
};
struct UpdateMatrices {
    UpdateMatrix m[kOrthGroup];
    int n;
};

}  // namespace pcm
