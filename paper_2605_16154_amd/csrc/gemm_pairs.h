// Products of matrices held as pairs (pairs.h), C[m, n] = sum_k A(m, k) B(n, k), for the orthogonalisation (internal header).
//
// Both operands are stored with the reduction index along their columns.  What the iteration multiplies is symmetric, or is
// kept in both orientations, so no other layout is needed: a product leaves its result as an operand, in one orientation or
// both.  Of a symmetric result only the tiles on and below the diagonal are computed.
#pragma once

#include "pairs.h"

namespace pcm {

// What becomes of a product: value = alpha * sum + beta * D + gamma * (m == n), then one of
enum PairResult : int {
    kPairs = 0,          // C and, if Ct is set, its transpose, as pairs
    kOutF32 = 1,         // out[m, n] = value
    kOutBf16 = 2,
    kOutWeights = 3      // out[m, n] (fp32) = decay * out - rate * value, and its bf16 copy to lowp if that is set
};

struct PairJob {
    const f16 *A, *B;
    int m_frags, n_frags;        // fragments of rows of the operands (even)
    int steps;                   // of 32 of k
    int symmetric;               // C = C^T: only tiles with n <= m, the others through Ct (= C)
    int result;
    f16 *C, *Ct;
    const f16* D;                // as C, or null
    float alpha, beta, gamma;
    void* out;
    uint16_t* lowp;
    int64_t ld;                  // of out (lowp: the same)
    int rows, cols;              // of out
    float decay, rate;
    int first_tile, tiles_n;     // filled in by the launch
};
constexpr int kMaxPairJobs = 16;
struct PairJobs {
    PairJob job[kMaxPairJobs];
    int n, tiles;
};

// Accumulators of a wavefront: tile (i, j), register t of a lane is row 16 i + (lane & 15), column 16 j + 4 (lane >> 4) + t.
template <int kW>
using PairAccumulators = f32x4[kW][kW];

__device__ inline f32x4 mfma_f16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// The wavefront's part of a tile: rows 16 (frag_m + i), columns 16 (frag_n + j).  off_diagonal: of a symmetric result, a tile whose
// transpose no other tile computes.
template <int kW>
__device__ __forceinline__ void pair_epilogue(const PairJob& p, const PairAccumulators<kW>& acc, int frag_m, int frag_n, bool off_diagonal) {
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    // Unit matrices that pick one half of a fragment's columns: a product with one is that half transposed, exactly.
    f16x8 unit[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        unit[0][e] = e < 4 && 4 * g + e == r ? (f16)1.f : (f16)0.f;
        unit[1][e] = e >= 4 && 4 * g + e - 4 == r ? (f16)1.f : (f16)0.f;
    }
    const bool transposed = p.Ct != nullptr && (!p.symmetric || off_diagonal);
#pragma unroll
    for (int i = 0; i < kW; i += 2)
#pragma unroll
        for (int j = 0; j < kW; j += 2) {
            const int fm = frag_m + i, fn = frag_n + j;
            if (fm >= p.m_frags || fn >= p.n_frags) continue;
            if (p.result == kPairs) {
                f16x8 hi[2], lo[2];
#pragma unroll
                for (int ii = 0; ii < 2; ++ii) {
                    const int64_t at = pair_fragment(fm + ii, fn / 2, p.m_frags) + lane * 8;
                    f16x8 dh = {0, 0, 0, 0, 0, 0, 0, 0}, dl = dh;
                    if (p.D != nullptr) {
                        dh = *reinterpret_cast<const f16x8*>(p.D + at);
                        dl = *reinterpret_cast<const f16x8*>(p.D + at + kPairPart);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float v = p.alpha * acc[i + ii][j + e / 4][e % 4];
                        if (p.D != nullptr) v += p.beta * ((float)dh[e] + (float)dl[e]);
                        if ((fm + ii) * 16 + r == fn * 16 + e / 4 * 16 + 4 * g + e % 4) v += p.gamma;
                        f16 h, l;
                        split_pair(v, h, l);
                        hi[ii][e] = h;
                        lo[ii][e] = l;
                    }
                    *reinterpret_cast<f16x8*>(p.C + at) = hi[ii];
                    *reinterpret_cast<f16x8*>(p.C + at + kPairPart) = lo[ii];
                }
                if (transposed) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int64_t at = pair_fragment(fn + h, fm / 2, p.n_frags) + lane * 8;
                        f16x8 th, tl;
#pragma unroll
                        for (int ii = 0; ii < 2; ++ii) {
                            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
                            const f32x4 a = mfma_f16(hi[ii], unit[h], zero), b = mfma_f16(lo[ii], unit[h], zero);
#pragma unroll
                            for (int t = 0; t < 4; ++t) {
                                th[4 * ii + t] = (f16)a[t];
                                tl[4 * ii + t] = (f16)b[t];
                            }
                        }
                        *reinterpret_cast<f16x8*>(p.Ct + at) = th;
                        *reinterpret_cast<f16x8*>(p.Ct + at + kPairPart) = tl;
                    }
                }
                continue;
            }
#pragma unroll
            for (int ii = 0; ii < 2; ++ii)
#pragma unroll
                for (int jj = 0; jj < 2; ++jj) {
                    const int m = (fm + ii) * 16 + r, n = (fn + jj) * 16 + 4 * g;
                    if (m >= p.rows) continue;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        if (n + t >= p.cols) continue;
                        const int64_t at = (int64_t)m * p.ld + n + t;
                        const float v = p.alpha * acc[i + ii][j + jj][t];
                        if (p.result == kOutF32) {
                            static_cast<float*>(p.out)[at] = v;
                        } else if (p.result == kOutBf16) {
                            static_cast<__bf16*>(p.out)[at] = (__bf16)v;
                        } else {
                            float* w = static_cast<float*>(p.out) + at;
                            const float now = p.decay * *w - p.rate * v;
                            *w = now;
                            if (p.lowp != nullptr) reinterpret_cast<__bf16*>(p.lowp)[at] = (__bf16)now;
                        }
                    }
                }
        }
}

// Tiles on and below the diagonal, row by row: the tile of row tm and column tn is number tm (tm + 1) / 2 + tn.
__device__ inline void triangle_tile(int number, int& tm, int& tn) {
    int row = (int)((sqrtf(8.f * (float)number + 1.f) - 1.f) * 0.5f);
    while ((row + 1) * (row + 2) / 2 <= number) ++row;
    while (row * (row + 1) / 2 > number) --row;
    tm = row;
    tn = number - row * (row + 1) / 2;
}

constexpr int kPairThreads = 256;

// Tiles of 32 kW x 32 kW by four wavefronts (2 x 2), operands from memory straight into registers.
template <int kW>
__global__ __launch_bounds__(kPairThreads) void pair_product(PairJobs jobs) {
    const int block = blockIdx.x;
    int q = 0;
    while (q + 1 < jobs.n && block >= jobs.job[q + 1].first_tile) ++q;
    const PairJob& p = jobs.job[q];
    const int number = block - p.first_tile;
    int tm, tn;
    if (p.symmetric) triangle_tile(number, tm, tn);
    else { tm = number / p.tiles_n; tn = number % p.tiles_n; }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int frag_m = (tm * 2 + (wave >> 1)) * kW, frag_n = (tn * 2 + (wave & 1)) * kW;

    // fragments beyond the last one are read from it: what they give is not stored
    const f16 *a[kW], *b[kW];
#pragma unroll
    for (int i = 0; i < kW; ++i) {
        a[i] = p.A + pair_fragment(min(frag_m + i, p.m_frags - 1), 0, p.m_frags) + lane * 8;
        b[i] = p.B + pair_fragment(min(frag_n + i, p.n_frags - 1), 0, p.n_frags) + lane * 8;
    }
    const int64_t a_step = pair_fragment(0, 1, p.m_frags), b_step = pair_fragment(0, 1, p.n_frags);
    PairAccumulators<kW> acc;
#pragma unroll
    for (int i = 0; i < kW; ++i)
#pragma unroll
        for (int j = 0; j < kW; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < p.steps; ++s) {
        f16x8 ah[kW], al[kW], bh[kW], bl[kW];
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            ah[i] = *reinterpret_cast<const f16x8*>(a[i]);
            al[i] = *reinterpret_cast<const f16x8*>(a[i] + kPairPart);
            bh[i] = *reinterpret_cast<const f16x8*>(b[i]);
            bl[i] = *reinterpret_cast<const f16x8*>(b[i] + kPairPart);
            a[i] += a_step;
            b[i] += b_step;
        }
#pragma unroll
        for (int i = 0; i < kW; ++i)
#pragma unroll
            for (int j = 0; j < kW; ++j) {
                acc[i][j] = mfma_f16(bl[j], ah[i], acc[i][j]);
                acc[i][j] = mfma_f16(bh[j], al[i], acc[i][j]);
                acc[i][j] = mfma_f16(bh[j], ah[i], acc[i][j]);
            }
    }
    pair_epilogue<kW>(p, acc, frag_m, frag_n, tm != tn);
}

template <int kW>
inline void launch_pair_tiles(PairJobs& jobs, hipStream_t s) {
    jobs.tiles = 0;
    for (int i = 0; i < jobs.n; ++i) {
        PairJob& p = jobs.job[i];
        const int tm = ceil_div(p.m_frags, 2 * kW), tn = ceil_div(p.n_frags, 2 * kW);
        p.first_tile = jobs.tiles;
        p.tiles_n = tn;
        jobs.tiles += p.symmetric ? tm * (tm + 1) / 2 : tm * tn;
    }
    pair_product<kW><<<(unsigned)jobs.tiles, kPairThreads, 0, s>>>(jobs);
}
inline void launch_pair_products(PairJobs& jobs, hipStream_t s) { launch_pair_tiles<2>(jobs, s); }

}  // namespace pcm
