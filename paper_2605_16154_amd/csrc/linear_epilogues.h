// Epilogues of the products around a vocabulary projection, and the arguments of what works on their results (internal header).
#pragma once

#include "linear_logprobs.h"

namespace pcm {

typedef _Float16 f16;
typedef __attribute__((ext_vector_type(4))) f16 f16x4;

// ---- statistics of blocks of logits ------------------------------------------------------------------

// What a part of a row's logits comes to: the largest z; sum 2^a; sum 2^a a, a = (z - largest) c.  A part that saw nothing has the sum 0.
struct RowSums {
    float m, s, t;
};
struct PartSums {
    f32x4* of;                           // [parts][ld], the fourth value unused
    int64_t ld;
    int parts;
};
__device__ __forceinline__ void merge(RowSums& a, const RowSums& b, float c) {
    const float m = fmaxf(a.s == 0.f ? b.m : a.m, b.s == 0.f ? a.m : b.m);
    const float da = fmaxf((a.m - m) * c, -1e30f), db = fmaxf((b.m - m) * c, -1e30f);
    const float ea = a.s == 0.f ? 0.f : __builtin_amdgcn_exp2f(da), eb = b.s == 0.f ? 0.f : __builtin_amdgcn_exp2f(db);
    a.t = ea * __builtin_fmaf(a.s, da, a.t) + eb * __builtin_fmaf(b.s, db, b.t);
    a.s = a.s * ea + b.s * eb;
    a.m = m;
}
// The sums of kN x 4 logits relative to m; -150 stands for what is as good as nothing (a is -inf where z is, or is that far below m).
template <int kN, class F>
__device__ __forceinline__ RowSums sums_of(float m, float c, F z) {
    RowSums r{m, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kN; ++j) {
        float s = 0.f, t = 0.f;                            // four terms before they are added to the others
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float a = (z(j, e) - m) * c, x = __builtin_amdgcn_exp2f(a);
            s += x;
            t = __builtin_fmaf(x, fmaxf(a, -150.f), t);
        }
        r.s += s;
        r.t += t;
    }
    return r;
}

// The largest of three, NaN if one of them is (fmaxf would let a NaN go, and first quieten each operand, an instruction more).
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_maximum3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

__device__ __forceinline__ float at_most(float x, float most) {    // (NaN stays)
    float r;
    asm("v_minimum3_f32 %0, %1, %2, %2" : "=v"(r) : "v"(x), "v"(most));
    return r;
}

// The logits of a tile, a wavefront's block of which is a part of its rows.  Vector instructions that no product runs beside: 11.5 issue
// slots per logit (the accumulator moved twice, half a maximum, difference, product, exponential, sum, moment and its guard).  A lane has a quarter of 16 neighbours' rows
// to itself; the quarters meet at the end, all rows together, so that the exchanges wait for one another only there.  8.7 us of the 57 that a tile takes whose
// reduction is 2048 long (main loop 45 at the clock that the power cap leaves, start 2.8).
struct EpiRowStats {
    PartSums out;
    float* token_z;                      // [padded]
    const int32_t* token;
    const float *h_unit, *w_unit;        // fp32, or null: powers of two
    float c;                             // log2 e / temperature
    int first, columns;                  // of the vocabulary in this piece
    int first_part;
    template <int kW>
    __device__ __forceinline__ void operator()(const TileCoord<kW>& tc, const Accumulators<kW>& acc, char*) const {
        constexpr int RW = kWaveRows<kW>;
        const int col0 = tc.col0();
        if (col0 >= columns) return;                       // no part of its own
        if (col0 + RW <= columns) rows<true>(tc, acc, col0);
        else rows<false>(tc, acc, col0);
    }
    template <bool kWhole, int kW>
    __device__ __forceinline__ void rows(const TileCoord<kW>& tc, const Accumulators<kW>& acc, int col0) const {
        constexpr int RW = kWaveRows<kW>;
        const int quarter = tc.lane >> 4, row0 = tc.row0() + (tc.lane & 15);
        const float w_scale = w_unit != nullptr ? *w_unit : 1.f;
        int at[kW];                                        // of the token in this block
        float unit[kW];
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            at[i] = token[row0 + i * 16] - first - col0;
            unit[i] = h_unit != nullptr ? h_unit[row0 + i * 16] * w_scale : 1.f;
        }
        RowSums r[kW];
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            auto z = [&](int j, int t) __attribute__((always_inline)) {
                const float x = accumulator(acc[i][j][t]);
                return kWhole || col0 + j * 16 + quarter * 4 + t < columns ? x : -__builtin_huge_valf();
            };
            float m = -__builtin_huge_valf();
#pragma unroll
            for (int j = 0; j < kW; ++j) {
                m = max3(z(j, 0), z(j, 1), m);
                m = max3(z(j, 2), z(j, 3), m);
            }
            r[i] = sums_of<kW>(m, c * unit[i], z);
            if (!kWhole && m == -__builtin_huge_valf()) r[i].s = r[i].t = 0.f;       // no column of this lane's (m of a NaN is NaN, and so are its sums)
            r[i].m = m * unit[i];
            if (__any(at[i] >= 0 && at[i] < RW)) {
                float x = 0.f;
#pragma unroll
                for (int j = 0; j < kW; ++j)
#pragma unroll
                    for (int t = 0; t < 4; ++t) x = at[i] == j * 16 + quarter * 4 + t ? z(j, t) : x;
                if (at[i] >= 0 && at[i] < RW && at[i] % 16 / 4 == quarter) token_z[row0 + i * 16] = x * unit[i];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int off = 16; off <= 32; off *= 2)
#pragma unroll
            for (int i = 0; i < kW; ++i)
                merge(r[i], RowSums{__shfl_xor(r[i].m, off, 64), __shfl_xor(r[i].s, off, 64), __shfl_xor(r[i].t, off, 64)}, c);
#pragma unroll
        for (int i = 0; i < kW; ++i)
            if (quarter == i % 4) out.of[(first_part + col0 / RW) * out.ld + row0 + i * 16] = f32x4{r[i].m, r[i].s, r[i].t, 0.f};
    }
};

struct RowResults {
    float *logp, *lse, *entropy;
};
// ---- dz -------------------------------------------------------------------------------------------

// Vector instructions that no product runs beside: 10 issue slots per logit (the accumulator's move, log p, exponential, factor, product, rounding and
// the way through LDS).  With what it writes 7.8 us of a tile's 50 (reduction 1536 long), as pairs 10 to 12 of 85.
// log p is a difference of rounded numbers and may come out above 0, where p has to stay at 1: far above where lse is large (2^-22 of it and more).  As pairs dz
// would leave the range that the power of two of its row was chosen for, so there every log p is bounded (630 us for 625 in 1111 fp32 rows of 1001 -> 32003); in bf16
// those of rows with |lse| from 1024 on are, in the loop that also serves blocks which the vocabulary does not fill (in all of them: 553 us for 545 in 2072 rows of
// 1536 -> 50021).
constexpr float kFarLse2 = 1024.f * kLog2E;
struct LogitGradient {
    const int32_t* live;
    const SlotGradient* of;
    const int32_t* token;
    const float *h_unit, *w_unit;        // fp32, or null: powers of two
    float c;                             // log2 e / temperature
    int first, columns;                  // of the vocabulary in this piece
    // Whether anything reads the rows of a wavefront's block: those that hold a row, and the rest of its step of 64 in the sum over rows.
    template <int kW>
    __device__ __forceinline__ bool read(const TileCoord<kW>& tc) const { return tc.row0() < (*live + kTileK - 1) / kTileK * kTileK; }
    // What is to be known of rows 16 i + (lane & 15) of a wavefront's block, asked for all at once.
    struct Row {
        float scale, lse2, along, rest, g;
        float most;                      // that log p may be
        int at;                          // of the token in this block
    };
    template <int kW>
    static __device__ __forceinline__ bool any_bounded(const Row (&row)[kW]) {
        bool x = false;
#pragma unroll
        for (int i = 0; i < kW; ++i) x |= row[i].most == 0.f;
        return __any(x);
    }
    template <int kW>
    __device__ __forceinline__ void load(Row (&row)[kW], const TileCoord<kW>& tc) const {
        const float w_scale = w_unit != nullptr ? *w_unit : 1.f;
        SlotGradient G[kW];
        float unit[kW];
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            const int slot = tc.row0() + i * 16 + (tc.lane & 15);
            G[i] = of[slot];
            row[i].at = token[slot] - first - tc.col0();
            unit[i] = h_unit != nullptr ? h_unit[slot] : 1.f;
        }
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            row[i].scale = c * (unit[i] * w_scale);
            row[i].lse2 = G[i].lse2;
            row[i].most = h_unit != nullptr || fabsf(G[i].lse2) >= kFarLse2 ? 0.f : __builtin_huge_valf();
            row[i].along = G[i].h * kLn2;
            row[i].rest = __builtin_fmaf(G[i].h, G[i].entropy, G[i].g);
            row[i].g = G[i].g;
        }
    }
    // dz of a row: store(tile column j, four neighbours).  Rows behind the last slot are zeros times W with a gradient of zero.
    template <bool kWhole, bool kBounded, int kW, class F>
    __device__ __forceinline__ void row(const Row& q, const TileCoord<kW>& tc, const Accumulators<kW>& acc, int i, F store) const {
        constexpr int RW = kWaveRows<kW>;
        const int quarter = tc.lane >> 4;
        f32x4 r[kW];
#pragma unroll
        for (int j = 0; j < kW; ++j)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const float log2p = __builtin_fmaf(accumulator(acc[i][j][t]), q.scale, -q.lse2), a = kBounded ? at_most(log2p, q.most) : log2p;
                // (where p is 0 log p may be -inf, which is not to become a NaN)
                const float x = -__builtin_amdgcn_exp2f(a) * __builtin_fmaf(q.along, fmaxf(a, -150.f), q.rest);
                r[j][t] = kWhole || tc.col0() + j * 16 + quarter * 4 + t < columns ? x : 0.f;
            }
        if (__any(q.at >= 0 && q.at < RW)) {
#pragma unroll
            for (int j = 0; j < kW; ++j)
#pragma unroll
                for (int t = 0; t < 4; ++t) r[j][t] += q.at == j * 16 + quarter * 4 + t ? q.g : 0.f;
        }
#pragma unroll
        for (int j = 0; j < kW; ++j) store(j, r[j]);
        __builtin_amdgcn_sched_barrier(0);
    }
};

// dz as bf16, once rounded: what the products with bf16 rows and weights take.  Kept in more bits it would be a second product for each result (hi + lo) or fp32
// copies of rows and weights.  Both results of 256 to 2072 rows are then off by 2.3e-3 to 2.5e-3 of their size against 64 bits, by 1.7e-3 from their own rounding alone.
struct EpiLogitGradient {
    LogitGradient gradient;
    bf16* dz;
    int64_t ld;
    template <bool kPlain, int kW>
    __device__ __forceinline__ void rows(const LogitGradient::Row (&row)[kW], const TileCoord<kW>& tc, const Accumulators<kW>& acc, char* st) const {
        constexpr int RW = kWaveRows<kW>, kStride = RW * 2 + 16;
        const int col0 = tc.col0();
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            char* const to = st + (i * 16 + (tc.lane & 15)) * kStride + 4 * (tc.lane >> 4) * 2;
            gradient.row<kPlain, !kPlain>(row[i], tc, acc, i, [&](int j, const f32x4& r) __attribute__((always_inline)) {
                *reinterpret_cast<bf16x4*>(to + j * 32) = to_bf16x4(r[0], r[1], r[2], r[3]);
            });
        }
        __builtin_amdgcn_wave_barrier();
        copy_rows_out<RW, RW * 2>(st, kStride, reinterpret_cast<char*>(dz + (int64_t)tc.row0() * ld + col0), ld * 2, RW, tc.lane);
    }
    template <int kW>
    __device__ __forceinline__ void operator()(const TileCoord<kW>& tc, const Accumulators<kW>& acc, char* lds) const {
        if (!gradient.read(tc)) return;
        char* st = wave_stage(tc, lds);
        LogitGradient::Row row[kW];
        gradient.load(row, tc);
        if (tc.col0() + kWaveRows<kW> <= gradient.columns && !gradient.any_bounded(row)) rows<true>(row, tc, acc, st);
        else rows<false>(row, tc, acc, st);
    }
};
// dz 2^z_shift as hi + lo of fp16.
struct EpiLogitGradientPairs {
    LogitGradient gradient;
    f16 *hi, *lo;
    int64_t ld;
    template <bool kWhole, int kW>
    __device__ __forceinline__ void rows(const TileCoord<kW>& tc, const Accumulators<kW>& acc, char* st) const {
        constexpr int RW = kWaveRows<kW>, kStride = RW * 4 + 16;
        LogitGradient::Row row[kW];
        gradient.load(row, tc);
        const int col0 = tc.col0();
#pragma unroll
        for (int half = 0; half < RW / 64; ++half) {       // 64 rows per pass
#pragma unroll
            for (int ii = 0; ii < 4; ++ii) {
                char* const to = st + (ii * 16 + (tc.lane & 15)) * kStride + 4 * (tc.lane >> 4) * 2;
                gradient.row<kWhole, true>(row[half * 4 + ii], tc, acc, half * 4 + ii, [&](int j, const f32x4& r) __attribute__((always_inline)) {
                    f16x4 h, l;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        h[t] = (f16)r[t];
                        l[t] = (f16)(r[t] - (float)h[t]);
                    }
                    *reinterpret_cast<f16x4*>(to + j * 32) = h;
                    *reinterpret_cast<f16x4*>(to + j * 32 + RW * 2) = l;
                });
            }
            __builtin_amdgcn_wave_barrier();
            const int64_t at = (int64_t)(tc.row0() + half * 64) * ld + col0;
            copy_rows_out<64, RW * 2>(st, kStride, reinterpret_cast<char*>(hi + at), ld * 2, 64, tc.lane);
            copy_rows_out<64, RW * 2>(st + RW * 2, kStride, reinterpret_cast<char*>(lo + at), ld * 2, 64, tc.lane);
            __builtin_amdgcn_wave_barrier();
        }
    }
    template <int kW>
    __device__ __forceinline__ void operator()(const TileCoord<kW>& tc, const Accumulators<kW>& acc, char* lds) const {
        if (!gradient.read(tc)) return;
        char* st = wave_stage(tc, lds);
        if (tc.col0() + kWaveRows<kW> <= gradient.columns) rows<true>(tc, acc, st);
        else rows<false>(tc, acc, st);
    }
};

// ---- results --------------------------------------------------------------------------------------

__device__ inline uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// What a product over all rows is to be multiplied by: 2^(most - 14) for pairs.
__device__ inline float weight_gradient_unit(const int32_t* most) { return most == nullptr || *most <= -(1 << 20) ? 1.f : ldexpf(1.f, *most - 14); }

// acc into rows and columns of a matrix that end anywhere, at any alignment of its type, through LDS so that whole lines leave (bf16 3 to 3.5 us a tile,
// fp32 8; bf16 rows that begin anywhere, by 16 bytes instead of value by value, 876 rows of 3077 -> 51202 two pieces of 291 -> 217 us).
template <class T>
struct EpiStoreAnywhere;
template <>
struct EpiStoreAnywhere<uint16_t> {                        // bf16
    uint16_t* C;
    int64_t ldc;
    int rows, cols;
    template <int kW>
    __device__ __forceinline__ void operator()(const TileCoord<kW>& tc, const Accumulators<kW>& acc, char* lds) const {
        constexpr int RW = kWaveRows<kW>, kStride = RW * 2 + 16;
        char* st = wave_stage(tc, lds);
        const int row0 = tc.row0(), col0 = tc.col0(), n_rows = min(RW, rows - row0), n_cols = min(RW, cols - col0);
        if (n_rows <= 0 || n_cols <= 0) return;
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            stage_tile_row<kW>(st, kStride, tc.lane, i * 16 + (tc.lane & 15), [&](int j) { return acc[i][j]; });
            __builtin_amdgcn_sched_barrier(0);             // one tile row's conversions at a time
        }
        __builtin_amdgcn_wave_barrier();
        if (n_cols == RW && ((reinterpret_cast<uintptr_t>(C) | (uintptr_t)(ldc * 2)) & 15u) == 0) {
            copy_rows_out<RW, RW * 2>(st, kStride, reinterpret_cast<char*>(C + (int64_t)row0 * ldc + col0), ldc * 2, n_rows, tc.lane);
            return;
        }
        typedef u32x4 __attribute__((aligned(2))) u32x4_any;
        constexpr int kLanes = RW / 8;                     // of a row, eight columns each
        const int c = tc.lane % kLanes * 8;
        for (int r = tc.lane / kLanes; r < n_rows; r += 64 / kLanes) {
            const u32x4 x = *reinterpret_cast<const u32x4*>(st + r * kStride + c * 2);
            uint16_t* const to = C + (int64_t)(row0 + r) * ldc + col0 + c;
            if (c + 8 <= n_cols) *reinterpret_cast<u32x4_any*>(to) = x;
            else
                for (int e = 0; e < 8; ++e)
                    if (c + e < n_cols) to[e] = (uint16_t)(x[e / 2] >> (e % 2 * 16));
        }
    }
};
template <>
struct EpiStoreAnywhere<float> {
    float* C;
    int64_t ldc;
    int rows, cols;
    const int32_t* most;                 // or null
    int accumulate;                      // added to what is there
    template <int kW>
    __device__ __forceinline__ void operator()(const TileCoord<kW>& tc, const Accumulators<kW>& acc, char* lds) const {
        typedef f32x4 __attribute__((aligned(4))) f32x4_any;
        constexpr int RW = kWaveRows<kW>, kStride = RW * 4 + 16;
        constexpr int kLanes = RW / 4;                     // of a row, four columns each
        char* st = wave_stage(tc, lds);
        const int col0 = tc.col0(), n_cols = min(RW, cols - col0), c = tc.lane % kLanes * 4;
        const float unit = weight_gradient_unit(most);
        if (n_cols <= 0) return;
#pragma unroll
        for (int i = 0; i < RW / 32; ++i) {                // 32 rows per pass
#pragma unroll
            for (int ii = 0; ii < 2; ++ii)
#pragma unroll
                for (int j = 0; j < kW; ++j)
                    *reinterpret_cast<f32x4*>(st + (ii * 16 + (tc.lane & 15)) * kStride + (j * 16 + 4 * (tc.lane >> 4)) * 4) = acc[2 * i + ii][j];
            __builtin_amdgcn_wave_barrier();
            const int row0 = tc.row0() + i * 32, n_rows = min(32, rows - row0);
            for (int r = tc.lane / kLanes; r < n_rows; r += 64 / kLanes) {
                f32x4 x = *reinterpret_cast<const f32x4*>(st + r * kStride + c * 4);
                x *= unit;
                float* const to = C + (int64_t)(row0 + r) * ldc + col0 + c;
                if (c + 4 <= n_cols) {
                    if (accumulate) x += *reinterpret_cast<const f32x4_any*>(to);
                    *reinterpret_cast<f32x4_any*>(to) = x;
                } else {
                    for (int e = 0; e < 4; ++e)
                        if (c + e < n_cols) to[e] = accumulate ? to[e] + x[e] : x[e];
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
};

// dhidden, as a product: in one part over the whole vocabulary straight to the rows, else fp32 parts, [parts][padded, dh_ld], to be added up
// (hidden_parts).
struct HiddenParts {
    float* of;
    int64_t ld, part;
    int most;
    int32_t* used;                       // how many there are, written by the product
};
template <class T>
struct EpiHidden {
    HiddenParts parts;
    const int32_t *live, *row_of;
    T* out;
    int64_t ld;
    int cols, whole, add;                    // whole: the only piece; add: a later one
    const int32_t* z_shift;                  // fp32, or null
    const float* w_unit;
    template <int kW>
    __device__ __forceinline__ void operator()(const TileCoord<kW>& tc, const Accumulators<kW>& acc, char* lds) const {
        constexpr int RW = kWaveRows<kW>, kStride = RW * 4 + 16;
        constexpr int kLanes = RW / 4;                     // of a row, four columns each
        char* st = wave_stage(tc, lds);
        const int col0 = tc.col0(), c = tc.lane % kLanes * 4, n_cols = min(RW, cols - col0);
        const bool direct = whole && tc.splits == 1;
        const int rows = *live;
        float* const C = parts.of + tc.split * parts.part;
        if (tc.m0 == 0 && tc.n0 == 0 && tc.split == 0 && threadIdx.x == 0) *parts.used = tc.splits;
        if (tc.row0() >= rows) return;
        // where the block's rows go, one or two to a lane (negative: nowhere); the lanes that write a row ask those
        constexpr int kHeld = (RW + 63) / 64;
        int to_row[kHeld];
        float unit[kHeld];
        if (direct) {
#pragma unroll
            for (int q = 0; q < kHeld; ++q) {
                const int slot = tc.row0() + q * 64 + tc.lane;
                const bool there = slot < rows;
                to_row[q] = there ? row_of[slot] : -1;
                unit[q] = z_shift != nullptr && there ? ldexpf(*w_unit, -z_shift[slot]) : 1.f;
            }
        }
#pragma unroll
        for (int i = 0; i < RW / 32; ++i) {                // 32 rows per pass
#pragma unroll
            for (int ii = 0; ii < 2; ++ii)
#pragma unroll
                for (int j = 0; j < kW; ++j)
                    *reinterpret_cast<f32x4*>(st + (ii * 16 + (tc.lane & 15)) * kStride + (j * 16 + 4 * (tc.lane >> 4)) * 4) = acc[2 * i + ii][j];
            __builtin_amdgcn_wave_barrier();
            const int row0 = tc.row0() + i * 32;
            if (!direct) {
                char* const dst = reinterpret_cast<char*>(C + (int64_t)row0 * parts.ld + col0);
                if (add) add_rows_out<32, RW * 4>(st, kStride, dst, parts.ld * 4, tc.lane);
                else copy_rows_out<32, RW * 4>(st, kStride, dst, parts.ld * 4, 32, tc.lane);
            } else {
#pragma unroll
                for (int pass = 0; pass < 32 * kLanes / 64; ++pass) {
                    const int r = pass * (64 / kLanes) + tc.lane / kLanes;
                    const int row = __shfl(to_row[i / 2], i % 2 * 32 + r, 64);
                    f32x4 x = *reinterpret_cast<const f32x4*>(st + r * kStride + c * 4);
                    x *= __shfl(unit[i / 2], i % 2 * 32 + r, 64);
                    if (row < 0) continue;
                    T* const to = out + row * ld + col0 + c;
                    if (c + 4 <= n_cols) store_four(to, x);
                    else
                        for (int e = 0; e < 4; ++e)
                            if (c + e < n_cols) store_one(to + e, x[e]);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
    }
    static __device__ __forceinline__ void store_one(float* to, float x) { *to = x; }
    static __device__ __forceinline__ void store_one(uint16_t* to, float x) { *to = bf16_bits(x); }
    static __device__ __forceinline__ void store_four(float* to, f32x4 x) {
        typedef f32x4 __attribute__((aligned(4))) f32x4_any;
        *reinterpret_cast<f32x4_any*>(to) = x;
    }
    static __device__ __forceinline__ void store_four(uint16_t* to, f32x4 x) {
        typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
        typedef u32x2 __attribute__((aligned(2))) u32x2_any;
        *reinterpret_cast<u32x2_any*>(to) = __builtin_bit_cast(u32x2, to_bf16x4(x[0], x[1], x[2], x[3]));
    }
};

// The sum of a row's parts: of dhidden, where they are not in place already, or of dweight.
struct PartSum {
    const float* parts;
    int64_t part, ld;
    int n, rows, cols, accumulate;
    const int32_t* most;                 // fp32: power of two of the whole, or null
    const int32_t *slot_of, *used;       // of dhidden: a row's slot, the number of parts
    int whole;                           // one part is in place already
    const int32_t* z_shift;
    const float* w_unit;                 // with z_shift
    int rows_each;                       // of a workgroup
};

}  // namespace pcm
