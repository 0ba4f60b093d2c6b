// Gradient of the log-probabilities through a vocabulary projection, in the hidden rows and in the projection.
//
// Piece by piece of the vocabulary:
//   z = h W of the piece; the epilogue makes dz of it (log p = z / temperature - lse is known) and writes that, the only matrix of rows x vocabulary
//       there is, in bf16 (fp32: as a pair of fp16)
//   dhidden += dz W^T, over the piece
//   dW of the piece = h^T dz, over all rows at once, so that it is written once and rounded once
// Six operations per row, value of a row and token, all on the matrix cores.
#include "linear_logprobs.h"

#include <type_traits>

namespace pcm {
namespace {

typedef _Float16 f16;
typedef __attribute__((ext_vector_type(4))) f16 f16x4;

// ---- dz -------------------------------------------------------------------------------------------

// Vector instructions that no product runs beside: 10 issue slots per logit (the accumulator's move, log p, exponential, factor, product, rounding and
// the way through LDS).
struct LogitGradient {
    const SlotGradient* of;
    const int32_t* token;
    const float *h_unit, *w_unit;        // fp32, or null: powers of two
    float c;                             // log2 e / temperature
    int first, columns;                  // of the vocabulary in this piece
    // What is to be known of rows 16 i + (lane & 15) of a wavefront's block, asked for all at once.
    struct Row {
        float scale, lse2, along, rest, g;
        int at;                          // of the token in this block
    };
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
            row[i].along = G[i].h * kLn2;
            row[i].rest = __builtin_fmaf(G[i].h, G[i].entropy, G[i].g);
            row[i].g = G[i].g;
        }
    }
    // dz of a row: store(tile column j, four neighbours).  Rows behind the last slot are zeros times W with a gradient of zero.
    template <bool kWhole, int kW, class F>
    __device__ __forceinline__ void row(const Row& q, const TileCoord<kW>& tc, const Accumulators<kW>& acc, int i, F store) const {
        constexpr int RW = kWaveRows<kW>;
        const int quarter = tc.lane >> 4;
        f32x4 r[kW];
#pragma unroll
        for (int j = 0; j < kW; ++j)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const float a = __builtin_fmaf(accumulator(acc[i][j][t]), q.scale, -q.lse2);
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

// dz as bf16.
struct EpiLogitGradient {
    LogitGradient gradient;
    bf16* dz;
    int64_t ld;
    template <bool kWhole, int kW>
    __device__ __forceinline__ void rows(const TileCoord<kW>& tc, const Accumulators<kW>& acc, char* st) const {
        constexpr int RW = kWaveRows<kW>, kStride = RW * 2 + 16;
        LogitGradient::Row row[kW];
        gradient.load(row, tc);
        const int col0 = tc.col0();
#pragma unroll
        for (int i = 0; i < kW; ++i) {
            char* const to = st + (i * 16 + (tc.lane & 15)) * kStride + 4 * (tc.lane >> 4) * 2;
            gradient.row<kWhole>(row[i], tc, acc, i, [&](int j, const f32x4& r) __attribute__((always_inline)) {
                *reinterpret_cast<bf16x4*>(to + j * 32) = to_bf16x4(r[0], r[1], r[2], r[3]);
            });
        }
        __builtin_amdgcn_wave_barrier();
        copy_rows_out<RW, RW * 2>(st, kStride, reinterpret_cast<char*>(dz + (int64_t)tc.row0() * ld + col0), ld * 2, RW, tc.lane);
    }
    template <int kW>
    __device__ __forceinline__ void operator()(const TileCoord<kW>& tc, const Accumulators<kW>& acc, char* lds) const {
        char* st = wave_stage(tc, lds);
        if (tc.col0() + kWaveRows<kW> <= gradient.columns) rows<true>(tc, acc, st);
        else rows<false>(tc, acc, st);
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
                gradient.row<kWhole>(row[half * 4 + ii], tc, acc, half * 4 + ii, [&](int j, const f32x4& r) __attribute__((always_inline)) {
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
        char* st = wave_stage(tc, lds);
        if (tc.col0() + kWaveRows<kW> <= gradient.columns) rows<true>(tc, acc, st);
        else rows<false>(tc, acc, st);
    }
};

// ---- results --------------------------------------------------------------------------------------

__device__ inline uint16_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// What a product over all rows is to be multiplied by: 2^(most - 14) for pairs.
__device__ inline float weight_gradient_unit(const int32_t* most) { return most == nullptr || *most <= -(1 << 20) ? 1.f : ldexpf(1.f, *most - 14); }

// acc into rows and columns of a matrix that end anywhere, at any alignment of its type, through LDS so that whole lines leave.
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
        uint16_t* const to = C + (int64_t)row0 * ldc + col0;
        if (n_cols == RW && ((reinterpret_cast<uintptr_t>(C) | (uintptr_t)(ldc * 2)) & 15u) == 0) {
            copy_rows_out<RW, RW * 2>(st, kStride, reinterpret_cast<char*>(to), ldc * 2, n_rows, tc.lane);
            return;
        }
        for (int r = 0; r < n_rows; ++r)
            for (int c = tc.lane; c < n_cols; c += 64) to[r * ldc + c] = *reinterpret_cast<const uint16_t*>(st + r * kStride + c * 2);
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
        const int rows = direct ? *live : 0x7fffffff;
        float* const C = parts.of + tc.split * parts.part;
        if (tc.m0 == 0 && tc.n0 == 0 && tc.split == 0 && threadIdx.x == 0) *parts.used = tc.splits;
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
// 1024 columns of some rows a workgroup.
template <class T>
__global__ __launch_bounds__(256) void linear_sum_parts(PartSum q, T* out, int64_t ld) {
    const int i = (blockIdx.x * 256 + threadIdx.x) * 4, first = (blockIdx.y * 65535 + blockIdx.z) * q.rows_each;
    const int n = q.used != nullptr ? *q.used : q.n;
    if ((q.whole && n == 1) || i >= q.cols) return;
    const float unit = weight_gradient_unit(q.most);
    for (int row = first; row < min(q.rows, first + q.rows_each); ++row) {
        const int slot = q.slot_of != nullptr ? q.slot_of[row] : row;
        if (slot < 0) continue;                            // zeros already
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        const float* from = q.parts + (int64_t)slot * q.ld + i;
#pragma unroll 4
        for (int p = 0; p < n; ++p) x += *reinterpret_cast<const f32x4*>(from + p * q.part);
        if (q.z_shift != nullptr) x *= ldexpf(*q.w_unit, -q.z_shift[slot]);
        x *= unit;
        T* const to = out + (int64_t)row * ld + i;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (i + e >= q.cols) break;
            if constexpr (sizeof(T) == 4) to[e] = q.accumulate ? to[e] + x[e] : x[e];
            else to[e] = bf16_bits(x[e]);
        }
    }
}
void sum_parts(PartSum q, void* out, int64_t ld, int dtype, hipStream_t s) {
    q.rows_each = std::max(1, std::min(8, ceil_div(q.cols, 1024) * ceil_div(q.rows, 2048)));      // (2048 workgroups or so)
    const int blocks = ceil_div(q.rows, q.rows_each);
    const dim3 grid((unsigned)ceil_div(q.cols, 1024), (unsigned)ceil_div(blocks, 65535), (unsigned)std::min(blocks, 65535));
    if (dtype == PCM_F32) linear_sum_parts<float><<<grid, 256, 0, s>>>(q, static_cast<float*>(out), ld);
    else linear_sum_parts<uint16_t><<<grid, 256, 0, s>>>(q, static_cast<uint16_t*>(out), ld);
}

// ---- host side --------------------------------------------------------------------------------------

// Tile and parts of the reduction of a product of M x N whose reduction takes `steps`, by an estimate: a step of the large tile takes 0.94 us, of the
// small one 0.46 (see tile_for); parts are written and read at 4.8 TB/s.
constexpr int kMostParts = 16;
struct ProductPlan {
    int kW, parts, cost;             // parts; what one costs, in steps
    ProductPlan() : kW(kSmallTile), parts(1), cost(1) {}
    ProductPlan(int M, int N, int steps) {
        double best = 1e30;
        for (const int tile : {kLargeTile, kSmallTile}) {
            const double step = tile == kLargeTile ? 0.94 : 0.46;
            const int tiles = ceil_div(M, 32 * tile) * ceil_div(N, 32 * tile), each = 1 + (int)(2.0 * M * N * 4.0 / 4.8e6 / step);
            const int n = parts_for(tiles, steps, std::min(kMostParts, std::max(1, steps / 8)), each);
            const double time = step * (((tiles * n + 255) / 256) * (ceil_div(steps, n) + 10) + (n > 1 ? n * each + 6 : 0));
            if (time < best) {
                best = time;
                kW = tile;
                parts = n;
                cost = each;
            }
        }
    }
};

struct BackwardPlan {
    int columns;                     // of a piece
    int64_t z_ld;
    Slots slots;
    SlotGradients grads;
    WeightCopy copy;
    half_bits *z, *z_low;            // [padded, z_ld]
    int z_tile;
    ProductPlan dh, dw;
    HiddenParts dh_parts;
    float* dw_parts;
    int dw_rows, dw_ld;              // of a part
    int pieces, dh_steps;            // dh_steps: of the first piece, in which all pieces' parts are chosen
    size_t bytes;
};
// `dw_direct`: whole products go straight to dweight.
BackwardPlan plan_backward(void* workspace, int rows, const WeightSource& src) {
    Carver c(workspace);
    BackwardPlan b{};
    b.slots = carve_slots(c, rows, src.d, src.dtype);
    b.grads = carve_gradients(c, b.slots, src.dtype);
    const int width = src.dtype == PCM_F32 ? 4 : 2;
    // at most 1 GB of dz
    int64_t columns = ((int64_t)1 << 30) / ((int64_t)b.slots.padded * width) / kTileN * kTileN;
    if (!src.in_place) columns = std::min<int64_t>(columns, copy_columns(src));
    b.columns = (int)std::min<int64_t>(std::max<int64_t>(columns, kTileN), round_up(src.V, kTileN));
    b.copy = carve_weight(c, src, b.columns);
    b.z_ld = b.columns;
    const size_t z = (size_t)b.slots.padded * (size_t)b.z_ld + kTileM;
    b.z = c.take<half_bits>(z);
    if (src.dtype == PCM_F32) b.z_low = c.take<half_bits>(z);
    b.z_tile = rows <= 128 ? kSmallTile : tile_for(b.slots.padded, b.columns, 1);
    b.pieces = ceil_div(src.V, b.columns);
    HiddenParts& h = b.dh_parts;
    h.ld = round_up(src.d, kTileN);
    h.part = (int64_t)b.slots.padded * h.ld;
    h.used = b.slots.parts;
    b.dh_steps = b.columns / kTileK * (width == 4 ? 3 : 1);
    b.dh = ProductPlan(b.slots.padded, (int)h.ld, b.dh_steps);
    const int tile = 32 * b.dh.kW;
    // Fewer rows with a token than rows take more parts: as many as fill the chip with one tile of rows, in at most 256 MB
    const int64_t room = ((int64_t)64 << 20) / h.part, alone = ceil_div(256, (kTileM / tile) * ceil_div(src.d, tile));
    h.most = (int)std::max<int64_t>(b.dh.parts, std::min<int64_t>({room, alone, kMostParts, std::max(1, b.dh_steps / 8)}));
    if (rows <= kTileM) h.most = b.dh.parts;
    if (h.most > 1 || b.pieces > 1) h.of = c.take<float>((size_t)(h.most * h.part));
    const int d256 = round_up(src.d, kTileM);
    b.dw_rows = src.layout == PCM_WEIGHT_OUT_IN ? b.columns : d256;
    b.dw_ld = src.layout == PCM_WEIGHT_OUT_IN ? d256 : b.columns;
    b.dw = ProductPlan(b.dw_rows, b.dw_ld, b.slots.padded / kTileK * (width == 4 ? 3 : 1));
    if (b.dw.parts > 1) b.dw_parts = c.take<float>((size_t)b.dw.parts * b.dw_rows * b.dw_ld);
    b.bytes = c.used();
    return b;
}

struct BackwardOut {
    void* dh;
    int64_t dh_ld;
    void* dw;
    int64_t dw_ld;
    int dw_dtype, accumulate;
};

template <bool kThirds, int kLayW>
void logit_gradient(const BackwardPlan& b, const WeightSource& src, const WeightOperand& w, int rows, int first, int columns, float c, hipStream_t s) {
    BoundedProblem<kThirds> p = slot_product<kThirds>(b.slots, kRowsAreM);
    p.M = rows <= 128 ? 128 : b.slots.padded;
    set_a(p, b.slots.h, b.slots.h_low, b.slots.d64);
    set_b<kLayW>(p, w.w, w.low, w.ld, columns, src.d);
    const LogitGradient gradient{b.grads.of, b.slots.token, kThirds ? b.slots.h_unit : nullptr, kThirds ? b.copy.unit : nullptr, c, first, columns};
    if constexpr (kThirds) {
        const EpiLogitGradientPairs epi{gradient, reinterpret_cast<f16*>(b.z), reinterpret_cast<f16*>(b.z_low), b.z_ld};
        SlotProduct<kThirds, kRowsByK, kLayW, EpiLogitGradientPairs>(p, b.z_tile, epi).launch(s);
    } else {
        const EpiLogitGradient epi{gradient, reinterpret_cast<bf16*>(b.z), b.z_ld};
        SlotProduct<kThirds, kRowsByK, kLayW, EpiLogitGradient>(p, b.z_tile, epi).launch(s);
    }
}

template <bool kThirds, int kLayW>
auto hidden_gradient(const BackwardPlan& b, const WeightSource& src, const WeightOperand& w, int first, int columns, const BackwardOut& out) {
    using T = std::conditional_t<kThirds, float, uint16_t>;
    BoundedProblem<kThirds> p = slot_product<kThirds>(b.slots, kRowsAreM);
    p.M = b.slots.padded;
    p.splits = b.dh_parts.most;
    p.part_cost = b.dh.cost;
    p.part_steps = b.dh_steps;
    set_a(p, b.z, b.z_low, b.z_ld);
    set_b<kLayW>(p, w.w, w.low, w.ld, src.d, columns);
    const EpiHidden<T> epi{b.dh_parts, b.slots.live, b.slots.row_of, static_cast<T*>(out.dh), out.dh_ld, src.d, b.pieces == 1, first > 0,
                           kThirds ? b.grads.z_shift : nullptr, kThirds ? b.copy.unit : nullptr};
    return SlotProduct<kThirds, kRowsByK, kLayW, EpiHidden<T>>(p, b.dh.kW, epi);
}

template <bool kThirds>
BoundedProblem<kThirds> weight_problem(const BackwardPlan& b, const WeightSource& src, int columns) {
    BoundedProblem<kThirds> p = slot_product<kThirds>(b.slots, kRowsAreK);
    const half_bits *h = kThirds ? b.grads.w_h : b.slots.h, *h_low = kThirds ? b.grads.w_h_low : nullptr;
    p.splits = b.dw.parts;
    // (both operands are of this call's scratch, whole tiles of them: the bounds are those of the scratch)
    if (src.layout == PCM_WEIGHT_OUT_IN) {
        set_a(p, b.z, b.z_low, b.z_ld);
        set_b<kKByRows>(p, h, h_low, b.slots.d64, src.d, b.slots.padded);
        p.M = round_up(columns, kTileM);
    } else {
        set_a(p, h, h_low, b.slots.d64);
        set_b<kKByRows>(p, b.z, b.z_low, b.z_ld, columns, b.slots.padded);
        p.M = round_up(src.d, kTileM);
    }
    return p;
}

// What both gradients take of a piece, beside one another where they are small.
template <bool kThirds, int kLayDh>
void piece_gradients(const BackwardPlan& b, const WeightSource& src, const WeightOperand& w, int first, int columns, const BackwardOut& out, hipStream_t s) {
    const bool by_token = src.layout == PCM_WEIGHT_OUT_IN;
    const int rows = by_token ? columns : src.d, cols = by_token ? src.d : columns;
    const int64_t at = by_token ? first * out.dw_ld : first;
    const int32_t* most = kThirds ? b.slots.most : nullptr;
    auto hidden = [&] { return hidden_gradient<kThirds, kLayDh>(b, src, w, first, columns, out); };
    if (out.dw == nullptr) return hidden().launch(s);
    const BoundedProblem<kThirds> p = weight_problem<kThirds>(b, src, columns);
    auto both = [&](const auto& epi) {
        const SlotProduct<kThirds, kKByRows, kKByRows, std::decay_t<decltype(epi)>> weight(p, b.dw.kW, epi);
        if (out.dh != nullptr) launch_pair(hidden(), weight, s);
        else weight.launch(s);
    };
    if (b.dw.parts > 1) {
        const EpiStoreF32 epi{b.dw_parts, b.dw_ld, (int64_t)b.dw_rows * b.dw_ld, 0, nullptr, FinalPanel{}};
        if (out.dh != nullptr) hidden().launch(s);
        SlotProduct<kThirds, kKByRows, kKByRows, EpiStoreF32>(p, b.dw.kW, epi).launch(s);
        const PartSum q{b.dw_parts, (int64_t)b.dw_rows * b.dw_ld, b.dw_ld, b.dw.parts, rows, cols, out.accumulate, most};
        sum_parts(q, static_cast<char*>(out.dw) + at * (out.dw_dtype == PCM_F32 ? 4 : 2), out.dw_ld, out.dw_dtype, s);
    } else if (out.dw_dtype == PCM_F32) {
        both(EpiStoreAnywhere<float>{static_cast<float*>(out.dw) + at, out.dw_ld, rows, cols, most, out.accumulate});
    } else if constexpr (!kThirds) {
        both(EpiStoreAnywhere<uint16_t>{static_cast<uint16_t*>(out.dw) + at, out.dw_ld, rows, cols});
    }
}

template <bool kThirds>
void backward(const BackwardPlan& b, const WeightSource& src, int rows, float c, const BackwardOut& out, hipStream_t s) {
    for (int first = 0; first < src.V; first += b.columns) {
        const int columns = std::min(b.columns, src.V - first);
        const WeightOperand w = weight_piece(src, b.copy, first, columns, s);
        if (src.layout == PCM_WEIGHT_OUT_IN) {
            logit_gradient<kThirds, kRowsByK>(b, src, w, rows, first, columns, c, s);
            piece_gradients<kThirds, kKByRows>(b, src, w, first, columns, out, s);
        } else {
            logit_gradient<kThirds, kKByRows>(b, src, w, rows, first, columns, c, s);
            piece_gradients<kThirds, kRowsByK>(b, src, w, first, columns, out, s);
        }
    }
    if (out.dh == nullptr || b.dh_parts.of == nullptr) return;
    PartSum q{b.dh_parts.of, b.dh_parts.part, b.dh_parts.ld, 0, rows, src.d, 0, nullptr};
    q.used = b.dh_parts.used;
    q.whole = b.pieces == 1;
    q.slot_of = b.slots.slot_of;
    q.z_shift = kThirds ? b.grads.z_shift : nullptr;
    q.w_unit = kThirds ? b.copy.unit : nullptr;
    sum_parts(q, out.dh, out.dh_ld, src.dtype, s);
}

}  // namespace
}  // namespace pcm

using namespace pcm;

extern "C" {

PCM_API size_t pcm_linear_logprobs_backward_workspace_bytes(int64_t rows, int d, int V, int dtype, int weight_layout, const void* weight,
                                                            int64_t weight_ld) {
    const void* const fine = reinterpret_cast<const void*>((uintptr_t)256);
    if (rows < 1 || check_linear(fine, d, weight, weight_ld, weight_layout, dtype, fine, PCM_TOKEN_U8, rows, d, V, 1.f) != PCM_OK) return 0;
    return plan_backward(nullptr, (int)rows, weight_source(weight, weight_ld, dtype, weight_layout, d, V)).bytes;
}

PCM_API int pcm_linear_logprobs_backward(const void* hidden, int64_t hidden_ld, const void* weight, int64_t weight_ld, int weight_layout,
                                         int dtype, const void* tokens, int token_type, int64_t rows, int d, int V, float temperature,
                                         const float* lse, const float* dlogp, const float* entropy, const float* dentropy, void* dhidden,
                                         int64_t dhidden_ld, void* dweight, int64_t dweight_ld, int dweight_dtype, int accumulate,
                                         void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_linear(hidden, hidden_ld, weight, weight_ld, weight_layout, dtype, tokens, token_type, rows, d, V, temperature);
    if (rc == PCM_EINVAL || (entropy == nullptr) != (dentropy == nullptr) || (!dhidden && !dweight)) return PCM_EINVAL;
    auto off = [](const void* p, int size) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(size - 1)) != 0; };
    if (dhidden && (dhidden_ld < d || off(dhidden, dtype == PCM_F32 ? 4 : 2))) return PCM_EINVAL;
    if (dweight && (dweight_ld < (weight_layout == PCM_WEIGHT_OUT_IN ? d : V) ||
                    (dweight_dtype != PCM_F32 && (dweight_dtype != PCM_BF16 || dtype != PCM_BF16 || accumulate)) ||
                    off(dweight, dweight_dtype == PCM_F32 ? 4 : 2)))
        return PCM_EINVAL;
    if (rows > 0 && (!lse || !dlogp || off(lse, 4) || off(dlogp, 4) || off(entropy, 4) || off(dentropy, 4))) return PCM_EINVAL;
    if (rc != PCM_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (rows == 0) {
        if (!dweight || accumulate) return PCM_OK;
        const bool by_token = weight_layout == PCM_WEIGHT_OUT_IN;
        const PartSum none{nullptr, 0, 0, 0, by_token ? V : d, by_token ? d : V, 0, nullptr};
        sum_parts(none, dweight, dweight_ld, dweight_dtype, s);
        return launch_status();
    }
    const WeightSource src = weight_source(weight, weight_ld, dtype, weight_layout, d, V);
    BackwardPlan b = plan_backward(workspace, (int)rows, src);
    if (!workspace_ok(workspace, workspace_bytes, b.bytes)) return PCM_EWORKSPACE;
    const LinearRows in{hidden, hidden_ld, tokens, token_type, (int)rows, d, V};
    const float inv_t = 1.f / temperature, c = inv_t * kLog2E;
    b.grads.lse = lse; b.grads.dlogp = dlogp; b.grads.entropy = entropy; b.grads.dentropy = dentropy;
    b.grads.inv_t = inv_t;
    b.grads.dh = dhidden;
    b.grads.dh_ld = dhidden_ld;
    const BackwardOut out{dhidden, dhidden_ld, dweight, dweight_ld, dweight_dtype, accumulate};
    StageTimer t(ST_LINEAR_LOGPROBS_GRAD, s);
    gather_slots(in, b.slots, &b.grads, dtype, s);
    prepare_weight(src, b.copy, s);
    if (dtype == PCM_F32) backward<true>(b, src, (int)rows, c, out, s);
    else backward<false>(b, src, (int)rows, c, out, s);
    return launch_status();
}

}  // extern "C"
