// What the two directions of the log-probabilities through a vocabulary projection share (internal header).
//
// z = h W over rows that have a token: these are gathered into slots 0 .. live - 1 of a matrix of their own, so that no product runs over
// the others and nothing that those hold is met.  How many there are is known on the device only; products skip tiles beyond.
//
// fp32: operands are pairs of fp16 matrices, value times a power of two = hi + lo, 22 significand bits, and a product is three of fp16 with
// fp32 sums: a third of the 16-bit rate, several times that of fp32 instructions.  What is lost is below 2^-22 of a value, or 2^-39 of the
// largest one that shares its power of two: a row of h and of dz has one each, W has one, and so have all rows of h as they are weighted for dW.
#pragma once

#include "gemm_bf16.h"

namespace pcm {

typedef uint16_t half_bits;          // 16 bits that only pass through: bf16, or fp16

struct LinearRows {
    const void* hidden;              // [rows] of d values, ld apart
    int64_t ld;
    const void* tokens;
    int token_type;
    int rows, d, V;
};
// The gradient that reaches a slot, over the temperature (fp32: times the power of two of its row of dz).
struct SlotGradient {
    float g, h;                      // of log p, of the entropy
    float lse2, entropy;             // lse in powers of two
};
struct Slots {
    int32_t* live;                   // [1]: how many slots hold a row
    int32_t* parts;                  // [1]: backward: in how many parts the product for dhidden was done
    int32_t* most;                   // [1]: fp32, backward: the largest exponent of h 2^-z_shift
    int32_t* mosts;                  // [kMosts], kMostPitch apart: of workgroups' shares of the rows (long lists only)
    int32_t* slot_of;                // [rows]: -1 for a row without a token
    int32_t* row_of;                 // [padded]: of the slots below live
    int32_t* token;                  // [padded]: in 0 .. V - 1; -1 from live up to the next multiple of 256
    half_bits *h, *h_low;            // [padded, d64]: the hidden rows, zeros behind d and from live up to the next multiple of 256
    float* h_unit;                   // fp32: [padded]: what a row of the pairs is to be multiplied by
    int32_t* counts;                 // rows with a token per kCountRows rows (long lists only)
    int padded, d64;
};
struct SlotGradients {
    const float *lse, *dlogp, *entropy, *dentropy;       // [rows]; the last two: both or none
    float inv_t;
    SlotGradient* of;                // [padded]
    // fp32
    int32_t* z_shift;                // [padded]: a row of dz is held times 2^z_shift; beyond any number for a row of zeros
    int32_t* exponent;               // [padded]: of h 2^-z_shift (short lists only, else the largest is gathered in slots.most)
    half_bits *w_h, *w_h_low;        // [padded, d64]: h 2^(14 - most - z_shift): what dz is multiplied with for dW (null: it is not asked for)
    void* dh;                        // [rows], dh_ld apart, or null: rows without a token are made zeros
    int64_t dh_ld;
};

constexpr int kCountRows = 1024;
// (one number for all took 90 us of 7,500 rows' atomics)
constexpr int kMosts = 64, kMostPitch = 32;
constexpr int kFewRows = 16;
constexpr int kAbsmaxParts = 1024;
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct WeightSource {
    const void* w;
    int64_t ld;
    int dtype, layout, d, V;
    bool in_place;                   // bf16 that the products can read where it is
};
// Whether the projection streams past the rows, 16 at a time, or they are multiplied in tiles.  Streaming reads W once per 16 rows (from the cache after the
// first); tiles need W in place or a copy first, of fp32 as pairs after a pass for its largest value.  So
//   bf16            up to 16 rows
//   bf16, copied    [d, V] up to 64, [V, d] up to 16: there a lane's 16 bytes begin anywhere and neighbours' lie far apart, which takes three times as long
//   fp32            [d, V] up to 96, [V, d] up to 64, and up to 1024 (as many as were measured) as long as what streams past all groups is 128 MB
// Calls streamed / in tiles, us, [d, V] and [V, d]:
//   bf16          16 rows of 1024 -> 32000 17 / 43 and 20 / 26, of 4096 -> 65536 100 / 115 and 120 / 140; 32 rows 125 / 116 and 193 / 140
//   bf16, copied  [d, V] 64 of 1023 -> 32003 42 / 44, of 4095 -> 65531 287 / 329; 80 50 / 43 and 353 / 326
//                 [V, d] 16 of 1023 -> 32003 50 / 44, of 4095 -> 65531 276 / 370; 32 93 / 44 and 548 / 371
//   fp32          64 of 1024 -> 32003 68 / 105 and 90 / 102, of 4096 -> 65536 432 / 998 and 649 / 1092; 100 108 / 106 and 151 / 104, 732 / 1000 and 1073 / 1093
//                 1024 of 256 -> 1024 17 / 26 and 23 / 26; 256 of 512 -> 4096 23 / 33 and 31 / 32, 512 39 / 35 and 55 / 34
inline bool streams(int rows, const WeightSource& src) {
    const bool by_token = src.layout == PCM_WEIGHT_OUT_IN;
    if (src.dtype != PCM_F32) return rows <= (src.in_place || by_token ? kFewRows : 64);
    return rows <= (by_token ? 64 : 96) || (rows <= 1024 && (int64_t)ceil_div(rows, kFewRows) * src.d * src.V * 4 <= 128 << 20);
}
// Scratch for a copy of up to `columns` of the vocabulary, rows of it, or of d, `ld` apart.
struct WeightCopy {
    half_bits *w, *low;
    int64_t ld;
    float* absmax;                   // fp32: [absmax_parts]
    int absmax_parts;
    float* unit;                     // fp32: [1]: what the pairs are to be multiplied by
    int columns;
};
// Rows of a matrix by workgroups of 256: 2^lanes neighbours of `each` values in a row, the other threads rows; a row in `chunks`.
struct RowSplit {
    int lanes, chunks, blocks;
    RowSplit() = default;
    RowSplit(int rows, int64_t cols, int each) {
        lanes = 0;
        while (lanes < 8 && ((int64_t)each << lanes) < cols) ++lanes;
        chunks = (int)((cols + ((int64_t)each << lanes) - 1) / ((int64_t)each << lanes));
        blocks = ((rows + (256 >> lanes) - 1) >> (8 - lanes)) * chunks;
    }
};
// The largest size of a value of the weight, part by part.
struct WeightAbsmax {
    const float* w;
    int64_t ld;
    int rows, cols, parts;
    RowSplit split;
    float* out;
};
// A piece of the weight to its copy, zeros behind its columns up to ld_to.
struct WeightPiece {
    const void* w;
    int64_t ld;
    int rows, cols;
    half_bits *to, *low;
    int64_t ld_to;
    RowSplit split;
    const float* absmax;             // fp32
    int absmax_parts;
    float* unit;
};
// A piece of the columns of the vocabulary as an operand.
struct WeightOperand {
    const half_bits *w, *low;
    int64_t ld;
};

inline int round_up(int x, int to) { return (x + to - 1) / to * to; }

Slots carve_slots(Carver& c, int rows, int d, int dtype);
SlotGradients carve_gradients(Carver& c, const Slots& slots, int dtype);
// sums_along_rows: a product of the call has the row's index as its reduction index.
WeightSource weight_source(const void* w, int64_t ld, int dtype, int layout, int d, int V, bool sums_along_rows);
// columns: of the pieces that the caller works in.
WeightCopy carve_weight(Carver& c, const WeightSource& src, int columns);
int copy_columns(const WeightSource& src);               // of a piece that is copied
// Rows to slots; hidden rows, and what reaches them, to the slots' matrices; the first `columns` of the weight to their copy, if it needs one.
void prepare_operands(const LinearRows& in, const Slots& slots, const SlotGradients* grads, const WeightSource& src, const WeightCopy& copy, int columns,
                      hipStream_t s);
// The operand of a piece, copied if it has to be and is not the first one.
WeightOperand weight_operand(const WeightSource& src, const WeightCopy& copy, int first, int columns, hipStream_t s);

// What both entry points ask of their common arguments.
int check_linear(const void* hidden, int64_t hidden_ld, const void* weight, int64_t weight_ld, int layout, int dtype, const void* tokens,
                 int token_type, int64_t rows, int d, int V, float temperature);

// An accumulator's value, moved where it is asked for: left to itself the compiler moves all 256 of a lane ahead of the first branch of an
// epilogue, and from there to scratch memory.
__device__ __forceinline__ float accumulator(float x) {
    float r;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(r) : "a"(x));
    return r;
}

// A product of all slots (M, or the reduction index) with whatever B is.
template <bool kThirds>
inline BoundedProblem<kThirds> slot_product(const Slots& slots, int rows_role) {
    BoundedProblem<kThirds> p{};
    p.splits = 1;
    p.kept = slots.live;
    p.kept_max = slots.padded;
    p.rows_per_kept = 1;
    p.rows_role = rows_role;
    return p;
}
template <bool kThirds>
inline void set_a(BoundedProblem<kThirds>& p, const half_bits* a, const half_bits* low, int64_t ld) {
    auto q = [](const half_bits* x) { return reinterpret_cast<const bf16*>(x); };
    p.A = q(a);
    p.A2 = q(a);
    p.A3 = q(kThirds ? low : a);
    p.lda = ld;
}
// (Rows of operands of this library's own go on with zeros, those in place end with whole 16-byte pieces.)
template <int kLayout, bool kThirds>
inline void set_b(BoundedProblem<kThirds>& p, const half_bits* b, const half_bits* low, int64_t ld, int N_real, int K_real) {
    auto q = [](const half_bits* x) { return reinterpret_cast<const bf16*>(x); };
    p.B = q(b);
    p.B2 = q(kThirds ? low : b);
    p.B3 = q(b);
    p.ldb = ld;
    p.N_real = kLayout == kKByRows ? round_up(N_real, 8) : N_real;
    p.K_real = kLayout == kRowsByK ? round_up(K_real, 8) : K_real;
    p.N = N_real;                        // to whole tiles by the launch
    p.K1 = round_up(K_real, kTileK);
}
// A product with its epilogue, ready to be launched.
template <bool kThirds, int kLayoutA, int kLayoutB, class E>
struct SlotProduct {
    using Problem = BoundedProblem<kThirds>;
    using Epilogue = E;
    static constexpr int kLayA = kLayoutA, kLayB = kLayoutB;
    Problem p;
    E epi;
    int kW;
    unsigned grid;
    SlotProduct(Problem problem, int tile, const E& e) : p(problem), epi(e), kW(tile) {
        p.N = round_up(p.N, 32 * kW);
        const int tiles_n = p.N / (32 * kW), tiles = p.M / (32 * kW) * tiles_n;
        grid = (unsigned)tiles * (unsigned)p.splits;
        if (p.splits == 1) p.part_cost = 0;
        if (p.part_cost == 0) return;
        grid = (unsigned)part_workgroups(tiles);           // the most that any number of rows takes
        const int rows_m = p.M / (32 * kW), each = kTileM / (32 * kW);      // row tiles, and those of 256 rows
        for (int live = std::min(ceil_div(rows_m, each), 2048 / (each * tiles_n) + 1); live > 0; --live) {
            const int n = std::min(rows_m, live * each) * tiles_n;
            grid = std::max(grid, (unsigned)(part_workgroups(n) * parts_for(n, p.part_steps, p.splits, p.part_cost)));
        }
    }
    int steps() const { return p.K1 / kTileK * (kThirds ? 3 : 1) / p.splits; }
    void launch(hipStream_t s) const {
        if (kW == kLargeTile) gemm_bounded<Problem, E, kLayA, kLayB, kLargeTile, kRingSlots><<<grid, kGemmThreads, 0, s>>>(p, epi);
        else if (grid <= 256 && steps() >= kDeepSteps) gemm_bounded<Problem, E, kLayA, kLayB, kSmallTile, kDeepRingSlots><<<grid, kGemmThreads, 0, s>>>(p, epi);   // as launch_gemm_tile
        else gemm_bounded<Problem, E, kLayA, kLayB, kSmallTile, kRingSlots><<<grid, kGemmThreads, 0, s>>>(p, epi);
    }
};
// Two products that depend on the same launches, on small tiles, as one launch where each leaves CUs idle (a launch of its own takes as long to
// begin and end as a few steps).
template <class A, class B>
__global__ __launch_bounds__(kGemmThreads, 2) void gemm_bounded_pair(typename A::Problem p, typename A::Epilogue e, int first, typename B::Problem q,
                                                                    typename B::Epilogue f) {
    __shared__ OperandRing<kSmallTile, kRingSlots> smem;
    const int block = blockIdx.x;
    if (block < first) gemm_tile<A::kLayA, A::kLayB, true>(p, e, block, smem);
    else gemm_tile<B::kLayA, B::kLayB, true>(q, f, block - first, smem);
}
template <class A, class B>
inline void launch_pair(const A& a, const B& b, hipStream_t s) {
    const int first = round_up((int)a.grid, kNumXcd);
    if (a.kW != kSmallTile || b.kW != kSmallTile || first + b.grid > 512) {
        a.launch(s);
        b.launch(s);
        return;
    }
    gemm_bounded_pair<A, B><<<first + b.grid, kGemmThreads, 0, s>>>(a.p, a.epi, first, b.p, b.epi);
}

}  // namespace pcm
