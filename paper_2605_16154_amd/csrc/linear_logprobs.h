// What the two directions of the log-probabilities through a vocabulary projection share (internal header).
//
// z = h W over rows that have a token: these are gathered into slots 0 .. live - 1 of a matrix of their own, so that no product runs over
// the others and nothing that those hold is met.  How many there are is known on the device only; products skip tiles beyond.
//
// fp32: operands are pairs of fp16 matrices, value times a power of two = hi + lo, 22 significand bits, and a product is three of fp16 with
// fp32 sums: a third of the 16-bit rate, several times that of fp32 instructions.  What is lost is below 2^-22 of a value, or 2^-40 of the
// largest one that shares its power of two: a row of h and of dz has one each, W has one.
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
    int32_t* most;                   // [1]: fp32, backward: the largest exponent of h 2^-z_shift
    int32_t* slot_of;                // [rows]: -1 for a row without a token
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
    int32_t* z_shift;                // [padded]: a row of dz is held times 2^z_shift
    half_bits *w_h, *w_h_low;        // [padded, d64]: h 2^(14 - most - z_shift): what dz is multiplied with for dW
};

constexpr int kCountRows = 1024;
constexpr int kFewRows = 16;         // rows up to which the projection streams past them instead of being multiplied in tiles
constexpr int kAbsmaxParts = 1024;
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

struct WeightSource {
    const void* w;
    int64_t ld;
    int dtype, layout, d, V;
    bool in_place;                   // bf16 that the products can read where it is
};
// Scratch for a copy of up to `columns` of the vocabulary, rows of it, or of d, `ld` apart.
struct WeightCopy {
    half_bits *w, *low;
    int64_t ld;
    float* absmax;                   // fp32: [kAbsmaxParts]
    float* unit;                     // fp32: [1]: what the pairs are to be multiplied by
    int columns;
};
// A piece of the columns of the vocabulary as an operand.
struct WeightOperand {
    const half_bits *w, *low;
    int64_t ld;
};

inline int round_up(int x, int to) { return (x + to - 1) / to * to; }

Slots carve_slots(Carver& c, int rows, int d, int dtype);
SlotGradients carve_gradients(Carver& c, const Slots& slots, int dtype);
// Rows to slots; hidden rows, and what reaches them, to the slots' matrices.
void gather_slots(const LinearRows& in, const Slots& slots, const SlotGradients* grads, int dtype, hipStream_t s);
WeightSource weight_source(const void* w, int64_t ld, int dtype, int layout, int d, int V);
// columns: of the pieces that the caller works in.
WeightCopy carve_weight(Carver& c, const WeightSource& src, int columns);
int copy_columns(const WeightSource& src);               // of a piece that is copied
void prepare_weight(const WeightSource& src, const WeightCopy& copy, hipStream_t s);     // once per call
WeightOperand weight_piece(const WeightSource& src, const WeightCopy& copy, int first, int columns, hipStream_t s);

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
template <bool kThirds, int kLayA, int kLayB, class Epilogue>
inline void launch_slot_product(BoundedProblem<kThirds> p, int kW, const Epilogue& epi, hipStream_t s) {
    p.N = round_up(p.N, 32 * kW);
    const unsigned grid = (unsigned)(p.M / (32 * kW)) * (unsigned)(p.N / (32 * kW)) * (unsigned)p.splits;
    if (kW == kLargeTile) gemm_bounded<BoundedProblem<kThirds>, Epilogue, kLayA, kLayB, kLargeTile, kRingSlots><<<grid, kGemmThreads, 0, s>>>(p, epi);
    else gemm_bounded<BoundedProblem<kThirds>, Epilogue, kLayA, kLayB, kSmallTile, kRingSlots><<<grid, kGemmThreads, 0, s>>>(p, epi);
}

}  // namespace pcm
