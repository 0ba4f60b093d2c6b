// fp32 matrices as pairs of fp16 matrices (internal header): what lets the products of an orthogonalisation run on the
// fp16 matrix cores at the accuracy of fp32.
//
// A value x is held as hi = fp16(s x) and lo = fp16(s x - hi) with s a power of two per matrix: 22 bits of significand, and
// an absolute floor of 2^-24 / s.  A product of two such matrices is hi hi + hi lo + lo hi; what is left out, lo lo, is below
// 2^-22 of it, less than what the fp32 sums round off.  (bf16 pairs carry 16 bits and are not enough: the iteration multiplies
// what is off in the directions that the matrix hardly has by up to 3.4445 per step, 485 over five.  In 64-bit arithmetic with
// the operands rounded like this, against exact operands: 1e-6 on matrices like gradients and 5e-5 on a matrix of rank one,
// where fp32 products give 2e-6 and 2e-4; with single fp16 operands 2e-3 to 0.15.)
//
// Layout: fragments of 16 rows x 32 columns, as the operand registers of v_mfma_f32_16x16x32_f16 take them.  Lane l holds row
// l & 15 and, of the columns, 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3 with g = l >> 4 (any order of the reduction index will
// do if both operands have it; with this one a lane's four values of two neighbouring accumulator tiles are its eight
// values of the fragment, so results are stored as operands without an exchange between lanes).  A fragment is 1 KB of hi,
// lane by lane, then 1 KB of lo: loads and LDS reads are contiguous and need no swizzle.  Fragments of the same 32 columns lie
// one behind the other by row, then come the next 32 columns: what a tile reads in a step is one piece of memory.
// Rows and columns are padded to multiples of 32, the padding zero.
#pragma once

#include "common.h"

namespace pcm {

typedef _Float16 f16;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;     // global memory takes them at every multiple of four bytes

constexpr int kPairRows = 16, kPairCols = 32;      // of a fragment
constexpr int kPairPart = kPairRows * kPairCols;   // values of its hi, and of its lo
constexpr int kPairFragment = 2 * kPairPart;

__host__ __device__ inline int pad32(int n) { return (n + 31) / 32 * 32; }
inline size_t pair_values(int rows, int cols) { return (size_t)pad32(rows) * (size_t)pad32(cols) * 2; }

// Where the fragment of rows 16 r .. and columns 32 c .. of a matrix of `frags` fragments of rows is.
__host__ __device__ inline int64_t pair_fragment(int64_t r, int64_t c, int64_t frags) { return (c * frags + r) * kPairFragment; }

// s x in two parts.  A value beyond the range of fp16 becomes infinite and then NaN: so does what is computed from it.
__device__ inline void split_pair(float x, f16& hi, f16& lo) {
    hi = (f16)x;
    lo = (f16)(x - (float)hi);
}

}  // namespace pcm
