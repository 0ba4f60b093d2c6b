// Log-probabilities of tokens through a vocabulary projection, without the logits.
//
//   slots      rows with a token -> slots (linear_logprobs.h), hidden rows gathered
//   products   z = h W on the matrix cores; the epilogue turns a wavefront's block of logits into three numbers per row: largest logit, sum of
//              2^a and of 2^a a, a = (z - largest) log2 e / temperature; the token's logit is written down where it passes by
//   join       the blocks of a row -> log-sum-exp, log p, entropy
// 4096 bf16 rows of 4096 -> 65536: 1,600 to 1,620 us a call in a row of them, 22 and 14 of it before and after the product, 1.4 PFLOP/s, bound by the power cap (as the
// gradient's products).
// Few rows (streams()) have the projection streamed past them, 16 in the registers of a wavefront, bound by its bytes.
#include "linear_epilogues.h"

#include <type_traits>

namespace pcm {
namespace {

typedef u32x4 __attribute__((aligned(2))) u32x4_any;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;

// ---- slots ---------------------------------------------------------------------------------------

__device__ inline int token_at(const LinearRows& in, int row) {          // -1: none
    int64_t t;
    if (in.token_type == PCM_TOKEN_U8) t = static_cast<const uint8_t*>(in.tokens)[row];
    else if (in.token_type == PCM_TOKEN_I32) t = static_cast<const int32_t*>(in.tokens)[row];
    else t = static_cast<const int64_t*>(in.tokens)[row];
    return t < 0 ? -1 : t >= in.V ? in.V - 1 : (int)t;
}

__device__ inline int block_count(int x) {                               // over 256 threads, in every thread
    __shared__ int lds[4];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

__global__ __launch_bounds__(256) void linear_counts(LinearRows in, int32_t* counts) {
    int n = 0;
    for (int i = threadIdx.x; i < kCountRows; i += 256) {
        const int row = blockIdx.x * kCountRows + i;
        n += row < in.rows && token_at(in, row) >= 0;
    }
    n = block_count(n);
    if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

constexpr int kNoExponent = -(1 << 20), kNoGradient = 1 << 21;
// Long lists: 1024 rows a workgroup, four neighbours a thread; where its rows begin among the slots it adds up from the counts of the launch before.
__global__ __launch_bounds__(256) void linear_slots(LinearRows in, Slots slots) {
    int before = 0;
    for (int b = threadIdx.x; b < (int)blockIdx.x; b += 256) before += slots.counts[b];
    before = block_count(before);
    const int first = blockIdx.x * kCountRows + threadIdx.x * 4;
    int token[4], mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        token[e] = first + e < in.rows ? token_at(in, first + e) : -1;
        mine += token[e] >= 0;
    }
    int upto = mine;                                                     // inclusive over the wavefront
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int x = __shfl_up(upto, off, 64);
        if ((int)(threadIdx.x & 63) >= off) upto += x;
    }
    __shared__ int wave_total[4];
    if ((threadIdx.x & 63) == 63) wave_total[threadIdx.x >> 6] = upto;
    __syncthreads();
    int slot = before + upto - mine;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) slot += wave_total[w];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (first + e < in.rows) slots.slot_of[first + e] = token[e] >= 0 ? slot : -1;
        if (token[e] >= 0) {
            slots.row_of[slot] = first + e;
            slots.token[slot++] = token[e];
        }
    }
    if (blockIdx.x != gridDim.x - 1) return;
    if (threadIdx.x == 255) *slots.live = slot;
    if (threadIdx.x < kMosts) slots.mosts[threadIdx.x * kMostPitch] = kNoExponent;
}

// Exponent e with 2^e <= x < 2^(e + 1); x > 0 and finite.
__device__ inline int exponent_of(float x) { return ilogbf(x); }
__device__ inline float finite_abs(float x) {
    x = fabsf(x);
    return x < __builtin_huge_valf() ? x : 0.f;       // not for infinities and NaN
}
__device__ inline float wave_max(float x) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
    return x;
}
__device__ inline float block_max(float x) {          // over 256 threads, in every thread
    __shared__ float lds[4];
    x = wave_max(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return fmaxf(fmaxf(lds[0], lds[1]), fmaxf(lds[2], lds[3]));
}
// The power of two that brings values below 2^(exponent + 1) below 2^15.
__device__ inline int shift_for(int exponent) { return min(126, max(-126, 14 - exponent)); }
__device__ inline half_bits high_part(float x) { return __builtin_bit_cast(half_bits, (f16)x); }
__device__ inline half_bits low_part(float x) { return __builtin_bit_cast(half_bits, (f16)(x - (float)(f16)x)); }

// 16 bytes at any address of their type; zeros behind the first n values.
__device__ inline u32x4 load_16B(const half_bits* p, int n) {
    if (n >= 8) return *reinterpret_cast<const u32x4_any*>(p);
    u32x4 x = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n) x[e / 2] |= (uint32_t)p[e] << (e % 2 * 16);
    return x;
}
__device__ inline f32x4 load_4(const float* p, int n) {
    if (n >= 4) return *reinterpret_cast<const f32x4_any*>(p);
    f32x4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < n) x[e] = p[e];
    return x;
}
__device__ inline u32x4 load_16B(const float* p, int n) { return __builtin_bit_cast(u32x4, load_4(p, n)); }

// Eight fp32 values times a power of two as pairs.
template <class F>
__device__ inline void store_pairs(half_bits* hi, half_bits* lo, F value) {
    u32x4 h = {0, 0, 0, 0}, l = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = value(e);
        h[e / 2] |= (uint32_t)high_part(x) << (e % 2 * 16);
        l[e / 2] |= (uint32_t)low_part(x) << (e % 2 * 16);
    }
    *reinterpret_cast<u32x4*>(hi) = h;
    *reinterpret_cast<u32x4*>(lo) = l;
}
// A row of d values times 2^shift as pairs, zeros up to d64, by a wavefront.
__device__ inline void pair_row(const float* from, int d, int shift, half_bits* hi, half_bits* lo, int d64, int lane) {
    for (int i = lane * 8; i < d64; i += 512) {
        const f32x4 a = load_4(from + i, d - i), b = load_4(from + i + 4, d - i - 4);
        store_pairs(hi + i, lo + i, [&](int e) { return ldexpf(e < 4 ? a[e] : b[e - 4], shift); });
    }
}
__device__ inline void zero_row(half_bits* to, int d64, int lane) {
    for (int i = lane * 8; i < d64; i += 512) *reinterpret_cast<u32x4*>(to + i) = u32x4{0, 0, 0, 0};
}

// A wavefront per row: bf16 rows are copied, fp32 rows become pairs.  256 more take the slots behind the last one.
// kList: the launch that lists the slots is part of this one, each workgroup counting the tokens before its rows (short lists; 256 rows of 256 bf16 take
// 5 us so instead of 8 in two launches).
constexpr int kGatherRows = 4;                        // per workgroup
template <class T, bool kList>
__device__ __forceinline__ void gather_rows(const LinearRows& in, const Slots& slots, const SlotGradients& grads, int block) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int first = block * kGatherRows, row = first + wave;
    int before = 0, token = -1;
    if (kList) {
        for (int i = threadIdx.x; i < min(first, in.rows); i += 256) before += token_at(in, i) >= 0;
        before = block_count(before);
        for (int w = 0; w < kGatherRows; ++w) {
            const int t = first + w < in.rows ? token_at(in, first + w) : -1;
            if (w == wave) token = t;
            if (w < wave) before += t >= 0;
        }
    }
    if (row >= in.rows) {
        // (a workgroup on the border has counted the rows before its own, so `before` is all of them)
        const int live = kList ? before : *slots.live, slot = live + row - in.rows;
        if (kList && row == in.rows && lane == 0) *slots.live = live;
        if (slot >= min(slots.padded, (live + 255) / 256 * 256)) return;
        zero_row(slots.h + (int64_t)slot * slots.d64, slots.d64, lane);
        if (sizeof(T) == 4) zero_row(slots.h_low + (int64_t)slot * slots.d64, slots.d64, lane);
        if (lane == 0) {
            slots.token[slot] = -1;
            if (sizeof(T) == 4) slots.h_unit[slot] = 0.f;      // (1 times the weight's over a low temperature may be infinite, and 0 times that no number)
            if (grads.of != nullptr) grads.of[slot] = SlotGradient{0.f, 0.f, 0.f, 0.f};
            if (sizeof(T) == 4 && grads.of != nullptr) grads.z_shift[slot] = 0;
        }
        return;
    }
    int slot;
    if (kList) {
        slot = token >= 0 ? before : -1;
        if (lane == 0) {
            slots.slot_of[row] = slot;
            if (slot >= 0) {
                slots.token[slot] = token;
                slots.row_of[slot] = row;
            }
        }
    } else {
        slot = slots.slot_of[row];
    }
    if (slot < 0) {
        if (grads.dh == nullptr) return;
        T* const dh = static_cast<T*>(grads.dh) + row * grads.dh_ld;
        for (int i = lane; i < in.d; i += 64) dh[i] = 0;
        return;
    }
    const T* const from = static_cast<const T*>(in.hidden) + row * in.ld;
    const int64_t to = (int64_t)slot * slots.d64;
    float largest = 0.f;
    if constexpr (sizeof(T) == 2) {
        for (int i = lane * 8; i < slots.d64; i += 512) *reinterpret_cast<u32x4*>(slots.h + to + i) = load_16B(from + i, in.d - i);
    } else {
        for (int i = lane * 4; i < in.d; i += 256) {
            const f32x4 x = load_4(from + i, in.d - i);
            largest = fmaxf(fmaxf(largest, fmaxf(finite_abs(x[0]), finite_abs(x[1]))), fmaxf(finite_abs(x[2]), finite_abs(x[3])));
        }
        largest = wave_max(largest);
        const int shift = largest > 0.f ? shift_for(exponent_of(largest)) : 0;
        pair_row(from, in.d, shift, slots.h + to, slots.h_low + to, slots.d64, lane);
        if (lane == 0) slots.h_unit[slot] = ldexpf(1.f, -shift);
    }
    if (grads.of == nullptr || lane != 0) return;
    SlotGradient of;
    of.g = grads.dlogp[row] * grads.inv_t;
    of.h = grads.dentropy != nullptr ? grads.dentropy[row] * grads.inv_t : 0.f;
    of.lse2 = grads.lse[row] * kLog2E;
    of.entropy = grads.dentropy != nullptr ? grads.entropy[row] : 0.f;
    if constexpr (sizeof(T) == 4) {
        // |p (log p + entropy)| is at most the larger of 1 / e and the entropy
        const float bound = fabsf(of.g) + fabsf(of.h) * (0.5f + fabsf(of.entropy));
        // (a row that no gradient reaches is not weighted by the others' power of two, which may be far too large for it)
        const int shift = bound == 0.f ? kNoGradient : bound < __builtin_huge_valf() ? shift_for(exponent_of(bound)) : 0;
        of.g = ldexpf(of.g, shift);
        of.h = ldexpf(of.h, shift);
        grads.z_shift[slot] = shift;
        const int exponent = bound > 0.f && largest > 0.f ? exponent_of(largest) - shift : kNoExponent;
        if (kList) grads.exponent[slot] = exponent;
        else {                                            // (the largest of whole numbers: their order does not matter)
            int32_t* const most = slots.mosts + block % kMosts * kMostPitch;
            if (exponent > __hip_atomic_load(most, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)) atomicMax(most, exponent);
        }
    }
    grads.of[slot] = of;
}

// h 2^(14 - most - z_shift) as pairs: dz 2^z_shift times it adds up over rows of any sizes.
__device__ __forceinline__ void weigh_rows(const LinearRows& in, const Slots& slots, const SlotGradients& grads, int block) {
    const int lane = threadIdx.x & 63, row = block * kGatherRows + (int)(threadIdx.x >> 6);
    const int live = *slots.live;
    // (a short list: each workgroup looks for the largest exponent itself)
    const bool shares = slots.counts != nullptr;
    float x = (float)kNoExponent;
    for (int i = threadIdx.x; i < (shares ? kMosts : live); i += 256) x = fmaxf(x, (float)(shares ? slots.mosts[i * kMostPitch] : grads.exponent[i]));
    const int most = (int)block_max(x);
    if (block == 0 && threadIdx.x == 0) *slots.most = most;
    if (row >= in.rows) {
        const int slot = live + row - in.rows;
        if (slot >= min(slots.padded, (live + 255) / 256 * 256)) return;
        zero_row(grads.w_h + (int64_t)slot * slots.d64, slots.d64, lane);
        zero_row(grads.w_h_low + (int64_t)slot * slots.d64, slots.d64, lane);
        return;
    }
    const int slot = slots.slot_of[row];
    if (slot < 0) return;
    const int64_t to = (int64_t)slot * slots.d64;
    pair_row(static_cast<const float*>(in.hidden) + row * in.ld, in.d, max(-300, 14 - most - grads.z_shift[slot]), grads.w_h + to, grads.w_h_low + to,
             slots.d64, lane);
}

// ---- weights that have to be copied ----------------------------------------------------------------

__device__ __forceinline__ void absmax_part(const WeightAbsmax& q, int block) {
    const int lanes = q.split.lanes, chunks = q.split.chunks;
    float most = 0.f;
    for (int at = block; at < q.split.blocks; at += q.parts) {
        const int row = (at / chunks << (8 - lanes)) + (int)(threadIdx.x >> lanes);
        const int64_t i = (((int64_t)(at % chunks) << (lanes + 2)) + (threadIdx.x & ((1 << lanes) - 1))) * 4;       // four loads, 4 << lanes apart
        if (row >= q.rows) continue;
        f32x4 x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t c = i + ((int64_t)e << (lanes + 2));
            x[e] = c < q.cols ? load_4(q.w + row * q.ld + c, (int)(q.cols - c)) : f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            most = fmaxf(fmaxf(most, fmaxf(finite_abs(x[e][0]), finite_abs(x[e][1]))), fmaxf(finite_abs(x[e][2]), finite_abs(x[e][3])));
    }
    most = block_max(most);
    if (threadIdx.x == 0) q.out[block] = most;
}
template <class T>
__device__ __forceinline__ void copy_piece(const WeightPiece& q, int block) {
    float scale = 1.f;
    if constexpr (sizeof(T) == 4) {
        float most = 0.f;
        for (int i = threadIdx.x; i < q.absmax_parts; i += 256) most = fmaxf(most, q.absmax[i]);
        most = block_max(most);
        const int shift = most > 0.f ? shift_for(exponent_of(most)) : 0;
        scale = ldexpf(1.f, shift);
        if (block == 0 && threadIdx.x == 0) *q.unit = ldexpf(1.f, -shift);
    }
    const int lanes = q.split.lanes, row = (block / q.split.chunks << (8 - lanes)) + (int)(threadIdx.x >> lanes);
    const int64_t i = (((int64_t)(block % q.split.chunks) << lanes) + (threadIdx.x & ((1 << lanes) - 1))) * 8;
    if (row >= q.rows || i >= q.ld_to) return;
    const T* const from = static_cast<const T*>(q.w) + row * q.ld + i;
    const int n = (int)(q.cols - i);
    half_bits* const out = q.to + row * q.ld_to + i;
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<u32x4*>(out) = load_16B(from, n);
    } else {
        const f32x4 a = load_4(from, n), b = load_4(from + 4, n - 4);
        store_pairs(out, q.low + row * q.ld_to + i, [&](int e) { return (e < 4 ? a[e] : b[e - 4]) * scale; });
    }
}

// ---- before the products: two launches at most, of work that does not wait for one another ------------------

// Rows to slots, and beside it the largest value of an fp32 weight or the first piece of a bf16 one.  4096 bf16 rows of 4096 22 us; 1111 fp32 rows of 1001 and
// a weight of 1001 x 32003 37, and 47 in the second launch, 4.6 TB/s together.
template <class T, bool kList>
__global__ __launch_bounds__(256) void linear_gather(LinearRows in, Slots slots, SlotGradients grads, int rows_blocks, WeightAbsmax absmax, WeightPiece piece) {
    const int block = blockIdx.x;
    if (block < rows_blocks) return gather_rows<T, kList>(in, slots, grads, block);
    if constexpr (sizeof(T) == 4) absmax_part(absmax, block - rows_blocks);
    else copy_piece<T>(piece, block - rows_blocks);
}
// fp32: rows weighted for dW, and the first piece of the weight.
__global__ __launch_bounds__(256) void linear_weigh(LinearRows in, Slots slots, SlotGradients grads, int rows_blocks, WeightPiece piece) {
    const int block = blockIdx.x;
    if (block < rows_blocks) return weigh_rows(in, slots, grads, block);
    copy_piece<float>(piece, block - rows_blocks);
}
template <class T>
__global__ __launch_bounds__(256) void linear_copy(WeightPiece piece) {
    copy_piece<T>(piece, blockIdx.x);
}

// ---- joining the parts -------------------------------------------------------------------------------

// Results of a row from its parts: kRows rows a workgroup, the other threads parts of them (one row of 2,048 parts 5.5 us, 4096 of 512 15).
template <int kRows>
__global__ __launch_bounds__(256) void linear_join(LinearRows in, const int32_t* slot_of, PartSums parts, const float* token_z, float inv_t,
                                                   RowResults out) {
    constexpr int kParts = 256 / kRows;
    __shared__ RowSums lds[kParts][kRows];
    const int r = threadIdx.x % kRows, k = threadIdx.x / kRows;
    const int row = blockIdx.x * kRows + r;
    const float c = inv_t * kLog2E;
    int slot = -1;
    if (row < in.rows) slot = slot_of != nullptr ? slot_of[row] : token_at(in, row) >= 0 ? row : -1;
    RowSums a = {0.f, 0.f, 0.f};
    if (slot >= 0) {
#pragma unroll 4
        for (int p = k; p < parts.parts; p += kParts) {
            const f32x4 b = parts.of[p * parts.ld + slot];
            merge(a, RowSums{b[0], b[1], b[2]}, c);
        }
    }
    lds[k][r] = a;
#pragma unroll
    for (int step = kParts / 2; step > 0; step >>= 1) {
        __syncthreads();
        if (k < step) {
            merge(a, lds[k + step][r], c);
            lds[k][r] = a;
        }
    }
    if (k != 0 || row >= in.rows) return;
    float logp = 0.f, lse = 0.f, entropy = 0.f;
    if (slot >= 0) {
        const float log_s = logf(a.s);
        lse = __builtin_fmaf(a.m, inv_t, log_s);
        logp = (token_z[slot] - a.m) * inv_t - log_s;
        entropy = log_s - kLn2 * (a.t / a.s);
        if (!(a.s < __builtin_huge_valf())) lse = logp = entropy = __builtin_nanf("");
    }
    out.logp[row] = logp;
    out.lse[row] = lse;
    if (out.entropy != nullptr) out.entropy[row] = entropy;
}

// ---- few rows --------------------------------------------------------------------------------------

// The 16 bytes of a row of d values that begin at value k, zeros behind its end; the row is that long at least, and nothing outside it is read.
template <class T>
__device__ __forceinline__ u32x4 load_tail(const T* row, int k, int d) {
    constexpr int kE = 16 / sizeof(T);
    const int from = min(k, d - kE), drop = (k - from) * (int)sizeof(T) * 8;        // bits that belong before k
    const u32x4 x = load_16B(row + from, kE);
    const uint64_t lo = (uint64_t)x[1] << 32 | x[0], hi = (uint64_t)x[3] << 32 | x[2];
    const uint64_t l = drop == 0 ? lo : drop < 64 ? lo >> drop | hi << (64 - drop) : drop < 128 ? hi >> (drop - 64) : 0;
    const uint64_t h = drop < 64 ? hi >> drop : 0;
    return u32x4{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
}

// z of up to 16 rows and a block of the vocabulary.  The four wavefronts of a workgroup take every fourth slice of the reduction index, their sums
// are added in LDS.  A slice is 4 lane groups x kE values of k (kE = 16 bytes of them).
//   [V][d]: a lane brings in kE values of k of one column and is its fragment; four fragments of 16 columns share one of the hidden rows.
//   [d][V]: a lane brings in kE columns at kE values of k and has the fragments of kE columns, bf16 after exchanging halves between pairs of rows.
// An XCD has neighbouring blocks: the lines that two of them share, where rows do not begin on a line, come out of its cache (7 fp32 rows of 1024 -> 32003 33.6 ->
// 26.6 us with what follows; one bf16 row of 4096 -> 131072 204 -> 195).  More than 16 rows are groups of 16 whose workgroups follow one another on an XCD, so
// that the projection comes from there after the first.
template <class T, int kLayout>
__global__ __launch_bounds__(256) void few_rows(LinearRows in, const T* w, int64_t ld, PartSums out, float* token_z, float c, int groups) {
    constexpr int kE = 16 / sizeof(T), kSlice = 4 * kE;
    constexpr int kTiles = kLayout == PCM_WEIGHT_OUT_IN ? 4 : kE, kLoads = kLayout == PCM_WEIGHT_OUT_IN ? 4 : kE;
    constexpr int kColumns = kTiles * 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane >> 4, at = lane & 15;
    const int each = (out.parts + kNumXcd - 1) / kNumXcd;              // blocks of an XCD
    const int block = blockIdx.x % kNumXcd * each + blockIdx.x / (kNumXcd * groups), row0 = blockIdx.x / kNumXcd % groups * kFewRows;
    const int n0 = block * kColumns;
    if (n0 >= in.V) return;
    f32x4 acc[kTiles];
#pragma unroll
    for (int j = 0; j < kTiles; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // (lanes of rows that are not there take the last one's values along)
    const T* const h_row = static_cast<const T*>(in.hidden) + min(row0 + at, in.rows - 1) * in.ld;
    const bool has_row = row0 + at < in.rows;
    // [d][V]: where the vocabulary ends lanes move back to its last kE columns and count those that are their own.
    const bool moves = kLayout == PCM_WEIGHT_IN_OUT && in.V >= kE;
    auto first_column = [&](int lane_of_16) { return moves ? min(n0 + lane_of_16 * kE, in.V - kE) : n0 + lane_of_16 * kE; };
    struct Slice {
        u32x4 w[kLoads], h;
    };
    // whole slices of k (rows of [V][d] behind the last one are the last one again)
    auto load = [&](Slice& x, int k0) __attribute__((always_inline)) {
        const int k = k0 + group * kE;
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            x.w[q] = load_16B(kLayout == PCM_WEIGHT_OUT_IN ? w + min(n0 + q * 16 + at, in.V - 1) * ld + k : w + (k + q) * ld + first_column(at), kE);
        x.h = load_16B(h_row + k, kE);
    };
    // the slice in which k ends: rows that are shorter than 16 bytes are read value by value
    const bool shifts = in.d >= kE && (kLayout == PCM_WEIGHT_OUT_IN || moves);
    auto load_edge = [&](Slice& x, int k0) __attribute__((always_inline)) {
        const int k = k0 + group * kE;
        if (shifts) {
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                if (kLayout == PCM_WEIGHT_OUT_IN) x.w[q] = load_tail(w + min(n0 + q * 16 + at, in.V - 1) * ld, k, in.d);
                else {
                    x.w[q] = load_16B(w + min(k + q, in.d - 1) * ld + first_column(at), kE);
                    if (k + q >= in.d) x.w[q] = u32x4{0, 0, 0, 0};
                }
            }
            x.h = load_tail(h_row, k, in.d);
            return;
        }
#pragma unroll
        for (int q = 0; q < kLoads; ++q) {
            const int v = kLayout == PCM_WEIGHT_OUT_IN ? n0 + q * 16 + at : first_column(at), row = kLayout == PCM_WEIGHT_OUT_IN ? k : k + q;
            x.w[q] = u32x4{0, 0, 0, 0};
            if (v < in.V && row < in.d) x.w[q] = kLayout == PCM_WEIGHT_OUT_IN ? load_16B(w + v * ld + k, in.d - k) : load_16B(w + row * ld + v, in.V - v);
        }
        x.h = u32x4{0, 0, 0, 0};
        if (k < in.d) x.h = load_16B(h_row + k, in.d - k);
    };
    auto multiply = [&](const Slice& x) __attribute__((always_inline)) {
        if constexpr (sizeof(T) == 2) {
            const bf16x8 hf = __builtin_bit_cast(bf16x8, x.h);
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
                u32x4 f;
                if constexpr (kLayout == PCM_WEIGHT_OUT_IN) f = x.w[j];
                else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)                  // column j of rows 2 q and 2 q + 1
                        f[q] = __builtin_amdgcn_perm(x.w[2 * q + 1][j / 2], x.w[2 * q][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
                }
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, f), hf, acc[j], 0, 0, 0);
            }
        } else {
            const f32x4 hf = __builtin_bit_cast(f32x4, x.h);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < kTiles; ++j) {
                    const f32x4 f = __builtin_bit_cast(f32x4, x.w[kLayout == PCM_WEIGHT_OUT_IN ? j : e]);
                    acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[kLayout == PCM_WEIGHT_OUT_IN ? e : j], hf[e], acc[j], 0, 0, 0);
                }
        }
    };
    // Whole slices: kAhead are under way while one is multiplied (past the end the last one again).
    constexpr int kAhead = kLoads > 4 ? 2 : 4, kStride = 4 * kSlice;
    int done = 0;
    if ((kLayout == PCM_WEIGHT_OUT_IN || moves) && wave * kSlice + kSlice <= in.d) {
        const int n = (in.d - kSlice - wave * kSlice) / kStride + 1;
        Slice x[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load(x[i], wave * kSlice + min(i, n - 1) * kStride);
        for (; done < n; done += kAhead)
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (done + i < n) multiply(x[i]);
                load(x[i], wave * kSlice + min(done + i + kAhead, n - 1) * kStride);
            }
        done = n;
    }
    for (int k0 = wave * kSlice + done * kStride; k0 < in.d; k0 += kStride) {
        Slice x;
        load_edge(x, k0);
        multiply(x);
    }
    __shared__ f32x4 sums[4][kTiles][64];
#pragma unroll
    for (int j = 0; j < kTiles; ++j) sums[wave][j][lane] = acc[j];
    __syncthreads();
    // a lane has row `at` and, of tile j, columns 4 group + t of 16
    constexpr int kMine = kTiles / 4;
    const int token = has_row ? token_at(in, row0 + at) : -1;
    float z[kMine][4], m = -__builtin_huge_valf();
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int j = wave * kMine + i;
        const f32x4 total = (sums[0][j][lane] + sums[1][j][lane]) + (sums[2][j][lane] + sums[3][j][lane]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int column = group * 4 + t, v = kLayout == PCM_WEIGHT_OUT_IN ? n0 + j * 16 + column : first_column(column) + j;
            const bool own = v < in.V && (kLayout == PCM_WEIGHT_OUT_IN || v >= n0 + column * kE);
            z[i][t] = own ? total[t] : -__builtin_huge_valf();
            m = fmaxf(m, z[i][t]);
            if (own && v == token) token_z[row0 + at] = z[i][t];
        }
    }
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
    RowSums r{m, 0.f, 0.f};
    if (m > -__builtin_huge_valf()) {
        r = sums_of<kMine>(m, c, [&](int i, int e) __attribute__((always_inline)) { return z[i][e]; });
    } else {
#pragma unroll
        for (int i = 0; i < kMine; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) r.s += z[i][e] == -__builtin_huge_valf() ? 0.f : z[i][e];       // nothing, or NaN
    }
    r.s += __shfl_xor(r.s, 16, 64);
    r.s += __shfl_xor(r.s, 32, 64);
    r.t += __shfl_xor(r.t, 16, 64);
    r.t += __shfl_xor(r.t, 32, 64);
    __shared__ RowSums part[4][16];
    if (group == 0) part[wave][at] = r;
    __syncthreads();
    if (threadIdx.x >= 16 || !has_row) return;
    RowSums a = part[0][at];
    for (int q = 1; q < 4; ++q) merge(a, part[q][at], c);
    out.of[block * out.ld + row0 + at] = f32x4{a.m, a.s, a.t, 0.f};
}

int few_columns(int dtype, int layout) { return layout == PCM_WEIGHT_OUT_IN || dtype == PCM_F32 ? 64 : 128; }
template <class T>
void launch_few(const LinearRows& in, const void* w, int64_t ld, int layout, const PartSums& parts, float* token_z, float c, hipStream_t s) {
    const T* const p = static_cast<const T*>(w);
    const int groups = ceil_div(in.rows, kFewRows);
    const unsigned grid = (unsigned)(round_up(parts.parts, kNumXcd) * groups);
    if (layout == PCM_WEIGHT_OUT_IN) few_rows<T, PCM_WEIGHT_OUT_IN><<<grid, 256, 0, s>>>(in, p, ld, parts, token_z, c, groups);
    else few_rows<T, PCM_WEIGHT_IN_OUT><<<grid, 256, 0, s>>>(in, p, ld, parts, token_z, c, groups);
}

// ---- the forward call --------------------------------------------------------------------------------

PartSums carve_parts(Carver& c, int64_t ld, int parts) {
    PartSums p{};
    p.ld = ld;
    p.parts = parts;
    p.of = c.take<f32x4>((size_t)(ld * parts));
    return p;
}
struct ForwardPlan {
    bool few;
    int tile, columns;               // of the products: kW, columns of a piece
    Slots slots;
    WeightCopy copy;
    PartSums parts;
    float* token_z;
    size_t bytes;
};
ForwardPlan plan_forward(void* workspace, int rows, const WeightSource& src) {
    Carver c(workspace);
    ForwardPlan f{};
    f.few = streams(rows, src);
    if (f.few) {
        f.parts = carve_parts(c, rows, ceil_div(src.V, few_columns(src.dtype, src.layout)));
        f.token_z = c.take<float>((size_t)rows);
    } else {
        f.slots = carve_slots(c, rows, src.d, src.dtype);
        f.columns = src.in_place ? src.V : copy_columns(src);
        // (a launch has fewer than 2^32 threads: 2^22 small tiles leave room)
        f.columns = (int)std::min<int64_t>(f.columns, std::max<int64_t>(kTileN, ((int64_t)1 << 36) / f.slots.padded / kTileN * kTileN));
        f.copy = carve_weight(c, src, f.columns);
        f.tile = rows <= 128 ? kSmallTile : tile_for(f.slots.padded, round_up(std::min(f.columns, src.V), kTileN), 1);
        // (pieces are multiples of 256 columns, so only the last one ends inside a wavefront's block)
        f.parts = carve_parts(c, f.slots.padded, ceil_div(src.V, 16 * f.tile));
        f.token_z = c.take<float>((size_t)f.slots.padded);
    }
    f.bytes = c.used();
    return f;
}

template <bool kThirds>
void forward_products(const ForwardPlan& f, const WeightSource& src, int rows, float c, hipStream_t s) {
    for (int first = 0; first < src.V; first += f.columns) {
        const int columns = std::min(f.columns, src.V - first);
        const WeightOperand w = weight_operand(src, f.copy, first, columns, s);
        BoundedProblem<kThirds> p = slot_product<kThirds>(f.slots, kRowsAreM);
        p.M = rows <= 128 ? 128 : f.slots.padded;
        set_a(p, f.slots.h, f.slots.h_low, f.slots.d64);
        const EpiRowStats epi{f.parts, f.token_z, f.slots.token, kThirds ? f.slots.h_unit : nullptr, kThirds ? f.copy.unit : nullptr, c, first,
                              columns, first / (16 * f.tile)};
        if (src.layout == PCM_WEIGHT_OUT_IN) {
            set_b<kRowsByK>(p, w.w, w.low, w.ld, columns, src.d);
            SlotProduct<kThirds, kRowsByK, kRowsByK, EpiRowStats>(p, f.tile, epi).launch(s);
        } else {
            set_b<kKByRows>(p, w.w, w.low, w.ld, columns, src.d);
            SlotProduct<kThirds, kRowsByK, kKByRows, EpiRowStats>(p, f.tile, epi).launch(s);
        }
    }
}

}  // namespace

// ---- shared ------------------------------------------------------------------------------------------

Slots carve_slots(Carver& c, int rows, int d, int dtype) {
    Slots q{};
    q.padded = round_up(rows, kTileM);
    q.d64 = round_up(d, kTileK);
    q.live = c.take<int32_t>(1);
    q.parts = c.take<int32_t>(1);
    q.most = c.take<int32_t>(1);
    q.slot_of = c.take<int32_t>((size_t)rows);
    q.row_of = c.take<int32_t>((size_t)q.padded);
    q.token = c.take<int32_t>((size_t)q.padded);
    // (a tile of the product over rows reads up to 255 columns past a row)
    const size_t h = (size_t)q.padded * q.d64 + kTileM;
    q.h = c.take<half_bits>(h);
    if (dtype == PCM_F32) {
        q.h_low = c.take<half_bits>(h);
        q.h_unit = c.take<float>((size_t)q.padded);
    }
    if (rows > 4 * kCountRows) {
        q.counts = c.take<int32_t>((size_t)ceil_div(rows, kCountRows));
        q.mosts = c.take<int32_t>(kMosts * kMostPitch);
    }
    return q;
}
SlotGradients carve_gradients(Carver& c, const Slots& slots, int dtype) {
    SlotGradients g{};
    g.of = c.take<SlotGradient>((size_t)slots.padded);
    if (dtype == PCM_F32) {
        const size_t h = (size_t)slots.padded * slots.d64 + kTileM;
        g.z_shift = c.take<int32_t>((size_t)slots.padded);
        g.exponent = c.take<int32_t>((size_t)slots.padded);
        g.w_h = c.take<half_bits>(h);
        g.w_h_low = c.take<half_bits>(h);
    }
    return g;
}
WeightSource weight_source(const void* w, int64_t ld, int dtype, int layout, int d, int V, bool sums_along_rows) {
    const int length = layout == PCM_WEIGHT_OUT_IN ? d : V;
    // 256 rows of a tile are addressed with 32 bits
    const bool reads = dtype == PCM_BF16 && (reinterpret_cast<uintptr_t>(w) & 15u) == 0 && ld % 8 == 0 && length % 8 == 0 && ld < (1 << 23);
    // A sum along a row goes on to the next multiple of 64 with zeros times what is there: the next row, whose NaN all results have anyway, or a
    // gap, whose none may have
    return WeightSource{w, ld, dtype, layout, d, V, reads && (!sums_along_rows || ld == length || length % kTileK == 0)};
}
// Pieces of at most 256 MB, in whole tiles.
int copy_columns(const WeightSource& src) {
    const int64_t most = (int64_t)(256 << 20) / (round_up(src.d, kTileM) * (src.dtype == PCM_F32 ? 4 : 2)) / kTileN * kTileN;
    return (int)std::min<int64_t>(std::max<int64_t>(most, kTileN), round_up(src.V, kTileN));
}
WeightCopy carve_weight(Carver& c, const WeightSource& src, int columns) {
    WeightCopy q{};
    if (src.in_place) return q;
    q.columns = round_up(columns, kTileN);
    const int rows = src.layout == PCM_WEIGHT_OUT_IN ? q.columns : round_up(src.d, kTileM);
    q.ld = src.layout == PCM_WEIGHT_OUT_IN ? round_up(src.d, kTileK) : q.columns;
    q.w = c.take<half_bits>((size_t)rows * q.ld);
    if (src.dtype == PCM_F32) {
        q.low = c.take<half_bits>((size_t)rows * q.ld);
        const int rows_all = src.layout == PCM_WEIGHT_OUT_IN ? src.V : src.d, cols = src.layout == PCM_WEIGHT_OUT_IN ? src.d : src.V;
        q.absmax_parts = std::min(kAbsmaxParts, RowSplit(rows_all, ceil_div(cols, 4), 4).blocks);
        q.absmax = c.take<float>(kAbsmaxParts);
        q.unit = c.take<float>(1);
    }
    return q;
}
static WeightPiece piece_of(const WeightSource& src, const WeightCopy& copy, int first, int columns) {
    const bool by_token = src.layout == PCM_WEIGHT_OUT_IN;
    const int64_t at = by_token ? first * src.ld : first;
    const int rows = by_token ? columns : src.d;
    const void* const w = static_cast<const char*>(src.w) + at * (src.dtype == PCM_F32 ? 4 : 2);
    return WeightPiece{w, src.ld, rows, by_token ? src.d : columns, copy.w, copy.low, copy.ld, RowSplit(rows, copy.ld, 8), copy.absmax, copy.absmax_parts, copy.unit};
}
void prepare_operands(const LinearRows& in, const Slots& slots, const SlotGradients* grads, const WeightSource& src, const WeightCopy& copy, int columns,
                      hipStream_t s) {
    const int rows_blocks = ceil_div(in.rows + kTileM, kGatherRows);
    const SlotGradients g = grads != nullptr ? *grads : SlotGradients{};
    const bool own_list = slots.counts == nullptr;
    if (!own_list) {
        const unsigned lists = (unsigned)ceil_div(in.rows, kCountRows);
        linear_counts<<<lists, 256, 0, s>>>(in, slots.counts);
        linear_slots<<<lists, 256, 0, s>>>(in, slots);
    }
    const WeightPiece piece = src.in_place ? WeightPiece{} : piece_of(src, copy, 0, std::min(columns, src.V));
    if (src.dtype == PCM_F32) {
        const int rows = src.layout == PCM_WEIGHT_OUT_IN ? src.V : src.d, cols = src.layout == PCM_WEIGHT_OUT_IN ? src.d : src.V;
        const WeightAbsmax absmax{static_cast<const float*>(src.w), src.ld, rows, cols, copy.absmax_parts, RowSplit(rows, ceil_div(cols, 4), 4), copy.absmax};
        if (own_list) linear_gather<float, true><<<rows_blocks + absmax.parts, 256, 0, s>>>(in, slots, g, rows_blocks, absmax, piece);
        else linear_gather<float, false><<<rows_blocks + absmax.parts, 256, 0, s>>>(in, slots, g, rows_blocks, absmax, piece);
        if (g.w_h != nullptr) linear_weigh<<<rows_blocks + piece.split.blocks, 256, 0, s>>>(in, slots, g, rows_blocks, piece);
        else linear_copy<float><<<piece.split.blocks, 256, 0, s>>>(piece);
    } else {
        if (own_list) linear_gather<half_bits, true><<<rows_blocks + piece.split.blocks, 256, 0, s>>>(in, slots, g, rows_blocks, WeightAbsmax{}, piece);
        else linear_gather<half_bits, false><<<rows_blocks + piece.split.blocks, 256, 0, s>>>(in, slots, g, rows_blocks, WeightAbsmax{}, piece);
    }
}
WeightOperand weight_operand(const WeightSource& src, const WeightCopy& copy, int first, int columns, hipStream_t s) {
    if (src.in_place) return WeightOperand{static_cast<const half_bits*>(src.w) + (src.layout == PCM_WEIGHT_OUT_IN ? first * src.ld : first), nullptr, src.ld};
    if (first > 0) {
        const WeightPiece piece = piece_of(src, copy, first, columns);
        if (src.dtype == PCM_F32) linear_copy<float><<<piece.split.blocks, 256, 0, s>>>(piece);
        else linear_copy<half_bits><<<piece.split.blocks, 256, 0, s>>>(piece);
    }
    return WeightOperand{copy.w, copy.low, copy.ld};
}

int check_linear(const void* hidden, int64_t hidden_ld, const void* weight, int64_t weight_ld, int layout, int dtype, const void* tokens,
                 int token_type, int64_t rows, int d, int V, float temperature) {
    if (rows < 0 || d < 1 || V < 1 || hidden_ld < d || (layout != PCM_WEIGHT_IN_OUT && layout != PCM_WEIGHT_OUT_IN) ||
        weight_ld < (layout == PCM_WEIGHT_OUT_IN ? d : V) || (dtype != PCM_F32 && dtype != PCM_BF16) ||
        (token_type != PCM_TOKEN_U8 && token_type != PCM_TOKEN_I32 && token_type != PCM_TOKEN_I64) || !(temperature >= 0x1p-126f) ||
        temperature == __builtin_huge_valf())
        return PCM_EINVAL;
    const int rc = rows > (1 << 24) || d > (1 << 16) || V > (1 << 22) ? PCM_EUNSUPPORTED : PCM_OK;
    if (rows == 0) return rc;
    const uintptr_t value = dtype == PCM_F32 ? 3 : 1, token = token_type == PCM_TOKEN_U8 ? 0 : token_type == PCM_TOKEN_I32 ? 3 : 7;
    const bool fine = hidden && weight && tokens && (reinterpret_cast<uintptr_t>(hidden) & value) == 0 && (reinterpret_cast<uintptr_t>(weight) & value) == 0 &&
                      (reinterpret_cast<uintptr_t>(tokens) & token) == 0;
    return fine ? rc : PCM_EINVAL;
}

}  // namespace pcm

using namespace pcm;

extern "C" {

PCM_API size_t pcm_linear_logprobs_workspace_bytes(int64_t rows, int d, int V, int dtype, int weight_layout, const void* weight,
                                                   int64_t weight_ld) {
    // (the addresses that are not given are taken to be fine)
    const void* const fine = reinterpret_cast<const void*>((uintptr_t)256);
    if (rows < 1 || check_linear(fine, d, weight, weight_ld, weight_layout, dtype, fine, PCM_TOKEN_U8, rows, d, V, 1.f) != PCM_OK) return 0;
    return plan_forward(nullptr, (int)rows, weight_source(weight, weight_ld, dtype, weight_layout, d, V, weight_layout == PCM_WEIGHT_OUT_IN)).bytes;
}

PCM_API int pcm_linear_logprobs(const void* hidden, int64_t hidden_ld, const void* weight, int64_t weight_ld, int weight_layout, int dtype,
                                const void* tokens, int token_type, int64_t rows, int d, int V, float temperature, float* logp, float* lse,
                                float* entropy, void* workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_linear(hidden, hidden_ld, weight, weight_ld, weight_layout, dtype, tokens, token_type, rows, d, V, temperature);
    if (rc == PCM_EINVAL || rows == 0) return rc;
    auto misaligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; };
    if (!logp || !lse || misaligned(logp) || misaligned(lse) || misaligned(entropy)) return PCM_EINVAL;
    if (rc != PCM_OK) return rc;
    const WeightSource src = weight_source(weight, weight_ld, dtype, weight_layout, d, V, weight_layout == PCM_WEIGHT_OUT_IN);
    const ForwardPlan f = plan_forward(workspace, (int)rows, src);
    if (!workspace_ok(workspace, workspace_bytes, f.bytes)) return PCM_EWORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const LinearRows in{hidden, hidden_ld, tokens, token_type, (int)rows, d, V};
    const float inv_t = 1.f / temperature, c = inv_t * kLog2E;
    const RowResults out{logp, lse, entropy};
    StageTimer t(ST_LINEAR_LOGPROBS, s);
    if (f.few) {
        if (dtype == PCM_F32) launch_few<float>(in, weight, weight_ld, weight_layout, f.parts, f.token_z, c, s);
        else launch_few<half_bits>(in, weight, weight_ld, weight_layout, f.parts, f.token_z, c, s);
        linear_join<1><<<(unsigned)rows, 256, 0, s>>>(in, nullptr, f.parts, f.token_z, inv_t, out);
        return launch_status();
    }
    prepare_operands(in, f.slots, nullptr, src, f.copy, f.columns, s);
    if (dtype == PCM_F32) forward_products<true>(f, src, (int)rows, c, s);
    else forward_products<false>(f, src, (int)rows, c, s);
    linear_join<4><<<(unsigned)ceil_div((int)rows, 4), 256, 0, s>>>(in, f.slots.slot_of, f.parts, f.token_z, inv_t, out);
    return launch_status();
}

}  // extern "C"
