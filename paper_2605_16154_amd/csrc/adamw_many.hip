// AdamW over all tensors of a model, states in 32 or in 8 bits.  Streaming work, bound by HBM:
//
//   pass 1  many_sumsq    fp64 partial sums of g^2 (only where the norm is asked for)
//   pass 2  many_update   norm and clip factor from the partial sums; m, v, weights in place, bf16 copy
//
// 341 M fp32 parameters: 0.27 + 1.88 ms, 5.1 and 5.5 TB/s; 203 M with bf16 gradients, bf16 copies and states in 8 bits 0.11 + 0.65, 3.8 and 5.1 TB/s (a copy reads
// and writes at 4.8).
//
// The tensors are one list of chunks of up to 2048 elements in device memory, each with the addresses it needs, so hundreds of
// tensors of any size are two launches, and a workgroup finds its work with one dependent load.
//
// States in 8 bits.  128 elements (a block) share an exponent E, that of the largest value; a code holds 3 bits behind the point and an
// exponent field f up to F: m a sign and 4 bits (F = 15), v 5 bits (F = 31: v is a square, so both reach equally far down).  f = F is E; f = 0
// holds the values below 2^(E - F + 1) at the spacing of f = 1, down to zero.  Values are rounded to one of their two neighbours with 16 random bits,
// so that their expectation is the value: v moves by a thousandth of itself per step, a hundredth of the spacing, and rounding to nearest
// would keep it where it is for good.  v > 0 never becomes 0, which would make the update m / eps.  The update itself takes m and v
// before they are rounded.  Moments and codes are integer arithmetic and fp32 without fused multiply-add, so that their bits are those of the definition (the weights
// of this form take the hardware's root and reciprocal and a fused multiply-add); none depend on the launch.
#include "adamw_many.h"

#include <algorithm>
#include <cstdlib>

#include "philox.h"

namespace pcm {
namespace {

constexpr int kThreads = 256;
static_assert(kManyChunk == kThreads * 8, "eight elements a lane");
constexpr int kSumsqGrid = 1024;
// Workgroups of the update, and how many a CU has registers for.  Steps over 341 M parameters in 32 bits / over 203 M in 8 and their values read out, by 768 / 1024 /
// 2048 workgroups, four to a CU: 2220 / 2203 / 2243 and 1039 / 982 / 978 us; by 1280, five to a CU, 2188 and 984.
constexpr int kUpdateGrid32 = 1280, kUpdatePerCu32 = 5, kUpdateGrid8 = 2048, kUpdatePerCu8 = 4;
constexpr int kSignField = 15, kSquareField = 31;

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
// Tensors lie where the caller put them: 16 bytes at a time at whatever alignment their type has.  Their addresses come out of memory, so it has
// to be said that they are global ones.
#define PCM_GLOBAL __attribute__((address_space(1)))
typedef PCM_GLOBAL f32x4 __attribute__((aligned(4))) four_floats;
typedef PCM_GLOBAL u32x4 __attribute__((aligned(2))) eight_halves;
typedef PCM_GLOBAL u32x2 __attribute__((aligned(2))) four_halves;
typedef PCM_GLOBAL u32x2 eight_codes;
typedef PCM_GLOBAL float global_float;
typedef PCM_GLOBAL uint16_t global_half;

// (a function per type: a template parameter would lose the alignment)
#define PCM_STREAMED(type, value, name)                                                                             \
    template <bool kStream>                                                                                         \
    __device__ __forceinline__ value load_##name(const type* p) { return kStream ? __builtin_nontemporal_load(p) : *p; } \
    template <bool kStream>                                                                                         \
    __device__ __forceinline__ void store_##name(type* p, value x) {                                                \
        if (kStream) __builtin_nontemporal_store(x, p);                                                             \
        else *p = x;                                                                                                \
    }
PCM_STREAMED(four_floats, f32x4, floats)
PCM_STREAMED(eight_halves, u32x4, halves)
PCM_STREAMED(four_halves, u32x2, few_halves)
PCM_STREAMED(eight_codes, u32x2, codes)
#undef PCM_STREAMED

__device__ inline uint32_t bf16_bits(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ inline float low_half(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
__device__ inline float high_half(uint32_t x) { return __builtin_bit_cast(float, x & 0xffff0000u); }

// Where a lane's eight elements of a chunk are: two fours.  States in 8 bits keep them together, 16 lanes to a block; else fours of neighbouring lanes are
// neighbours, which every access takes as whole lines.
template <bool kTogether>
__device__ inline int four_at(int h) { return kTogether ? threadIdx.x * 8 + h * 4 : h * (kManyChunk / 2) + threadIdx.x * 4; }

// A lane's gradients of a chunk as they come: fp32, or bf16 in the first half (kHalvesTogether: those are eight neighbours).
template <bool kTogether, bool kStream, bool kHalvesTogether = kTogether>
struct Gradients {
    f32x4 x[2];
    __device__ __forceinline__ void load(const AdamwChunk& k) {
        if (k.grad_bf16) {
            const global_half* p = (const global_half*)k.grad;
            u32x4 both = {0, 0, 0, 0};
            if (k.count == kManyChunk) {
                if (kHalvesTogether) both = load_halves<kStream>((const eight_halves*)(p + four_at<true>(0)));
                else {
                    const u32x2 a = load_few_halves<kStream>((const four_halves*)(p + four_at<false>(0)));
                    const u32x2 b = load_few_halves<kStream>((const four_halves*)(p + four_at<false>(1)));
                    both = u32x4{a[0], a[1], b[0], b[1]};
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = four_at<kHalvesTogether>(e / 4) + e % 4;
                    if (i < k.count) both[e / 2] |= (uint32_t)p[i] << (e % 2 * 16);
                }
            }
            x[0] = __builtin_bit_cast(f32x4, both);
        } else {
            const global_float* p = (const global_float*)k.grad;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = four_at<kTogether>(h);
                x[h] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (k.count == kManyChunk) x[h] = load_floats<kStream>((const four_floats*)(p + i));
                else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (i + e < k.count) x[h][e] = p[i + e];
                }
            }
        }
    }
    __device__ __forceinline__ void get(float (&g)[8], const AdamwChunk& k) const {
        const u32x4 both = __builtin_bit_cast(u32x4, x[0]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            g[2 * e] = k.grad_bf16 ? low_half(both[e]) : x[e / 2][e % 2 * 2];
            g[2 * e + 1] = k.grad_bf16 ? high_half(both[e]) : x[e / 2][e % 2 * 2 + 1];
        }
    }
};
// Eight fp32 values at two fours of a matrix; those from `count` on are left alone, and 0.
template <bool kTogether, bool kStream>
__device__ __forceinline__ void load_eight(f32x4 (&x)[2], const float* from, int count) {
    const global_float* p = (const global_float*)from;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = four_at<kTogether>(h);
        x[h] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (count == kManyChunk) x[h] = load_floats<kStream>((const four_floats*)(p + i));
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < count) x[h][e] = p[i + e];
        }
    }
}
template <bool kTogether, bool kStream>
__device__ __forceinline__ void store_eight(float* to, const float (&x)[8], int count) {
    global_float* p = (global_float*)to;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int i = four_at<kTogether>(h);
        if (count == kManyChunk) store_floats<kStream>((four_floats*)(p + i), f32x4{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]});
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < count) p[i + e] = x[4 * h + e];
        }
    }
}
template <bool kTogether>
__device__ __forceinline__ void store_bf16(uint16_t* to, const float (&x)[8], int count) {
    global_half* p = (global_half*)to;
    u32x4 a;
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = bf16_bits(x[2 * e]) | bf16_bits(x[2 * e + 1]) << 16;
    if (count == kManyChunk) {
        if (kTogether) store_halves<false>((eight_halves*)(p + four_at<true>(0)), a);
        else {
            store_few_halves<false>((four_halves*)(p + four_at<false>(0)), u32x2{a[0], a[1]});
            store_few_halves<false>((four_halves*)(p + four_at<false>(1)), u32x2{a[2], a[3]});
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int i = four_at<kTogether>(e / 4) + e % 4;
            if (i < count) p[i] = (uint16_t)(a[e / 2] >> (e % 2 * 16));
        }
    }
}

// Sum over the workgroup, in every thread; the same order whatever the values.
__device__ inline double block_sum(double x) {
    __shared__ double lds[kThreads / 64];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) x += __shfl_xor(x, off, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__global__ __launch_bounds__(kThreads) void many_sumsq(const AdamwChunk* chunks, int64_t n, double* partial) {
    double acc[8] = {};
    auto add = [&](const AdamwChunk& k, const Gradients<false, false, true>& x) __attribute__((always_inline)) {
        float g[8];
        x.get(g, k);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = __builtin_fma((double)g[e], (double)g[e], acc[e]);
    };
    // four chunks under way
    constexpr int kAhead = 4;
    int64_t at = blockIdx.x;
    for (; at + (int64_t)(kAhead - 1) * gridDim.x < n; at += (int64_t)kAhead * gridDim.x) {
        AdamwChunk k[kAhead];
        Gradients<false, false, true> x[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            k[q] = chunks[at + (int64_t)q * gridDim.x];
            x[q].load(k[q]);
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) add(k[q], x[q]);
    }
    for (; at < n; at += gridDim.x) {
        const AdamwChunk k = chunks[at];
        Gradients<false, false, true> x;
        x.load(k);
        add(k, x);
    }
    const double total = block_sum(((acc[0] + acc[1]) + (acc[2] + acc[3])) + ((acc[4] + acc[5]) + (acc[6] + acc[7])));
    if (threadIdx.x == 0) partial[blockIdx.x] = total;
}

// Largest value among the 16 lanes that hold a block.
__device__ inline uint32_t block_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x128, 0xf, 0xf, true));       // rotated by 8, 4, 2 and 1 lanes
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x124, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x122, 0xf, 0xf, true));
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x121, 0xf, 0xf, true));
}
// Eight values of a block whose exponent is `top`, from their codes.  A code is the upper bits of an fp32 number whose exponent field is f, numbers below the
// normal ones for f = 0 included: in place, it is that number times a power of two.
template <int kField>
__device__ __forceinline__ void values_of(float (&x)[8], u32x2 codes, int top) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t word = codes[e / 4];
        const uint32_t bits = kField == kSquareField ? (word >> (e % 4 * 8) & 255u) << 20
                                                     : (uint32_t)((int32_t)(word << (24 - e % 4 * 8)) >> 4) & 0x87f00000u;
        x[e] = ldexpf(__builtin_bit_cast(float, bits), top - kField);
    }
    if (!__any(top == 255)) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = top == 255 ? __builtin_nanf("") : x[e];
}
// Exponent of a block, from each lane's eight values (as bits without a sign) and these with their random bits added.
__device__ __forceinline__ int exponent_of(const uint32_t (&bits)[8], const uint32_t (&sum)[8]) {
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, sum[e]);
    most = block_max(most);
    // zeros and what is below the normal numbers count as nothing, which matters where there is nothing else
    if (__any(most < 3u << 23)) {
        most = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) most = max(most, bits[e] < 1u << 23 ? 0u : sum[e]);
        most = block_max(most);
    }
    return (int)min(most >> 23, 255u);
}
// Codes of eight values, without signs.  True where those of the wavefront are all of blocks of zeros or at least 8 (f > 0): an addition and a shift.
// Others are rare, and the lanes go the long way together.
template <int kField>
__device__ __forceinline__ bool codes_of(uint32_t (&code)[8], const uint32_t (&bits)[8], const uint32_t (&sum)[8], const uint32_t (&random)[8], int top) {
    const int base = top > 0 ? (top - kField) << 3 : 1 << 12;
    int least = base;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = (int)(sum[e] >> 20) - base;
        least = e == 0 ? c : min(least, c);
        code[e] = (uint32_t)max(c, 0);
    }
    if (!__any(top > 0 && (least < 8 || top <= kField || top == 255))) return true;
    // below 2^(top - kField + 1): multiples of 2^(top - kField - 2), of which 16 bits behind the point count
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (bits[e] < 1u << 23) code[e] = 0;
        else if (code[e] < 8) {
            code[e] = ((uint32_t)ldexpf(__builtin_bit_cast(float, bits[e]), 16 + 129 + kField - top) + (random[e] >> 4)) >> 16;
            if (kField == kSquareField) code[e] = max(code[e], 1u);
        }
    }
    return false;
}
// A lane's eight values of a block as codes; the first n count, the others pad a tensor.
template <int kField>
__device__ __forceinline__ u32x2 coded(int& top, const float (&x)[8], const uint32_t (&random)[8], int n) {
    uint32_t bits[8], sum[8], code[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) bits[e] = __builtin_bit_cast(uint32_t, x[e]) & 0x7fffffffu;
    if (__any(n < 8)) {
#pragma unroll
        for (int e = 0; e < 8; ++e) bits[e] = e < n ? bits[e] : 0u;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = bits[e] + random[e];
    top = exponent_of(bits, sum);
    const bool plain = codes_of<kField>(code, bits, sum, random, top);
    if (kField == kSignField) {
        const uint32_t sign = top > 0 ? 128u : 0u;            // (a code of 0 has none)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            code[e] = (plain ? code[e] : code[e] & 127u) | (__builtin_bit_cast(uint32_t, x[e]) >> 24 & (plain || code[e] != 0 ? sign : 0u));
    } else if (!plain) {
#pragma unroll
        for (int e = 0; e < 8; ++e) code[e] &= 255u;
    }
    u32x2 out = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e / 4] |= code[e] << (e % 4 * 8);
    return out;
}

// Norm and clip factor; every workgroup forms them from the partial sums by itself.  They are asked for before anything else.
struct ClipFactor {
    static constexpr int kEach = kSumsqGrid / kThreads;
    double part[kEach];
    __device__ __forceinline__ void load(const ManyStep& s) {
#pragma unroll
        for (int q = 0; q < kEach; ++q) {
            const int i = q * kThreads + threadIdx.x;
            part[q] = i < s.parts ? s.partial[i] : 0.0;
        }
    }
    __device__ __forceinline__ float get(const ManyStep& s) const {
        if (s.parts == 0) return 1.f;
        const double norm = sqrt(block_sum((part[0] + part[1]) + (part[2] + part[3])));
        if (s.norm_out != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *s.norm_out = (float)norm;
        // (a norm that is NaN makes the factor NaN: fmin alone would let every gradient through at its full size)
        if (s.max_norm == __builtin_huge_val()) return 1.f;
        return norm == norm ? (float)fmin(1.0, s.max_norm / (norm + 1e-6)) : __builtin_nanf("");
    }
};
static_assert(ClipFactor::kEach == 4, "");

// What a lane takes up of a chunk.
template <int kBits, bool kStream>
struct Eight;
template <bool kStream>
struct Eight<32, kStream> {
    AdamwChunk k;
    Gradients<false, kStream> g;
    f32x4 w[2], m[2], v[2];
    __device__ __forceinline__ void load(const ManyStep& s, int64_t chunk) {
        k = s.chunks[chunk];
        const float* const state = reinterpret_cast<const float*>(s.state) + k.at;
        g.load(k);
        load_eight<false, kStream>(w, k.weight, k.count);
        load_eight<false, kStream>(m, state, k.count);
        load_eight<false, kStream>(v, state + s.elements, k.count);
    }
    __device__ __forceinline__ void get(float (&mm)[8], float (&vv)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) { mm[e] = m[e / 4][e % 4]; vv[e] = v[e / 4][e % 4]; }
    }
    __device__ __forceinline__ void put(const ManyStep& s, const float (&mm)[8], const float (&vv)[8]) const {
        float* const state = reinterpret_cast<float*>(s.state) + k.at;
        store_eight<false, kStream>(state, mm, k.count);
        store_eight<false, kStream>(state + s.elements, vv, k.count);
    }
};
template <bool kStream>
struct Eight<8, kStream> {
    AdamwChunk k;
    Gradients<true, kStream> g;
    f32x4 w[2];
    u32x2 m, v;
    int m_top, v_top;
    __device__ __forceinline__ bool in_block() const { return (int)threadIdx.x * 8 < (k.count + kManyBlock - 1) / kManyBlock * kManyBlock; }
    __device__ __forceinline__ void load(const ManyStep& s, int64_t chunk) {
        k = s.chunks[chunk];
        g.load(k);
        // (a line of weights is two loads of a lane's neighbours: the second finds it in the cache)
        load_eight<true, false>(w, k.weight, k.count);
        m = v = u32x2{0, 0};
        m_top = v_top = 0;
        if (!in_block()) return;
        const int64_t j = k.at + threadIdx.x * 8;
        const PCM_GLOBAL uint8_t* const state = (const PCM_GLOBAL uint8_t*)s.state;
        const PCM_GLOBAL uint8_t* const tops = state + 2 * s.elements + j / kManyBlock;
        m = load_codes<kStream>((const eight_codes*)(state + j));
        v = load_codes<kStream>((const eight_codes*)(state + s.elements + j));
        m_top = tops[0];
        v_top = tops[s.elements / kManyBlock];
    }
    __device__ __forceinline__ void get(float (&mm)[8], float (&vv)[8]) const {
        values_of<kSignField>(mm, m, m_top);
        values_of<kSquareField>(vv, v, v_top);
    }
    __device__ __forceinline__ void put(const ManyStep& s, const float (&mm)[8], const float (&vv)[8]) const {
        if (!in_block()) return;                              // by whole blocks, so the lanes of a block stay together
        const int64_t j = k.at + threadIdx.x * 8;
        const int n = k.count - (int)threadIdx.x * 8;
        const uint64_t group = (uint64_t)(j / 8);
        const PhiloxWords bits = philox4x32((uint32_t)group, (uint32_t)(group >> 32), s.step[0], s.step[1], s.seed[0], s.seed[1]);
        uint32_t random[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) random[e] = (bits.w[e / 2] >> (e % 2 * 16) & 0xffffu) << 4;
        int m_new, v_new;
        const u32x2 mc = coded<kSignField>(m_new, mm, random, n);
        __builtin_amdgcn_sched_barrier(0);                    // (registers for one of the two)
        const u32x2 vc = coded<kSquareField>(v_new, vv, random, n);
        PCM_GLOBAL uint8_t* const state = (PCM_GLOBAL uint8_t*)s.state;
        store_codes<kStream>((eight_codes*)(state + j), mc);
        store_codes<kStream>((eight_codes*)(state + s.elements + j), vc);
        if ((threadIdx.x & 15) == 0) {
            PCM_GLOBAL uint8_t* const tops = state + 2 * s.elements + j / kManyBlock;
            tops[0] = (uint8_t)m_new;
            tops[s.elements / kManyBlock] = (uint8_t)v_new;
        }
    }
};

// A workgroup takes every gridDim-th chunk, the next one's values under way while one is worked on; the first one's while the norm is formed.
template <int kBits, bool kStream>
__global__ __launch_bounds__(kThreads, kBits == 8 ? kUpdatePerCu8 : kUpdatePerCu32) void many_update(ManyStep s) {
    constexpr bool kTogether = kBits == 8;
    const AdamConst& c = s.c;
    int64_t at = blockIdx.x;
    auto chunk = [&](int64_t i) { return kStream ? s.n - 1 - i : i; };
    ClipFactor clip;
    clip.load(s);
    Eight<kBits, kStream> x;
    if (at < s.n) x.load(s, chunk(at));
    const float scale = clip.get(s);
    for (; at < s.n; at += gridDim.x) {
        const Eight<kBits, kStream> now = x;
        if (at + gridDim.x < s.n) x.load(s, chunk(at + gridDim.x));
        float g[8], w[8], m[8], v[8];
        now.g.get(g, now.k);
        now.get(m, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = g[e] * scale;
            m[e] = c.beta1 * m[e] + c.one_minus_beta1 * y;
            v[e] = c.beta2 * v[e] + c.one_minus_beta2 * (y * y);
            // (8 bits: root and reciprocal of the hardware, 1 ulp each: with the exact ones the update of 203 M parameters takes 10 % longer)
            const float root = kBits == 8 ? __builtin_amdgcn_sqrtf(v[e]) : sqrtf(v[e]);
            const float old = now.w[e / 4][e % 4] * c.decay;
            if constexpr (kBits == 8)
                w[e] = __builtin_fmaf(-c.step_size, m[e] * __builtin_amdgcn_rcpf(__builtin_fmaf(root, c.inv_sqrt_bc2, c.eps)), old);
            else w[e] = old - c.step_size * (m[e] / (root * c.inv_sqrt_bc2 + c.eps));
        }
        store_eight<kTogether, kStream && !kTogether>(now.k.weight, w, now.k.count);
        if (now.k.lowp != nullptr) store_bf16<kTogether>(now.k.lowp, w, now.k.count);
        now.put(s, m, v);
    }
}

// The values of 8-bit states: bf16 holds them exactly, as fp32 does (down to the least bf16 value, 2^-133).
template <bool kBf16>
__global__ __launch_bounds__(kThreads) void many_states(const uint8_t* state, int64_t elements, void* m_out, void* v_out) {
    for (int64_t j = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 8; j < elements; j += (int64_t)gridDim.x * kManyChunk) {
        const uint8_t* const tops = state + 2 * elements + j / kManyBlock;
        const u32x2 mc = *reinterpret_cast<const u32x2*>(state + j), vc = *reinterpret_cast<const u32x2*>(state + elements + j);
        const int m_top = tops[0], v_top = tops[elements / kManyBlock];
        float m[8], v[8];
        values_of<kSignField>(m, mc, m_top);
        values_of<kSquareField>(v, vc, v_top);
        auto write = [&](void* out, const float (&x)[8]) {
            if (kBf16) {
                u32x4 a;
#pragma unroll
                for (int e = 0; e < 4; ++e) a[e] = bf16_bits(x[2 * e]) | bf16_bits(x[2 * e + 1]) << 16;
                store_halves<false>((eight_halves*)(static_cast<uint16_t*>(out) + j), a);
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    store_floats<false>((four_floats*)(static_cast<float*>(out) + j + 4 * h), f32x4{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]});
            }
        };
        write(m_out, m);
        write(v_out, v);
    }
}

// ---- host side -----------------------------------------------------------------------------------

constexpr int64_t kMostElements = (int64_t)1 << 42;

bool layout_of(int n_tensors, const int64_t* numel, int state_bits, pcm_adamw_many_layout& out) {
    if (n_tensors < 1 || numel == nullptr || (state_bits != 8 && state_bits != 32)) return false;
    int64_t chunks = 0, elements = 0;
    for (int i = 0; i < n_tensors; ++i) {
        if (numel[i] < 0 || numel[i] > kMostElements) return false;
        chunks += ceil_div64(numel[i], kManyChunk);
        elements += ceil_div64(numel[i], kManyBlock) * kManyBlock;
        if (elements > kMostElements) return false;
    }
    out.chunks = chunks;
    out.elements = elements;
    out.plan_bytes = (size_t)chunks * sizeof(AdamwChunk);
    out.state_bytes = state_bits == 32 ? (size_t)elements * 8 : (size_t)elements * 2 + (size_t)(elements / kManyBlock) * 2;
    out.state_bits = state_bits;
    return true;
}
bool layout_ok(const pcm_adamw_many_layout* l) {
    return l != nullptr && l->chunks >= 0 && l->elements >= 0 && l->elements <= kMostElements && l->elements % kManyBlock == 0 &&
           l->chunks <= l->elements / kManyBlock && l->elements <= l->chunks * kManyChunk && (l->state_bits == 8 || l->state_bits == 32);
}
bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
int sumsq_grid(int64_t chunks) { return (int)std::min<int64_t>(kSumsqGrid, chunks); }

struct Extent {
    uintptr_t begin, end;
    bool written;
};
void sift(Extent* x, int64_t n, int64_t i) {
    for (int64_t child; (child = 2 * i + 1) < n; i = child) {
        if (child + 1 < n && x[child].begin < x[child + 1].begin) ++child;
        if (x[i].begin >= x[child].begin) return;
        const Extent t = x[i];
        x[i] = x[child];
        x[child] = t;
    }
}
// Whether something that is written shares memory with anything else (sorted in place: nothing here may throw).
bool share_memory(Extent* x, int64_t n) {
    for (int64_t i = n / 2 - 1; i >= 0; --i) sift(x, n, i);
    for (int64_t last = n - 1; last > 0; --last) {
        const Extent t = x[0];
        x[0] = x[last];
        x[last] = t;
        sift(x, last, 0);
    }
    uintptr_t end = 0, written_end = 0;               // of those that begin earlier
    for (int64_t i = 0; i < n; ++i) {
        if (x[i].begin < (x[i].written ? end : written_end)) return true;
        if (x[i].end > end) end = x[i].end;
        if (x[i].written && x[i].end > written_end) written_end = x[i].end;
    }
    return false;
}

// The update has eps in fp32; where neither moment has met a gradient it divides by nothing else, and the hardware's reciprocal takes what is below the
// normal numbers for 0.
constexpr double kLeastEps = 0x1p-126;
// Parameters beyond which a step's arrays outgrow the 256 MB memory-side cache.
constexpr int64_t kStreamElements = 20 << 20;

}  // namespace
}  // namespace pcm

using namespace pcm;

extern "C" {

PCM_API int pcm_adamw_many_describe(int n_tensors, const int64_t* numel, int state_bits, pcm_adamw_many_layout* layout) {
    pcm_adamw_many_layout l{};
    if (layout == nullptr || !layout_of(n_tensors, numel, state_bits, l)) return PCM_EINVAL;
    *layout = l;
    return PCM_OK;
}

PCM_API int pcm_adamw_many_plan(int n_tensors, const int64_t* numel, const void* const* grads, const int* grad_dtypes,
                                float* const* weights, void* const* weights_bf16, void* plan, size_t plan_bytes) {
    pcm_adamw_many_layout l{};
    if (!layout_of(n_tensors, numel, 32, l) || !grads || !grad_dtypes || !weights || !aligned(plan, 8)) return PCM_EINVAL;
    if (plan_bytes < l.plan_bytes || (plan == nullptr && l.plan_bytes > 0)) return PCM_EWORKSPACE;
    int64_t extents = 0;
    for (int i = 0; i < n_tensors; ++i) {
        if (grad_dtypes[i] != PCM_F32 && grad_dtypes[i] != PCM_BF16) return PCM_EINVAL;
        if (numel[i] == 0) continue;
        void* lowp = weights_bf16 ? weights_bf16[i] : nullptr;
        if (!grads[i] || !weights[i] || !aligned(grads[i], grad_dtypes[i] == PCM_F32 ? 4 : 2) || !aligned(weights[i], 4) || !aligned(lowp, 2))
            return PCM_EINVAL;
        extents += lowp ? 3 : 2;
    }
    if (extents == 0) return PCM_OK;
    Extent* const extent = static_cast<Extent*>(malloc((size_t)extents * sizeof(Extent)));
    if (extent == nullptr) return PCM_EWORKSPACE;
    int64_t n = 0;
    for (int i = 0; i < n_tensors; ++i) {
        if (numel[i] == 0) continue;
        auto add = [&](const void* p, int64_t bytes, bool written) { extent[n++] = Extent{(uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes, written}; };
        add(grads[i], numel[i] * (grad_dtypes[i] == PCM_F32 ? 4 : 2), false);
        add(weights[i], numel[i] * 4, true);
        if (weights_bf16 && weights_bf16[i]) add(weights_bf16[i], numel[i] * 2, true);
    }
    const bool shared = share_memory(extent, n);
    free(extent);
    if (shared) return PCM_EINVAL;
    AdamwChunk* to = static_cast<AdamwChunk*>(plan);
    int64_t first = 0;
    for (int i = 0; i < n_tensors; ++i) {
        const bool half = grad_dtypes[i] == PCM_BF16;
        for (int64_t at = 0; at < numel[i]; at += kManyChunk) {
            const int64_t count = numel[i] - at < kManyChunk ? numel[i] - at : kManyChunk;
            *to++ = AdamwChunk{static_cast<const char*>(grads[i]) + at * (half ? 2 : 4), weights[i] + at,
                               weights_bf16 && weights_bf16[i] ? static_cast<uint16_t*>(weights_bf16[i]) + at : nullptr, first + at,
                               (int32_t)count, half};
        }
        first += ceil_div64(numel[i], kManyBlock) * kManyBlock;
    }
    return PCM_OK;
}

PCM_API size_t pcm_adamw_many_step_workspace_bytes(const pcm_adamw_many_layout* layout) {
    if (!layout_ok(layout)) return 0;
    Carver c(nullptr);
    c.take<double>(kSumsqGrid);
    return c.used();
}

PCM_API int pcm_adamw_many_step(const void* plan, const pcm_adamw_many_layout* layout, void* state, int64_t step, double lr, double beta1,
                                double beta2, double eps, double weight_decay, double max_grad_norm, uint64_t seed, float* grad_norm_out,
                                void* workspace, size_t workspace_bytes, void* stream) {
    if (!layout_ok(layout) || !adam_arguments_ok(step, lr, beta1, beta2, eps, weight_decay, max_grad_norm) || !aligned(plan, 8) ||
        !aligned(state, 16) || !aligned(grad_norm_out, 4) || !(eps >= kLeastEps))
        return PCM_EINVAL;
    if (layout->chunks > 0 && (!plan || !state)) return PCM_EINVAL;
    const bool want_norm = max_grad_norm < __builtin_huge_val() || grad_norm_out != nullptr;
    if (want_norm && !workspace_ok(workspace, workspace_bytes, pcm_adamw_many_step_workspace_bytes(layout))) return PCM_EWORKSPACE;
    if (layout->chunks == 0 && grad_norm_out == nullptr) return PCM_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    ManyStep a{};
    a.chunks = static_cast<const AdamwChunk*>(plan);
    a.n = layout->chunks;
    a.state = static_cast<char*>(state);
    a.elements = layout->elements;
    a.max_norm = max_grad_norm;
    a.norm_out = grad_norm_out;
    a.c = adam_const(step, lr, beta1, beta2, eps, weight_decay);
    a.step[0] = (uint32_t)step; a.step[1] = (uint32_t)((uint64_t)step >> 32);
    a.seed[0] = (uint32_t)seed; a.seed[1] = (uint32_t)(seed >> 32);
    if (want_norm) {
        Carver c(workspace);
        double* const partial = c.take<double>(kSumsqGrid);
        a.partial = partial;
        a.parts = a.n > 0 ? sumsq_grid(a.n) : 1;
        StageTimer t(ST_OPT_NORM, s);
        many_sumsq<<<(unsigned)a.parts, kThreads, 0, s>>>(a.chunks, a.n, partial);
    }
    StageTimer t(ST_OPT_ADAMW, s);
    const int64_t most = layout->state_bits == 8 ? kUpdateGrid8 : kUpdateGrid32;
    const unsigned grid = (unsigned)(a.n < 1 ? 1 : a.n < most ? a.n : most);
    const bool past = a.elements > kStreamElements;
    if (layout->state_bits == 32) {
        if (past) many_update<32, true><<<grid, kThreads, 0, s>>>(a);
        else many_update<32, false><<<grid, kThreads, 0, s>>>(a);
    } else {
        if (past) many_update<8, true><<<grid, kThreads, 0, s>>>(a);
        else many_update<8, false><<<grid, kThreads, 0, s>>>(a);
    }
    return launch_status();
}

PCM_API int pcm_adamw_many_states(const pcm_adamw_many_layout* layout, const void* state, int dtype, void* m_out, void* v_out, void* stream) {
    if (!layout_ok(layout) || layout->state_bits != 8 || (dtype != PCM_F32 && dtype != PCM_BF16) || !aligned(state, 16) ||
        !aligned(m_out, dtype == PCM_F32 ? 4 : 2) || !aligned(v_out, dtype == PCM_F32 ? 4 : 2))
        return PCM_EINVAL;
    if (layout->elements == 0) return PCM_OK;
    if (!state || !m_out || !v_out) return PCM_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    StageTimer t(ST_OPT_ADAMW, s);
    const int64_t groups = ceil_div64(layout->elements, kManyChunk);
    const unsigned grid = (unsigned)(groups < 8192 ? groups : 8192);
    if (dtype == PCM_BF16) many_states<true><<<grid, kThreads, 0, s>>>(static_cast<const uint8_t*>(state), layout->elements, m_out, v_out);
    else many_states<false><<<grid, kThreads, 0, s>>>(static_cast<const uint8_t*>(state), layout->elements, m_out, v_out);
    return launch_status();
}

}  // extern "C"
