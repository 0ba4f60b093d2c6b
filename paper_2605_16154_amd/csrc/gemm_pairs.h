// Products of matrices held as pairs (pairs.h), C[m, n] = sum_k A(m, k) B(n, k), for the orthogonalisation (internal header).
//
// Both operands are stored with the reduction index along their columns.  What the iteration multiplies is symmetric, or is
// kept in both orientations, so no other layout is needed: a product leaves its result as an operand, in one orientation or
// both.  Of a symmetric result only the tiles on and below the diagonal are computed.
#pragma once

#include "gemm_bf16.h"
#include "pairs.h"

namespace pcm {

// What becomes of a product: value = alpha * sum, with D also + beta * D + gamma * (m == n), then one of
enum PairResult : int {
    kPairs = 0,          // C and, if Ct is set, its transpose, as pairs
    kOutF32 = 1,         // out[m, n] = value
    kOutBf16 = 2,
    kOutWeights = 3      // out[m, n] (fp32) = decay * out - rate * value, and its bf16 copy to lowp if that is set
};

struct PairJob {
    const f16 *A, *B;
    union { f16* C; void* out; };
    union { f16* Ct; int64_t ld; };              // ld: of out (lowp: the same)
    union { const f16* D; uint16_t* lowp; };     // D: as C, or null
    int m_frags, n_frags;                        // fragments of rows of the operands (even)
    int steps;                                   // of 32 of k
    int16_t symmetric;                           // C = C^T: only tiles with n <= m, the others through Ct (= C)
    int16_t result;
    float alpha;
    union { float beta, decay; };
    union { float gamma, rate; };
    int rows, cols;                              // of out
    int first, tiles_m, tiles_n;                 // first workgroup, tiles: filled in by the launch
    int splits, first_part;                      // parts that a tile's reduction is done in, number of the first: as well
    __host__ __device__ int tiles() const { return symmetric ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n; }
};
constexpr int kMaxPairJobs = 16;
// The argument of a launch.  A launch with 2.7 KB of arguments takes two microseconds longer than one with 256 bytes, so few jobs on small
// tiles go as kFewPairJobs.
constexpr int kFewPairJobs = 4;
template <int kMax>
struct PairJobList {
    PairJob job[kMax];
    int n;
    f32x4* parts;                                // sums of the parts of tiles, or null
};
struct PairJobs : PairJobList<kMaxPairJobs> {
    int blocks;
};
// Reductions in parts are done on tiles of 64: by at most as many workgroups as run side by side, which is what the buffer of parts holds.
constexpr int kPairPartTile = 2, kPairParts = 512;
constexpr size_t kPairPartsBytes = (size_t)kPairParts * 64 * 64 * 4;

// Accumulators of a wavefront: tile (i, j), register t of a lane is row 16 i + (lane & 15), column 16 j + 4 (lane >> 4) + t.
template <int kW>
using PairAccumulators = f32x4[kW][kW];

__device__ inline f32x4 mfma_f16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// The wavefront's part of a tile: rows 16 (frag_m + i), columns 16 (frag_n + j).  off_diagonal: of a symmetric result, a tile whose
// transpose no other tile computes.  In blocks of 32 x 32, which a matrix has whole or not at all.
template <int kW>
__device__ __forceinline__ void store_pairs(const PairJob& p, const PairAccumulators<kW>& acc, int frag_m, int frag_n, bool off_diagonal) {
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    // Unit matrices that pick one half of a fragment's columns: a product with one is that half transposed, exactly.
    f16x8 unit[2];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        unit[0][e] = e < 4 && 4 * g + e == r ? (f16)1.f : (f16)0.f;
        unit[1][e] = e >= 4 && 4 * g + e - 4 == r ? (f16)1.f : (f16)0.f;
    }
    const bool transposed = p.Ct != nullptr && (!p.symmetric || off_diagonal);
    static_for<kW * kW / 4>([&](auto block) __attribute__((always_inline)) {
        constexpr int i = decltype(block)::value / (kW / 2) * 2, j = decltype(block)::value % (kW / 2) * 2;
        const int fm = frag_m + i, fn = frag_n + j;
        if (fm >= p.m_frags || fn >= p.n_frags) return;
        f16x8 hi[2], lo[2];
#pragma unroll
        for (int ii = 0; ii < 2; ++ii) {
            const int64_t at = pair_fragment(fm + ii, fn / 2, p.m_frags) + lane * 8;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = p.alpha * acc[i + ii][j + e / 4][e % 4];
            if (p.D != nullptr) {
                const f16x8 dh = *reinterpret_cast<const f16x8*>(p.D + at), dl = *reinterpret_cast<const f16x8*>(p.D + at + kPairPart);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] += p.beta * ((float)dh[e] + (float)dl[e]);
                    if ((fm + ii) * 16 + r == fn * 16 + e / 4 * 16 + 4 * g + e % 4) v[e] += p.gamma;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f16 h, l;
                split_pair(v[e], h, l);
                hi[ii][e] = h;
                lo[ii][e] = l;
            }
            *reinterpret_cast<f16x8*>(p.C + at) = hi[ii];
            *reinterpret_cast<f16x8*>(p.C + at + kPairPart) = lo[ii];
        }
        if (!transposed) return;
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
    });
}
template <int kW>
__device__ __forceinline__ void store_result(const PairJob& p, const PairAccumulators<kW>& acc, int frag_m, int frag_n) {
    const int lane = threadIdx.x & 63;
    const int m0 = frag_m * 16 + (lane & 15), n0 = frag_n * 16 + 4 * (lane >> 4), rows = p.rows, cols = p.cols, result = p.result;
    const float alpha = p.alpha, decay = p.decay, rate = p.rate;
    void* const out = p.out;
    __bf16* const lowp = reinterpret_cast<__bf16*>(p.lowp);
    const int64_t ld = p.ld;
    auto store = [&](int i, int j, const f32x4& sum) __attribute__((always_inline)) {
        const int m = m0 + 16 * i, n = n0 + 16 * j;
        if (m >= rows || n >= cols) return;
        const int64_t at = (int64_t)m * ld + n;
        float v[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) v[t] = alpha * sum[t];
        if (result == kOutBf16) {
            __bf16* const to = static_cast<__bf16*>(out) + at;
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (n + t < cols) to[t] = (__bf16)v[t];
            return;
        }
        float* const to = static_cast<float*>(out) + at;
        const bool whole = n + 4 <= cols;
        if (result == kOutWeights) {
            f32x4 w = {0.f, 0.f, 0.f, 0.f};
            if (whole) w = *reinterpret_cast<const f32x4_any*>(to);
            else
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (n + t < cols) w[t] = to[t];
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] = decay * w[t] - rate * v[t];
            if (lowp != nullptr)
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (n + t < cols) lowp[at + t] = (__bf16)v[t];
        }
        if (whole) *reinterpret_cast<f32x4_any*>(to) = f32x4_any{v[0], v[1], v[2], v[3]};
        else
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (n + t < cols) to[t] = v[t];
    };
    static_for<kW>([&](auto i) __attribute__((always_inline)) {
        static_for<kW>([&](auto j) __attribute__((always_inline)) { store(decltype(i)::value, decltype(j)::value, acc[decltype(i)::value][decltype(j)::value]); });
    });
}
// kFinal: the jobs of the launch leave results, not pairs.
template <int kW, bool kFinal>
__device__ __forceinline__ void pair_epilogue(const PairJob& p, const PairAccumulators<kW>& acc, int frag_m, int frag_n, bool off_diagonal) {
    if constexpr (kFinal) store_result<kW>(p, acc, frag_m, frag_n);
    else store_pairs<kW>(p, acc, frag_m, frag_n, off_diagonal);
}

constexpr int kPairThreads = 256;

// Tile number `l` of a launch's job.  Consecutive numbers are columns of bands of four rows of tiles, so that 32 of them are a
// block of 4 x 8; of a symmetric result the tiles on and below the diagonal: band b has its 16 b tiles left of column 4 b, then the
// triangle that is left.
__device__ __forceinline__ void pair_tile_at(const PairJob& p, int tiles_m, int l, int& tm, int& tn) {
    if (!p.symmetric) {
        const int first = l / (4 * p.tiles_n) * 4, rows = min(4, tiles_m - first), at = l - first * p.tiles_n;
        tm = first + at % rows;
        tn = at / rows;
        return;
    }
    int b = (int)((sqrtf(4.f + 32.f * (float)l) - 2.f) * (1.f / 16.f));      // 8 b^2 + 2 b tiles before band b
    while (8 * (b + 1) * (b + 1) + 2 * (b + 1) <= l) ++b;
    while (8 * b * b + 2 * b > l) --b;
    const int rows = min(4, tiles_m - 4 * b);
    int at = l - (8 * b * b + 2 * b);
    if (at < 4 * b * rows) {
        tm = 4 * b + at % rows;
        tn = at / rows;
        return;
    }
    at -= 4 * b * rows;
    const int row = at < 1 ? 0 : (at < 3 ? 1 : (at < 6 ? 2 : 3));
    tm = 4 * b + row;
    tn = 4 * b + at - row * (row + 1) / 2;
}
// Workgroup -> tile number, or -1: consecutive workgroups go to different XCDs, which take blocks of kBlock neighbouring tiles
// in turn and share the rest evenly (see tile_of_workgroup).
template <int kBlock>
__device__ __forceinline__ int dealt_tile(int wg, int tiles) {
    const int xcd = wg % kNumXcd, idx = wg / kNumXcd, full = tiles / (kBlock * kNumXcd);
    if (idx < full * kBlock) return ((idx / kBlock) * kNumXcd + xcd) * kBlock + idx % kBlock;
    const int rest = tiles - full * kBlock * kNumXcd, at = idx - full * kBlock;
    if (at >= rest / kNumXcd + (xcd < rest % kNumXcd ? 1 : 0)) return -1;
    return full * kBlock * kNumXcd + xcd * (rest / kNumXcd) + min(xcd, rest % kNumXcd) + at;
}
template <int kMax>
__device__ __forceinline__ PairJob job_of(const PairJobList<kMax>& jobs, int block) {
    int q = 0;
    while (q + 1 < jobs.n && block >= jobs.job[q + 1].first) ++q;
    return jobs.job[__builtin_amdgcn_readfirstlane(q)];
}

// Tiles of 32 kW x 32 kW by four wavefronts (2 x 2).
//
// A step is 32 of k: its four parts (hi and lo of both operands, 2 kW fragments each) are loaded once and take part in three
// products, in the order A_hi B_lo, A_hi B_hi, A_lo B_hi ("phases" of kW x kW MFMAs), so that between two phases one operand stays:
// the fragments of the four parts have a set of registers each, which is filled again in the phase after its last use.
// Parts are numbered 4 s + {0: B_lo, 1: A_hi, 2: B_hi, 3: A_lo} in the order of their use and live in a ring of kSlots places in LDS, filled
// by direct loads.  The one barrier of a step is behind its first phase: B_lo, A_hi and B_hi of the step have been read by then, so the
// parts up to 4 s + 2 make room, and those that will be read up to the next barrier, up to 4 s + 6, must have landed.  From one barrier to
// the next four parts are requested, 4 s + kSlots - 1 and the three after it.
// The places of a step's parts repeat after kPairPeriod steps, which the loop is unrolled by: a scalar instruction costs a quarter of an
// MFMA, and more than three of them between two MFMAs hold up the matrix pipe.  (4096 x 11008 over 4096: 766 -> 727 us, on tiles of 192
// 822 -> 783.)  One workgroup per CU for kW = 8 and 6, two for 4 and 2.
template <int kW> constexpr int kPairSlots = kW == 6 ? 12 : kW == 2 ? 16 : 10;
template <int kW> constexpr int kPairPeriod = kW == 6 ? 3 : kW == 2 ? 4 : 5;
// What bounds it: with few workgroups the matrix pipe (256-wide tile, 192 MFMAs a step: 1.28 us, at 2.4 GHz every cycle); with all CUs at work the
// board's power cap, which takes the clock to 1.9 GHz (symmetric 4096 over 4096 1.6 us a step on 136 CUs, the matrix pipes 72 to 80 % busy over whole
// launches).  Without the epilogue 3 to 10 % less time, with all loads from the first step 3 to 8.
template <int kW> constexpr uint32_t kPairPartBytes = 2u * kW * kPairPart * 2u;
// Steps beyond the last one that a tile requests (and nobody reads): so far behind a matrix there has to be memory.
constexpr int kPairStepsBeyond = 4;
template <int kW>
struct PairRing {
    __attribute__((aligned(1024))) f16 data[kPairSlots<kW> * kPairPartBytes<kW> / 2];
};

__device__ __forceinline__ void mfma_pairs(f32x4& acc, f16x8 b, f16x8 a) {
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(acc) : "v"(b), "v"(a));
}
// (see mfma_16x16x32_and_load)
template <uint32_t kLdsOffset>
__device__ __forceinline__ void mfma_pairs_and_load(f32x4& acc, f16x8 b, f16x8 a, const char* base, uint32_t lane_offset, uint32_t lds_addr) {
    asm volatile("s_add_u32 m0, %1, %2\n\t"
                 "v_mfma_f32_16x16x32_f16 %0, %3, %4, %0\n\t"
                 "global_load_lds_dwordx4 %5, %6"
                 : "+a"(acc)
                 : "s"(lds_addr), "n"(kLdsOffset), "v"(b), "v"(a), "v"(lane_offset), "s"(base)
                 : "memory", "scc");
}

template <int kW, bool kFinal, int kMax>
__global__ __launch_bounds__(kPairThreads, kW >= 6 ? 1 : 2) void pair_product(PairJobList<kMax> jobs) {
    constexpr int kSlots = kPairSlots<kW>, kLoads = kW / 2;            // loads of a part per wavefront
    constexpr uint32_t kPart = kPairPartBytes<kW>, kRing = kSlots * kPart;
    __shared__ PairRing<kW> smem;
    const PairJob p = job_of(jobs, blockIdx.x);
    constexpr bool kInParts = kW == kPairPartTile && !kFinal;
    int number = dealt_tile<(kW >= 6 ? 32 : 64)>(blockIdx.x - p.first, p.tiles() * (kInParts ? p.splits : 1));
    if (number < 0) return;
    int steps = __builtin_amdgcn_readfirstlane(p.steps), first_step = 0, part = 0;
    if constexpr (kInParts) {
        part = p.first_part + number;
        if (p.splits > 1) {              // (up to 32 parts of up to 2^15 steps)
            const int split = number % p.splits;
            number /= p.splits;
            first_step = __builtin_amdgcn_readfirstlane(steps * split / p.splits);
            steps = __builtin_amdgcn_readfirstlane(steps * (split + 1) / p.splits) - first_step;
        }
    }
    int tm, tn;
    pair_tile_at(p, p.tiles_m, number, tm, tn);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave >> 1, wn = wave & 1;
    const int first_m = tm * 2 * kW, first_n = tn * 2 * kW;           // fragments

    // Global -> LDS: load r of a part brings in fragment kLoads * wave + r, lane l its 16 bytes l.  Fragments beyond the last one are
    // read from it: what they give is not stored.
    const uint32_t lds_base = (uint32_t)(uintptr_t)PCM_AS_LDS(smem.data);
    uint32_t off[2][kLoads];
#pragma unroll
    for (int r = 0; r < kLoads; ++r) {
        const int f = kLoads * wave + r;
        off[0][r] = (uint32_t)(min(first_m + f, p.m_frags - 1) - first_m) * (kPairFragment * 2u) + (uint32_t)lane * 16u;
        off[1][r] = (uint32_t)(min(first_n + f, p.n_frags - 1) - first_n) * (kPairFragment * 2u) + (uint32_t)lane * 16u;
    }
    const char* const origin_a = tile_address<true>(p.A + pair_fragment(first_m, first_step, p.m_frags));
    const char* const origin_b = tile_address<true>(p.B + pair_fragment(first_n, first_step, p.n_frags));
    // (assembly takes them in scalar registers, and the compiler may lose sight of their being the same in every lane)
    const int64_t step_bytes[2] = {pair_fragment(0, 1, __builtin_amdgcn_readfirstlane(p.m_frags)) * 2,
                                   pair_fragment(0, 1, __builtin_amdgcn_readfirstlane(p.n_frags)) * 2};
    // by type of part: where the next one to be requested is
    const char* from[4] = {origin_b + kPairPart * 2, origin_a, origin_b, origin_a + kPairPart * 2};
    constexpr auto operand = [](int type) { return type == 0 || type == 2 ? 1 : 0; };
    const uint32_t my_lds = lds_base + (uint32_t)(kLoads * wave) * 1024u;

    // Small tiles have the registers for the sums of the two products with a lo by themselves: the sums of hi hi then round a third as often
    // (short side 40 over 1505 fp32: errors 1.9 times those of fp32 products, so 1.1).
    constexpr bool kApart = kW <= 4;
    PairAccumulators<kW> acc;
    PairAccumulators<kApart ? kW : 1> low;
#pragma unroll
    for (int i = 0; i < kW; ++i)
#pragma unroll
        for (int j = 0; j < kW; ++j) {
            acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            if constexpr (kApart) low[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

    f16x8 set[4][kW];                                    // fragments, by type of part
    const uint32_t read_base[2] = {lds_base + (uint32_t)(wm * kW) * 1024u + (uint32_t)lane * 16u,
                                   lds_base + (uint32_t)(wn * kW) * 1024u + (uint32_t)lane * 16u};
    // fragment i of this wavefront in the part that lies at place `slot`: an address per 48 KB of LDS, the rest is the instruction's offset
    constexpr uint32_t kReach = 48 * 1024;
    constexpr int kBases = (kRing + kReach - 1) / kReach;
    uint32_t at[2][kBases];
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
        for (int q = 0; q < kBases; ++q) {
            at[o][q] = read_base[o] + q * kReach;
            asm volatile("" : "+v"(at[o][q]));
        }
    auto read = [&](int o, int slot, int i) __attribute__((always_inline)) -> f16x8 {
        const uint32_t offset = (uint32_t)slot * kPart + (uint32_t)i * 1024u;
        return *(const __attribute__((address_space(3))) f16x8*)(uintptr_t)(at[o][offset / kReach] + offset % kReach);
    };

    // Prologue: parts 0 .. kSlots - 3; the first phase requests the next one.
#pragma unroll
    for (int n = 0; n < kSlots - 2; ++n) {
#pragma unroll
        for (int r = 0; r < kLoads; ++r) direct_load_16B(from[n & 3], off[operand(n & 3)][r], my_lds + (uint32_t)n * kPart + (uint32_t)r * 1024u);
        from[n & 3] += step_bytes[operand(n & 3)];
    }
    wait_direct_loads<(kSlots - 5) * kLoads>();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kW; ++i) {
        set[0][i] = read(1, 0, i);
        set[1][i] = read(0, 1, i);
    }

    // A phase: kW x kW MFMAs, row by row.  first_part: the number, modulo the ring, of the first part requested meanwhile, of kParts (one or
    // two); its loads are spread over the phase, one to an MFMA, and the pointer moves on one MFMA later.  reads(n): fragment read n of
    // kReads, one behind an MFMA, early enough for all to have landed when the phase ends.
    auto phase = [&](auto a_type, auto b_type, auto first_type, auto first_slot, auto n_parts, auto n_reads, auto reads) __attribute__((always_inline)) {
        constexpr int kA = decltype(a_type)::value, kB = decltype(b_type)::value;
        constexpr int kType = decltype(first_type)::value, kSlot = decltype(first_slot)::value;
        constexpr int kMfmas = kW * kW, kTotal = decltype(n_parts)::value * kLoads, kReads = decltype(n_reads)::value;
        constexpr int kEvery = kReads * 2 <= kMfmas - kW ? 2 : 1;
        static_for<kMfmas>([&](auto number) __attribute__((always_inline)) {
            constexpr int n = decltype(number)::value, i = n / kW, j = (i & 1) ? kW - 1 - n % kW : n % kW;
            // load l is issued at MFMA l * kMfmas / kTotal
            constexpr int l = (n * kTotal + kMfmas - 1) / kMfmas, type = (kType + l / kLoads) & 3;
            f32x4& sum = [&]() -> f32x4& {
                if constexpr (kApart && !(kA == 1 && kB == 2)) return low[i][j];
                else return acc[i][j];
            }();
            if constexpr (l < kTotal && l * kMfmas / kTotal == n) {
                constexpr uint32_t to = (uint32_t)((kSlot + l / kLoads) % kSlots) * kPart + (l % kLoads) * 1024u;
                mfma_pairs_and_load<to>(sum, set[kB][j], set[kA][i], from[type], off[operand(type)][l % kLoads], my_lds);
            } else {
                mfma_pairs(sum, set[kB][j], set[kA][i]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (l < kTotal && l * kMfmas / kTotal == n && l % kLoads == kLoads - 1) from[type] += step_bytes[operand(type)];
            if constexpr (n % kEvery == 0 && n / kEvery < kReads) reads(Index<n / kEvery>{});
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    auto step = [&](auto which) __attribute__((always_inline)) {
        constexpr int k0 = 4 * decltype(which)::value;                 // number of the step's first part, modulo the ring
        phase(Index<1>{}, Index<0>{}, Index<(kSlots - 2) & 3>{}, Index<(k0 + kSlots - 2) % kSlots>{}, Index<1>{}, Index<kW>{},
              [&](auto n) { set[2][decltype(n)::value] = read(1, (k0 + 2) % kSlots, decltype(n)::value); });
        wait_direct_loads<(kSlots - 8) * kLoads>();
        __syncthreads();
        phase(Index<1>{}, Index<2>{}, Index<(kSlots - 1) & 3>{}, Index<(k0 + kSlots - 1) % kSlots>{}, Index<2>{}, Index<2 * kW>{}, [&](auto n) {
            constexpr int f = decltype(n)::value;
            if constexpr (f < kW) set[3][f] = read(0, (k0 + 3) % kSlots, f);
            else set[0][f - kW] = read(1, (k0 + 4) % kSlots, f - kW);
        });
        phase(Index<3>{}, Index<2>{}, Index<(kSlots + 1) & 3>{}, Index<(k0 + kSlots + 1) % kSlots>{}, Index<1>{}, Index<kW>{},
              [&](auto n) { set[1][decltype(n)::value] = read(0, (k0 + 5) % kSlots, decltype(n)::value); });
    };
    for (int left = steps;;) {
        bool done = false;
        static_for<kPairPeriod<kW>>([&](auto which) __attribute__((always_inline)) {
            if (done) return;
            step(which);
            done = --left == 0;
        });
        if (done) break;
    }
    wait_direct_loads<0>();
    // the compiler does not know how long an MFMA in inline assembly takes to write its results
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
#pragma unroll
    for (int i = 0; i < kW; ++i)
#pragma unroll
        for (int j = 0; j < kW; ++j) {
            asm volatile("" : "+a"(acc[i][j]));
            if constexpr (kApart) {
                asm volatile("" : "+a"(low[i][j]));
                acc[i][j] += low[i][j];
            }
        }
    if constexpr (kInParts)
        if (p.splits > 1) {
            f32x4* const to = jobs.parts + (int64_t)(part * 4 + wave) * (kW * kW * 64) + lane;
#pragma unroll
            for (int i = 0; i < kW * kW; ++i) to[i * 64] = acc[i / kW][i % kW];
            return;
        }
    pair_epilogue<kW, kFinal>(p, acc, first_m + wm * kW, first_n + wn * kW, tm != tn);
}

// The sums of the parts, in order, and what is to become of them: a workgroup per tile.  Products with it, in one part / as planned: symmetric 64 over 2048
// 11.0 / 9.0 us, over 11008 45 / 12.8, 256 over 4096 19.4 / 11.0, 512 over 11008 51 / 21.7.
template <int kMax>
__global__ __launch_bounds__(kPairThreads) void pair_join(PairJobList<kMax> jobs) {
    constexpr int kW = kPairPartTile;
    const PairJob p = job_of(jobs, blockIdx.x);
    const int number = blockIdx.x - p.first;
    if (number >= p.tiles()) return;
    int tm, tn;
    pair_tile_at(p, p.tiles_m, number, tm, tn);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    PairAccumulators<kW> acc;
#pragma unroll
    for (int i = 0; i < kW * kW; ++i) acc[i / kW][i % kW] = f32x4{0.f, 0.f, 0.f, 0.f};
    const f32x4* from = jobs.parts + (int64_t)((p.first_part + number * p.splits) * 4 + wave) * (kW * kW * 64) + lane;
    constexpr int kStride = 4 * kW * kW * 64, kRead = 4;              // parts whose loads are under way together
    int part = 0;
    for (; part + kRead <= p.splits; part += kRead, from += kRead * kStride) {
        f32x4 one[kRead][kW * kW];
#pragma unroll
        for (int r = 0; r < kRead; ++r)
#pragma unroll
            for (int i = 0; i < kW * kW; ++i) one[r][i] = from[r * kStride + i * 64];
#pragma unroll
        for (int r = 0; r < kRead; ++r)
#pragma unroll
            for (int i = 0; i < kW * kW; ++i) acc[i / kW][i % kW] += one[r][i];
    }
    for (; part < p.splits; ++part, from += kStride)
#pragma unroll
        for (int i = 0; i < kW * kW; ++i) acc[i / kW][i % kW] += from[i * 64];
    store_pairs<kW>(p, acc, (tm * 2 + (wave >> 1)) * kW, (tn * 2 + (wave & 1)) * kW, tm != tn);
}

// The microseconds a launch of the jobs is expected to take on tiles of 32 kW: what begins and ends it, its results at 4 TB/s, and per round of
// workgroups its steps.  A step takes `alone` where few workgroups run (the matrix pipe; kW = 2: loads and barriers), `shared` for each of
// those that a CU has more than one of, and `share` for each of the chip's where that is more: at full load the power cap sets the clock, at
// 1.3 to 1.6 PFLOP/s of fp16 products (kW = 2: the path from L2 into LDS, 70 GB/s per CU).  Measured, in us, tiles of 64 / 128 / 192 / 256:
// symmetric 256 over 1024 7.5 / 15.9 / 30 / 50 (estimated 7.4 / 19.5 / 30 / 62), 1024 over 1024 8.5 / 17.2 / 33 / 54 (8.3 / 20.4 / 31 / 63),
// 2048 over 2048 38 / 36 / 62 / 98 (44 / 39 / 58 / 114), 4096 over 4096 255 / 202 / 176 / 220 (266 / 215 / 175 / 223); 1024 x 2816 over 1024 23 /
// 22 / 37 / 57 (29 / 25 / 36 / 68), 4096 x 11008 over 4096 1170 / 877 / 850 / 790 (1315 / 888 / 864 / 813).
struct PairTiming {
    double fixed, alone, shared, share;
    int slots;
};
template <int kW>
constexpr PairTiming kPairTiming = kW == 8   ? PairTiming{14.0, 1.50, 1.50, 7.9e-3, 256}
                                   : kW == 6 ? PairTiming{6.0, 0.74, 0.74, 4.7e-3, 256}
                                   : kW == 4 ? PairTiming{4.4, 0.47, 0.36, 2.25e-3, 512}
                                             : PairTiming{3.5, 0.121, 0.22, 0.86e-3, 512};
// Tiles and workgroups of the jobs with every reduction in `splits` parts.
inline void place_pair_jobs(PairJobs& jobs, int kW, int splits = 1) {
    jobs.blocks = 0;
    for (int i = 0; i < jobs.n; ++i) {
        PairJob& p = jobs.job[i];
        p.tiles_m = ceil_div(p.m_frags, 2 * kW);
        p.tiles_n = ceil_div(p.n_frags, 2 * kW);
        p.splits = splits;
        p.first = p.first_part = jobs.blocks;
        jobs.blocks += ceil_div(p.tiles() * splits, kNumXcd) * kNumXcd;
    }
}
// How the products of a launch are done: on which tiles, and in how many parts where few tiles have long reductions (the sums then take a
// launch of their own, see pair_join).
struct PairPlan {
    int tile, splits;
    double us;
};
constexpr double kPairJoin = 5.0;                // us that the launch of the sums takes, beside its bytes
template <int kW>
inline double pair_time(PairJobs& jobs, int splits = 1) {
    constexpr PairTiming t = kPairTiming<kW>;
    place_pair_jobs(jobs, kW, splits);
    double tiles = 0.0, tile_steps = 0.0, bytes = 0.0, longest = 0.0;
    for (int i = 0; i < jobs.n; ++i) {
        const PairJob& p = jobs.job[i];
        tiles += p.tiles() * splits;
        tile_steps += (double)p.tiles() * p.steps;
        bytes += (double)p.m_frags * p.n_frags * 1024.0 * (p.result == kPairs && !p.symmetric ? 2 : 1);
        longest = longest > p.steps ? longest : p.steps;
    }
    const double full = floor(tiles / t.slots), rest = tiles - full * t.slots;
    auto round = [&](double n) {
        const double each = n > 256.0 ? ceil(n / 256.0) * t.shared : t.alone;
        return n > 0.0 ? (each > n * t.share ? each : n * t.share) : 0.0;
    };
    const double steps = (full * round(t.slots) + round(rest)) * (tile_steps / tiles), least = longest / splits * t.alone;
    const double join = splits > 1 ? kPairJoin + tiles * 2.0 * 16384.0 / 4.0e6 : 0.0;
    return t.fixed + bytes / 4.0e6 + join + (steps > least ? steps : least);
}
inline PairPlan plan_pair_products(PairJobs& jobs) {
    PairPlan best{2, 1, pair_time<2>(jobs)};
    auto consider = [&](int tile, int splits, double us) {
        if (us < best.us) best = PairPlan{tile, splits, us};
    };
    consider(4, 1, pair_time<4>(jobs));
    consider(6, 1, pair_time<6>(jobs));
    consider(8, 1, pair_time<8>(jobs));
    if (jobs.parts == nullptr || jobs.job[0].result != kPairs) return best;
    int steps = jobs.job[0].steps;
    for (int i = 1; i < jobs.n; ++i) steps = steps < jobs.job[i].steps ? steps : jobs.job[i].steps;
    for (int splits = 2; splits <= 32 && splits * 4 <= steps; splits *= 2) {
        const double us = pair_time<kPairPartTile>(jobs, splits);
        if (jobs.blocks > kPairParts) break;
        consider(kPairPartTile, splits, us);
    }
    return best;
}
template <int kW, int kMax>
inline void launch_pair_list(const PairJobs& jobs, hipStream_t s) {
    PairJobList<kMax> list{};
    list.n = jobs.n;
    list.parts = jobs.parts;
    int tiles = 0;
    for (int i = 0; i < jobs.n; ++i) list.job[i] = jobs.job[i];
    if (jobs.job[0].result != kPairs) pair_product<kW, true, kMax><<<(unsigned)jobs.blocks, kPairThreads, 0, s>>>(list);
    else pair_product<kW, false, kMax><<<(unsigned)jobs.blocks, kPairThreads, 0, s>>>(list);
    if (jobs.job[0].splits == 1) return;
    for (int i = 0; i < jobs.n; ++i) {
        list.job[i].first = tiles;
        tiles += list.job[i].tiles();
    }
    pair_join<kMax><<<(unsigned)tiles, kPairThreads, 0, s>>>(list);
}
template <int kW>
inline void launch_pair_tiles(PairJobs& jobs, int splits, hipStream_t s) {
    place_pair_jobs(jobs, kW, splits);
    if constexpr (kW <= 4)
        if (jobs.n <= kFewPairJobs) return launch_pair_list<kW, kFewPairJobs>(jobs, s);
    launch_pair_list<kW, kMaxPairJobs>(jobs, s);
}
inline void launch_pair_products(PairJobs& jobs, hipStream_t s) {
    const PairPlan plan = plan_pair_products(jobs);
    if (plan.tile == 8) launch_pair_tiles<8>(jobs, 1, s);
    else if (plan.tile == 6) launch_pair_tiles<6>(jobs, 1, s);
    else if (plan.tile == 4) launch_pair_tiles<4>(jobs, 1, s);
    else launch_pair_tiles<2>(jobs, plan.splits, s);
}

}  // namespace pcm
