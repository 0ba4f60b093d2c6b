// Log-probabilities of given tokens, entropy and the likeliest alternatives from rows of logits, and their gradient.
//
// With x = logit / temperature over the allowed tokens of a row: lse = log sum e^x, log p(token) = x_token - lse,
// entropy = lse - sum p x, and the `top` tokens of the largest logits (of equal ones the lower index).  One pass over the row:
// every lane keeps s = sum 2^a and t = sum 2^a a with a = (logit - r) (log2 e) / temperature relative to the largest logit r that it has met,
// which moves once per chunk of eight logits at most; of two lanes' sums the larger logit stays.  So a <= 0 <= log s in the end: entropy
// = log s - (t / s) ln 2 and -logp are sums of terms of one sign, and as exact for a row that is all but certain (relative to some other
// logit both are differences of numbers that may be much larger).  All sums are fp32.
//
// Bound by memory where there is much of it: a logit costs ten instructions and a chunk some ten more, one of them an exponential at a
// quarter of the rate, which is 6.5 TB/s of bf16 logits.
//
// Gradient: d logit_j = ([j = token] d_logp - p_j (d_logp + d_entropy (log p_j + entropy))) / temperature, from lse and entropy as
// the forward pass left them: every logit is read once and its gradient written once.  (Rows whose lse is too large: see kLseCarries.)
#include <algorithm>
#include <type_traits>

#include "token_logprobs.h"

namespace pcm {
namespace {

constexpr int kTopMost = 64;                 // one list entry per lane
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

constexpr float kLowest = -3.402823466e38f;  // of the finite values

__device__ inline float infinity() { return __builtin_huge_valf(); }
__device__ inline int ceil_div_device(int a, int b) { return (int)(((int64_t)a + b - 1) / b); }

// The token of a row: -1 where it has none, V - 1 where it is beyond the last.
__device__ inline int token_of(const Logits& q, int64_t row) {
    const int64_t t = q.token_type == PCM_TOKEN_U8    ? (int64_t) static_cast<const uint8_t*>(q.tokens)[row]
                      : q.token_type == PCM_TOKEN_I32 ? (int64_t) static_cast<const int32_t*>(q.tokens)[row]
                                                      : static_cast<const int64_t*>(q.tokens)[row];
    return t < 0 ? -1 : (t >= q.V ? q.V - 1 : (int)t);
}

template <class T> __device__ inline float to_float(T x);
template <> __device__ inline float to_float<float>(float x) { return x; }
template <> __device__ inline float to_float<uint16_t>(uint16_t x) { return __builtin_bit_cast(float, (uint32_t)x << 16); }

// Eight logits of a row from j on; ok: bit e is set where token j + e exists and is allowed.  The others read as -inf.  (Rows
// start at any multiple of the type's size: global memory takes 8- and 16-byte accesses at every address.)
typedef __attribute__((ext_vector_type(4), aligned(4))) float f32x4_any;
typedef __attribute__((ext_vector_type(8), aligned(2))) uint16_t u16x8_any;
typedef __attribute__((aligned(1))) uint64_t u64_any;

template <class T> struct Eight;
template <>
struct Eight<float> {
    f32x4_any a, b;
    __device__ void load(const float* p) {
        a = *reinterpret_cast<const f32x4_any*>(p);
        b = *reinterpret_cast<const f32x4_any*>(p + 4);
    }
    __device__ float operator[](int e) const { return e < 4 ? a[e] : b[e - 4]; }
};
template <>
struct Eight<uint16_t> {
    u16x8_any a;
    __device__ void load(const uint16_t* p) { a = *reinterpret_cast<const u16x8_any*>(p); }
    __device__ float operator[](int e) const { return to_float<uint16_t>(a[e]); }
};
// All eight are in the row: the loads, which may be well ahead of the use, and the use.
template <class T, bool kMask>
struct WholeChunk {
    Eight<T> z;
    uint64_t mask;
    __device__ void load(const T* row, const uint8_t* allowed, int j) {
        z.load(row + j);
        if (kMask) mask = *reinterpret_cast<const u64_any*>(allowed + j);
    }
    __device__ uint32_t get(float (&out)[8]) const {
        uint32_t ok = 0xFF;
        if (kMask) {
            ok = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) ok |= (uint32_t)((mask >> (8 * e) & 0xFF) != 0) << e;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = !kMask || (ok >> e & 1) ? z[e] : -infinity();
        return ok;
    }
};
template <class T, bool kMask>
__device__ inline uint32_t load_chunk(const T* row, const uint8_t* allowed, int j, int V, float (&z)[8]) {
    if (j + 8 <= V) {
        WholeChunk<T, kMask> c;
        c.load(row, allowed, j);
        return c.get(z);
    }
    uint32_t ok = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bool in = j + e < V && (!kMask || allowed[j + e] != 0);
        z[e] = in ? to_float<T>(row[j + e]) : -infinity();
        ok |= (uint32_t)in << e;
    }
    return ok;
}
// f(j, z, ok) for the chunks from `begin` to `end` that this thread of kStride has, the loads of kAhead chunks under way while as many
// are worked on: with one at a time a wavefront waits for each (4096 rows of 65536 bf16 164 us).
// start() is called once the first of them are under way: false ends it there.
constexpr int kAhead = 2;
template <class T, bool kMask, int kStride, class Start, class F>
__device__ __forceinline__ bool each_chunk(const T* row, const uint8_t* allowed, int begin, int end, int V, int lane, Start start, F f) {
    constexpr int kUnit = kStride * 8;
    const int rounds = max(0, min(end, V) - begin) / (kAhead * kUnit);           // of chunks that are whole in every lane
    int j = begin + lane * 8;
    if (rounds > 0) {
        WholeChunk<T, kMask> now[kAhead], next[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) now[u].load(row, allowed, j + u * kUnit);
        if (!start()) return false;
        for (int i = 0; i < rounds; ++i) {
            if (i + 1 < rounds)
#pragma unroll
                for (int u = 0; u < kAhead; ++u) next[u].load(row, allowed, j + (kAhead + u) * kUnit);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                float z[8];
                const uint32_t ok = now[u].get(z);
                f(j + u * kUnit, z, ok);
                now[u] = next[u];
            }
            j += kAhead * kUnit;
        }
    } else if (!start()) {
        return false;
    }
    for (int first = begin + rounds * kAhead * kUnit; first < end; first += kUnit, j += kUnit) {
        float z[8];
        const uint32_t ok = load_chunk<T, kMask>(row, allowed, j, V, z);
        f(j, z, ok);
    }
    return true;
}

constexpr RowSums kNothing{kLowest, 0.f, 0.f};
// Half the difference of two logits, which does not overflow, and c = 2 (log2 e) / temperature that goes with it.
__device__ __forceinline__ float half_gap(float z, float r) { return __builtin_fmaf(z, 0.5f, -0.5f * r); }
__device__ __forceinline__ float exponent_scale(const Logits& q) { return 2.f * q.inv_t * kLog2E; }
// 0 * -inf would be NaN, and 2^-300 is zero
__device__ __forceinline__ float times(float p, float a) { return p * fmaxf(a, -300.f); }

// A logit above the reference becomes the reference.
__device__ __forceinline__ void move_reference(RowSums& a, float to, float c) {
    const float d = half_gap(a.r, to) * c, f = __builtin_amdgcn_exp2f(d);
    a = RowSums{to, f * a.s, f * (a.t + times(a.s, d))};
}
// kAny: also logits of -inf (excluded tokens), or so far below the reference that the exponent overflows.
template <bool kEntropy, bool kAny>
__device__ __forceinline__ void add_chunk(RowSums& a, const float (&z)[8], float c) {
    float s = 0.f, t = 0.f;              // of the chunk: what a lane adds up one by one is then an eighth as long
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = half_gap(z[e], a.r) * c;
        const float p = __builtin_amdgcn_exp2f(x), y = kAny ? fmaxf(x, -300.f) : x;
        s = e == 0 ? p : s + p;
        if (kEntropy) t = e == 0 ? p * y : __builtin_fmaf(p, y, t);
    }
    a.s += s;
    if (kEntropy) a.t += t;
}
__device__ __forceinline__ float chunk_max(const float (&z)[8]) {
    return fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(fmaxf(z[0], z[1]), z[2]), z[3]), z[4]), z[5]), z[6]), z[7]);
}
__device__ __forceinline__ RowSums join(RowSums a, RowSums b, float c) {
    if (a.r < b.r) { const RowSums x = a; a = b; b = x; }
    move_reference(b, a.r, c);
    return RowSums{a.r, a.s + b.s, a.t + b.t};
}
template <int kLanes = 64>
__device__ __forceinline__ RowSums join_lanes(RowSums a, float c) {
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) a = join(a, RowSums{__shfl_xor(a.r, d, 64), __shfl_xor(a.s, d, 64), __shfl_xor(a.t, d, 64)}, c);
    return a;
}

// Selection of the largest logits.  A token is one 64-bit number, its logit as an integer of the same order above the complement of
// its index, so that of equal logits the lower index is larger; 0 stands for none.
__device__ __forceinline__ uint64_t token_key(float z, int id) {
    const int bits = __builtin_bit_cast(int, z + 0.f);            // -0 as 0
    return (uint64_t)(uint32_t)(bits ^ ((bits >> 31) | (int)0x80000000)) << 32 | (uint32_t)~id;
}
__device__ __forceinline__ float key_logit(uint64_t key) {
    const int bits = (int)(uint32_t)(key >> 32);
    return __builtin_bit_cast(float, bits ^ (~(bits >> 31) | (int)0x80000000));
}
__device__ __forceinline__ int key_token(uint64_t key) { return (int)~(uint32_t)key; }

// The value of lane ^ kD.
template <int kD>
__device__ __forceinline__ int lane_xor(int x) {
    if constexpr (kD == 1) return __builtin_amdgcn_update_dpp(0, x, 0xB1, 0xF, 0xF, false);                 // quad_perm 1 0 3 2
    else if constexpr (kD == 2) return __builtin_amdgcn_update_dpp(0, x, 0x4E, 0xF, 0xF, false);            // quad_perm 2 3 0 1
    else if constexpr (kD == 4) return __builtin_amdgcn_update_dpp(0, __builtin_amdgcn_update_dpp(0, x, 0x141, 0xF, 0xF, false), 0x1B, 0xF, 0xF, false);
    else if constexpr (kD == 8) return __builtin_amdgcn_update_dpp(0, x, 0x128, 0xF, 0xF, false);           // row_ror 8
    else return __shfl_xor(x, kD, 64);
}
// A step of a sorting network: of lanes kD apart, the one with `larger` keeps the larger key.
template <int kD>
__device__ __forceinline__ uint64_t sort_step(uint64_t key, bool larger) {
    const uint64_t other = (uint64_t)(uint32_t)lane_xor<kD>((int)(key >> 32)) << 32 | (uint32_t)lane_xor<kD>((int)key);
    return (other > key) == larger ? other : key;
}
// Keys whose halves by lanes are sorted in opposite directions -> descending by lane (or ascending).
template <int kD>
__device__ __forceinline__ uint64_t sort_bitonic(uint64_t key, bool ascending) {
    const int lane = threadIdx.x & 63;
    key = sort_step<kD>(key, ((lane & kD) == 0) != ascending);
    if constexpr (kD > 1) return sort_bitonic<kD / 2>(key, ascending);
    else return key;
}
__device__ __forceinline__ uint64_t sort_ascending(uint64_t key) {
    const int lane = threadIdx.x & 63;
    key = sort_bitonic<1>(key, (lane & 2) == 0);
    key = sort_bitonic<2>(key, (lane & 4) == 0);
    key = sort_bitonic<4>(key, (lane & 8) == 0);
    key = sort_bitonic<8>(key, (lane & 16) == 0);
    key = sort_bitonic<16>(key, (lane & 32) == 0);
    return sort_bitonic<32>(key, true);
}

__device__ __forceinline__ uint64_t key_of_lane(uint64_t x, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, lane);
}
// The 64 largest of 64 keys descending by lane and 64 ascending ones.
__device__ __forceinline__ uint64_t merge_keys(uint64_t descending, uint64_t ascending) {
    return sort_bitonic<32>(ascending > descending ? ascending : descending, false);
}

// A row's results, by one lane; and logp of a logit.
struct RowResult {
    __device__ RowResult(const RowSums& a, const Logits& q) {
        empty = a.s == 0.f;          // nothing allowed, or only logits of -inf
        const float log2_s = __builtin_amdgcn_logf(a.s);
        r = a.r;
        scale = 2.f * q.inv_t;
        log_s = kLn2 * log2_s;
        lse = empty ? -infinity() : a.r / q.t + log_s;
        entropy = empty ? 0.f : kLn2 * (log2_s - a.t / a.s);
    }
    __device__ float logp(float z) const { return empty ? -infinity() : __builtin_fmaf(half_gap(z, r), scale, -log_s); }
    bool empty;
    float r, scale, log_s, lse, entropy;
};
template <class T>
__device__ __forceinline__ void store_row(const Logits& q, const LogprobsOut& o, int64_t row, const RowResult& res) {
    const int token = token_of(q, row);
    float logp = 0.f;
    if (token >= 0) {
        const bool in = q.allowed == nullptr || q.allowed[row * q.allowed_ld + token] != 0;
        logp = in ? res.logp(to_float<T>(static_cast<const T*>(q.z)[row * q.ld + token])) : -infinity();
    }
    o.logp[row] = logp;
    o.lse[row] = res.lse;
    if (o.entropy != nullptr) o.entropy[row] = res.entropy;
}
__device__ __forceinline__ void store_top(const LogprobsOut& o, int64_t row, uint64_t key, const RowResult& res) {
    const int lane = threadIdx.x & 63;
    if (lane >= o.top) return;
    o.top_ids[row * o.top + lane] = key != 0 ? key_token(key) : -1;
    o.top_logp[row * o.top + lane] = key != 0 ? res.logp(key_logit(key)) : -infinity();
}

// The largest chunk of every lane: its largest logit and where it is, the first of equal ones; j < 0: none yet.
struct Best {
    float z;
    int j;
    __device__ __forceinline__ void look(int at, float most, const float (&logits)[8], uint32_t ok) {
        if (most > z) {
            z = most;
            j = at;
        }
        if (__any(j < 0)) {                              // logits of -inf count, NaN does not
            bool any = false;
#pragma unroll
            for (int e = 0; e < 8; ++e) any |= (ok >> e & 1) && logits[e] == logits[e];
            if (j < 0 && any) j = at;
        }
    }
};
// The `top` largest tokens of a part of a row, in the first wavefront, descending by lane.  The pass over the logits has only noted the largest
// of every lane.  The lanes that have the `top` largest of those (of equal ones the lower chunk first) hold all that is asked for: a token of
// another lane is behind the largest of each of them.  So their logits, `top` lanes of one in kThreads, are looked at again, and those not
// below the last of the lanes' largest are sorted.  (Kept while passing over the logits, sorted lists take 40 us of 140 at 4096 x 65536.)
// What it costs: 777 rows of 32003 fp32 none / 1 / 20 / 64 alternatives 20 / 24 / 26 / 34 us, with a mask per row of half the tokens 25 / 30 / 35 / 50.
template <int kThreads>
struct TopScratch {
    uint64_t lists[kThreads / 64][64];
    // Found so far when another round, of up to kThreads * 8, is begun without sorting them.  64 / 512 / 2048: 4096 rows of 65536 bf16, 5 alternatives
    // 108 / 109 / 117 us, 64 of them 201 / 200 / 192; rows that rise, where most of what is looked at is kept, 20 of them 118 / 122 / 137.
    static constexpr int kRoom = 512;
    uint64_t found[kRoom + kThreads * 8];
    int lane_of[kTopMost];
    int lanes, n;
    float floor;
};
template <class T, bool kMask, int kThreads>
__device__ __forceinline__ uint64_t select_top(TopScratch<kThreads>& lds, const Best& best, const T* row, const uint8_t* allowed, int begin, int end, int V,
                                               int top) {
    constexpr int kWaves = kThreads / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t mine = sort_ascending(best.j < 0 ? 0 : token_key(best.z, best.j));
    if (kWaves > 1) lds.lists[wave][lane] = mine;
    __syncthreads();
    uint64_t key = 0;
    if (wave == 0) {
        key = merge_keys(0, mine);
        for (int w = 1; w < kWaves; ++w) key = merge_keys(key, lds.lists[w][lane]);
        const uint64_t last = key_of_lane(key, top - 1);
        const int lanes = __popcll(__ballot(lane < top && key != 0));
        if (lane < lanes) lds.lane_of[lane] = (key_token(key) - begin) / 8 % kThreads;
        if (lane == 0) {
            lds.lanes = lanes;
            lds.n = 0;
            lds.floor = last != 0 ? key_logit(last) : -infinity();
        }
        key = 0;
    }
    __syncthreads();
    const int chunks = ceil_div_device(end - begin, kThreads * 8), tasks = lds.lanes * chunks;
    for (int first = 0; first < tasks; first += kThreads) {
        const int task = first + (int)threadIdx.x;
        const float floor = lds.floor;
        if (task < tasks) {
            const int j = begin + (task % chunks * kThreads + lds.lane_of[task / chunks]) * 8;
            float z[8];
            const uint32_t ok = j < end ? load_chunk<T, kMask>(row, allowed, j, V, z) : 0;
            for (int e = 0; e < 8; ++e)
                if ((ok >> e & 1) && z[e] >= floor) lds.found[atomicAdd(&lds.n, 1)] = token_key(z[e], j + e);
        }
        __syncthreads();
        const int n = lds.n;
        __syncthreads();
        if (first + kThreads < tasks && n <= lds.kRoom) continue;
        if (wave == 0) {
            for (int i = 0; i < n; i += 64) key = merge_keys(key, sort_ascending(i + lane < n ? lds.found[i + lane] : 0));
            const uint64_t last = key_of_lane(key, top - 1);
            if (lane == 0) {
                lds.n = 0;
                if (last != 0) lds.floor = key_logit(last);
            }
        }
        __syncthreads();
    }
    return key;
}

// A workgroup per part of a row (a wavefront for rows of up to kWaveRow), in chunks of eight logits per lane.  Measured: 4096 rows of 65536 bf16 with
// the entropy 100 us (5.4 TB/s), with five alternatives 109; fp32 178 (6.0 TB/s).  8 rows of 131072 with eight alternatives, all latency: 8.2 us in 32
// parts and 5.1 for the launch that joins them (69 in one part).
template <class T, bool kMask, bool kEntropy, bool kTop, int kThreads>
__global__ __launch_bounds__(kThreads) void token_logprobs_parts(Logits q, LogprobsOut o, RowParts parts) {
    constexpr int kWaves = kThreads / 64;
    __shared__ RowSums wave_sums[kWaves];
    const int64_t row = blockIdx.x / parts.parts;
    const int part = blockIdx.x % parts.parts;
    const T* z_row = static_cast<const T*>(q.z) + row * q.ld;
    const uint8_t* allowed = kMask ? q.allowed + row * q.allowed_ld : nullptr;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float c = exponent_scale(q);
    RowSums a = kNothing;
    Best best{-infinity(), -1};
    bool any = kMask;                                    // of the whole wavefront: logits may be -inf
    const int units = ceil_div_device(q.V, kThreads * 8), per_part = ceil_div_device(units, parts.parts);
    const int begin = min(q.V, part * per_part * kThreads * 8), end = min(q.V, begin + per_part * kThreads * 8);
    each_chunk<T, kMask, kThreads>(z_row, allowed, begin, end, q.V, threadIdx.x, [] { return true; }, [&](int j, const float (&z)[8], uint32_t ok) __attribute__((always_inline)) {
        const float most = chunk_max(z);
        move_reference(a, fmaxf(a.r, most), c);
        if (kTop) best.look(j, most, z, ok);
        const float s = a.s, t = a.t;
        if (!any) {
            add_chunk<kEntropy, false>(a, z, c);
            if (kEntropy && __any(a.t != a.t)) {         // 0 * -inf: again, with care
                a.s = s;
                a.t = t;
                any = true;
                add_chunk<kEntropy, true>(a, z, c);
            }
        } else {
            add_chunk<kEntropy, true>(a, z, c);
        }
    });
    a = join_lanes(a, c);
    if (kWaves > 1 && lane == 0) wave_sums[wave] = a;
    uint64_t key = 0;
    if constexpr (kTop) {
        __shared__ TopScratch<kThreads> scratch;
        key = select_top<T, kMask, kThreads>(scratch, best, z_row, allowed, begin, end, q.V, o.top);
    } else if (kWaves > 1) {
        __syncthreads();
    }
    if (wave != 0) return;
    for (int w = 1; w < kWaves; ++w) a = join(a, wave_sums[w], c);
    if (parts.parts > 1) {
        if (lane == 0) parts.sums[blockIdx.x] = a;
        if (kTop && lane < o.top) parts.keys[(int64_t)blockIdx.x * o.top + lane] = key;
        return;
    }
    const RowResult res(a, q);
    if (lane == 0) store_row<T>(q, o, row, res);
    if (kTop) store_top(o, row, key, res);
}

// A workgroup per row: the parts of the row.
constexpr int kJoinThreads = 256;
template <class T>
__global__ __launch_bounds__(kJoinThreads) void token_logprobs_join(Logits q, LogprobsOut o, RowParts parts) {
    constexpr int kWaves = kJoinThreads / 64;
    __shared__ uint64_t lists[kWaves][64];
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float c = exponent_scale(q);
    uint64_t key = 0;
    if (o.top > 0) {
        const int n = parts.parts * o.top;
        for (int first = wave * 64; first < n; first += kJoinThreads)
            key = merge_keys(key, sort_ascending(first + lane < n ? parts.keys[row * n + first + lane] : 0));
        lists[wave][63 - lane] = key;
        __syncthreads();
    }
    if (wave != 0) return;
    RowSums a = kNothing;
    for (int i = lane; i < parts.parts; i += 64) a = join(a, parts.sums[row * parts.parts + i], c);
    a = join_lanes(a, c);
    const RowResult res(a, q);
    if (lane == 0) store_row<T>(q, o, row, res);
    if (o.top == 0) return;
    for (int w = 1; w < kWaves; ++w) key = merge_keys(key, lists[w][lane]);
    store_top(o, row, key, res);
}

// Rows of up to 16 kLanes logits: kLanes lanes per row, all of it in registers, and the sums relative to its largest logit.  43008 rows of 256 bf16:
// 6.9 us (22 MB; as much latency as memory), where a workgroup per row takes 55.
template <int kLanes>
__device__ __forceinline__ float lanes_max(float x) {
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
    return x;
}
template <int kLanes>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
    for (int d = kLanes / 2; d > 0; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}
constexpr int kNarrowThreads = 256;
template <class T, bool kMask, int kLanes>
__global__ __launch_bounds__(kNarrowThreads) void token_logprobs_narrow(Logits q, LogprobsOut o) {
    const int64_t row = (int64_t)blockIdx.x * (kNarrowThreads / kLanes) + threadIdx.x / kLanes;
    if (row >= q.rows) return;
    const T* z_row = static_cast<const T*>(q.z) + row * q.ld;
    const uint8_t* allowed = kMask ? q.allowed + row * q.allowed_ld : nullptr;
    const int lane = threadIdx.x % kLanes;
    const float c = exponent_scale(q);
    float z[2][8];
#pragma unroll
    for (int h = 0; h < 2; ++h) load_chunk<T, kMask>(z_row, allowed, (h * kLanes + lane) * 8, q.V, z[h]);
    RowSums a{fmaxf(lanes_max<kLanes>(fmaxf(chunk_max(z[0]), chunk_max(z[1]))), kLowest), 0.f, 0.f};
    add_chunk<true, true>(a, z[0], c);
    add_chunk<true, true>(a, z[1], c);
    a.s = lanes_sum<kLanes>(a.s);
    a.t = lanes_sum<kLanes>(a.t);
    if (lane == 0) store_row<T>(q, o, row, RowResult(a, q));
}

template <class T>
__device__ inline void store_chunk(T* row, int j, int V, const float (&g)[8]);
template <>
__device__ inline void store_chunk<float>(float* row, int j, int V, const float (&g)[8]) {
    if (j + 8 <= V) {
        *reinterpret_cast<f32x4_any*>(row + j) = f32x4_any{g[0], g[1], g[2], g[3]};
        *reinterpret_cast<f32x4_any*>(row + j + 4) = f32x4_any{g[4], g[5], g[6], g[7]};
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (j + e < V) row[j + e] = g[e];
    }
}
template <>
__device__ inline void store_chunk<uint16_t>(uint16_t* row, int j, int V, const float (&g)[8]) {
    u16x8_any b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = __builtin_bit_cast(uint16_t, (__bf16)g[e]);
    if (j + 8 <= V) {
        *reinterpret_cast<u16x8_any*>(row + j) = b;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (j + e < V) row[j + e] = b[e];
    }
}

// What a row's lse no longer tells: from kLseCarries on it is rounded by 2^-15 and more, and so is every log p taken from it (at 10^10 nothing
// is left of the log of the sum, and a token's own x / temperature may be hundreds above or below it).  Such rows, which training hardly
// has, take their sums from the logits again (all rows of 4096 x 131072 bf16 such: 730 us instead of 419; 8 rows, which are then not
// in parts, 46 instead of 6).
constexpr float kLseCarries = 1024.f;
__device__ __forceinline__ bool lse_carries(float lse) { return fabsf(lse) < kLseCarries; }          // (not where it is NaN)
// What log p is relative to: log p = (z - r) / temperature - log_s.
struct RowScale {
    float r, log_s;
};
template <int kLanes>
__device__ __forceinline__ RowScale scale_of(RowSums a, float c) {
    a = join_lanes<kLanes < 64 ? kLanes : 64>(a, c);
    if constexpr (kLanes > 64) {
        __shared__ RowSums wave_sums[kLanes / 64];
        if ((threadIdx.x & 63) == 0) wave_sums[threadIdx.x >> 6] = a;
        __syncthreads();
        a = kNothing;
        for (int w = 0; w < kLanes / 64; ++w) a = join(a, wave_sums[w], c);
    }
    return RowScale{a.r, a.s == 0.f ? -infinity() : kLn2 * __builtin_amdgcn_logf(a.s)};
}
__device__ __forceinline__ void add_moved(RowSums& a, const float (&z)[8], float c) {
    move_reference(a, fmaxf(a.r, chunk_max(z)), c);
    add_chunk<false, true>(a, z, c);
}

// The gradient of a row's logits, eight at a time.
template <class T, bool kMask>
struct RowGradient {
    RowScale of;
    int token, V;
    float dlogp, along, scale, inv_t;
    T* dz_row;
    // (the values of a row are asked for before its logits, so as not to wait for those)
    __device__ __forceinline__ RowGradient(const Logits& q, const LogprobsGradient& b, int64_t row) {
        of = RowScale{0.f, b.lse[row]};
        token = token_of(q, row);
        V = q.V;
        dz_row = static_cast<T*>(b.dz) + row * b.dz_ld;
        inv_t = q.inv_t;
        dlogp = token < 0 ? 0.f : b.dlogp[row] * q.inv_t;
        if (kMask && token >= 0 && q.allowed[row * q.allowed_ld + token] == 0) token = -1;          // its own gradient is zero
        along = 0.f;
        scale = -dlogp;                                  // g = p (scale + along a), a = log2 sqrt p
        if (b.dentropy != nullptr) {
            const float dh = b.dentropy[row] * q.inv_t;
            along = -2.f * dh * kLn2;
            scale -= dh * b.entropy[row];
        }
    }
    __device__ __forceinline__ void relative_to(RowScale scale_of_row) {
        of = scale_of_row;
        if (of.log_s == -infinity()) {                   // nothing to choose from: every p is zero
            of.log_s = infinity();
            token = -1;
        }
    }
    // kMoved: log p may be relative to a logit; with lse alone it is an instruction less.
    template <bool kMoved>
    __device__ __forceinline__ void store(int j, const float (&z)[8], uint32_t ok) const {
        float g[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float log_p = kMoved ? __builtin_fmaf(half_gap(z[e], of.r), 2.f * inv_t, -of.log_s) : __builtin_fmaf(z[e], inv_t, -of.log_s);
            const float a = log_p * (0.5f * kLog2E);
            const float root = __builtin_amdgcn_exp2f(a);            // (the instruction leaves no subnormal results, a product does)
            g[e] = kMask && !(ok >> e & 1) ? 0.f : root * root * __builtin_fmaf(along, fmaxf(a, -150.f), scale);
        }
        if (token >= j && token < j + 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) g[e] += j + e == token ? dlogp : 0.f;
        }
        store_chunk<T>(dz_row, j, V, g);
    }
};

// Rows of up to 16 kLanes logits: kLanes lanes per row, all of it in registers; 43008 rows of 256 bf16 9.3 us.  Wider ones (kLanes = 256): a workgroup
// per row, or per part of one.  Bound by memory: 4096 rows of 131072 bf16 419 us, 1111 of 50021 fp32 with a mask 86 (5.1 TB/s read and
// written, both; a large copy has 4.8).
constexpr int kGradientThreads = 256;
template <class T, bool kMask, int kLanes>
__global__ __launch_bounds__(kGradientThreads) void token_logprobs_gradient(Logits q, LogprobsGradient b, int parts) {
    const int64_t row = (int64_t)(blockIdx.x / parts) * (kGradientThreads / kLanes) + threadIdx.x / kLanes;
    if (row >= q.rows) return;
    const T* z_row = static_cast<const T*>(q.z) + row * q.ld;
    const uint8_t* allowed = kMask ? q.allowed + row * q.allowed_ld : nullptr;
    const int lane = threadIdx.x % kLanes;
    const float c = exponent_scale(q);
    RowGradient<T, kMask> gradient(q, b, row);
    if constexpr (kLanes <= 64) {
        float z[2][8];
        uint32_t ok[2];
        WholeChunk<T, kMask> whole[2];                   // both are asked for before the first is looked at
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if ((h * kLanes + lane) * 8 + 8 <= q.V) whole[h].load(z_row, allowed, (h * kLanes + lane) * 8);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int j = (h * kLanes + lane) * 8;
            ok[h] = j + 8 <= q.V ? whole[h].get(z[h]) : load_chunk<T, kMask>(z_row, allowed, j, q.V, z[h]);
        }
        if (!__any(!lse_carries(gradient.of.log_s))) {
#pragma unroll
            for (int h = 0; h < 2; ++h) gradient.template store<false>((h * kLanes + lane) * 8, z[h], ok[h]);
            return;
        }
        RowSums a = kNothing;
#pragma unroll
        for (int h = 0; h < 2; ++h) add_moved(a, z[h], c);
        const RowScale of = scale_of<kLanes>(a, c);
        if (!lse_carries(gradient.of.log_s)) gradient.relative_to(of);
#pragma unroll
        for (int h = 0; h < 2; ++h) gradient.template store<true>((h * kLanes + lane) * 8, z[h], ok[h]);
    } else {
        const int part = blockIdx.x % parts;
        const int units = ceil_div_device(q.V, kLanes * 8), per_part = ceil_div_device(units, parts);
        const int begin = min(q.V, part * per_part * kLanes * 8), end = min(q.V, begin + per_part * kLanes * 8);
        auto store = [&](int j, const float (&z)[8], uint32_t ok) __attribute__((always_inline)) { gradient.template store<false>(j, z, ok); };
        const bool done = each_chunk<T, kMask, kLanes>(z_row, allowed, begin, end, q.V, lane, [&]() __attribute__((always_inline)) { return lse_carries(gradient.of.log_s); }, store);
        // Otherwise one workgroup has the row: its logits may become the gradient, which no other part may see.
        if (done || part != 0) return;
        RowSums a = kNothing;
        for (int j = lane * 8; j < q.V; j += kLanes * 8) {
            float z[8];
            load_chunk<T, kMask>(z_row, allowed, j, q.V, z);
            add_moved(a, z, c);
        }
        gradient.relative_to(scale_of<kLanes>(a, c));
        for (int j = lane * 8; j < q.V; j += kLanes * 8) {
            float z[8];
            const uint32_t ok = load_chunk<T, kMask>(z_row, allowed, j, q.V, z);
            gradient.template store<true>(j, z, ok);
        }
    }
}

// Lanes per row: a row of up to 1024 logits has 16 of them to a lane, longer ones go through workgroups of their own.
constexpr int kNarrow = 1024;
template <class F>
void with_lanes(int V, F f) {
    if (V <= 64) f(std::integral_constant<int, 4>{});
    else if (V <= 128) f(std::integral_constant<int, 8>{});
    else if (V <= 256) f(std::integral_constant<int, 16>{});
    else if (V <= 512) f(std::integral_constant<int, 32>{});
    else f(std::integral_constant<int, 64>{});
}
// Parts of a row: as many as make `fill` workgroups of all rows, of two chunks per lane or more (one / two / four at least, eight alternatives: 8 rows of
// 131072 bf16 13.3 / 12.0 / 12.4 us, 8 of 32003 fp32 12.0 / 12.0 / 12.7; their gradients 3.3 / 3.3 / 3.9 and 3.6 / 3.6 / 4.3).  The pass over the logits is joined by another
// launch, so it stays whole where rows fill the chip (workgroups 512 / 1024 / 2048 / 4096 at most, eight alternatives: 300 rows of 50021 bf16
// 18.1 / 19.3 / 22.7 / 28.1 us, 777 of 32003 fp32 24.5 / 24.5 / 30.6 / 31.7).  The gradient has nothing to join, and short parts even out
// (2048 / 4096 / 8192 / 16384: 1111 rows of 50021 fp32 106 / 97 / 88 / 92 us, 2500 of 30000 bf16 57 / 57 / 52 / 58).
constexpr int kForwardFill = 1024, kGradientFill = 8192, kWide = 256, kWaveRow = 4096;
int row_parts(int64_t rows, int V, int fill) {
    if (V <= kWaveRow || rows < 1) return 1;
    const int64_t parts = std::min<int64_t>(fill / rows, V / (kWide * 16));
    return parts < 1 ? 1 : (int)parts;
}

template <class T, bool kMask, bool kEntropy, bool kTop>
void launch_parts(const Logits& q, const LogprobsOut& o, const RowParts& p, hipStream_t s) {
    if (q.V <= kWaveRow) token_logprobs_parts<T, kMask, kEntropy, kTop, 64><<<(unsigned)q.rows, 64, 0, s>>>(q, o, p);
    else token_logprobs_parts<T, kMask, kEntropy, kTop, kWide><<<(unsigned)(q.rows * p.parts), kWide, 0, s>>>(q, o, p);
    if (p.parts > 1) token_logprobs_join<T><<<(unsigned)q.rows, kJoinThreads, 0, s>>>(q, o, p);
}
template <class T, bool kMask>
void launch_forward(const Logits& q, const LogprobsOut& o, const RowParts& p, hipStream_t s) {
    if (q.V <= kNarrow && o.top == 0) {
        with_lanes(q.V, [&](auto lanes) {
            constexpr int kLanes = decltype(lanes)::value, kRows = kNarrowThreads / kLanes;
            token_logprobs_narrow<T, kMask, kLanes><<<(unsigned)ceil_div64(q.rows, kRows), kNarrowThreads, 0, s>>>(q, o);
        });
        return;
    }
    if (o.entropy != nullptr && o.top > 0) launch_parts<T, kMask, true, true>(q, o, p, s);
    else if (o.entropy != nullptr) launch_parts<T, kMask, true, false>(q, o, p, s);
    else if (o.top > 0) launch_parts<T, kMask, false, true>(q, o, p, s);
    else launch_parts<T, kMask, false, false>(q, o, p, s);
}
template <class T>
void launch_forward(const Logits& q, const LogprobsOut& o, const RowParts& p, hipStream_t s) {
    if (q.allowed != nullptr) launch_forward<T, true>(q, o, p, s);
    else launch_forward<T, false>(q, o, p, s);
}
template <class T, bool kMask>
void launch_backward(const Logits& q, const LogprobsGradient& b, hipStream_t s) {
    if (q.V <= kNarrow) {
        with_lanes(q.V, [&](auto lanes) {
            constexpr int kLanes = decltype(lanes)::value, kRows = kGradientThreads / kLanes;
            token_logprobs_gradient<T, kMask, kLanes><<<(unsigned)ceil_div64(q.rows, kRows), kGradientThreads, 0, s>>>(q, b, 1);
        });
        return;
    }
    const int parts = row_parts(q.rows, q.V, kGradientFill);
    token_logprobs_gradient<T, kMask, kGradientThreads><<<(unsigned)(q.rows * parts), kGradientThreads, 0, s>>>(q, b, parts);
}
template <class T>
void launch_backward(const Logits& q, const LogprobsGradient& b, hipStream_t s) {
    if (q.allowed != nullptr) launch_backward<T, true>(q, b, s);
    else launch_backward<T, false>(q, b, s);
}

RowParts carve_parts(Carver& c, int64_t rows, int V, int top) {
    RowParts p{};
    p.parts = top == 0 && V <= kNarrow ? 1 : row_parts(rows, V, kForwardFill);
    if (p.parts == 1) return p;
    p.sums = c.take<RowSums>((size_t)(rows * p.parts));
    p.keys = c.take<uint64_t>((size_t)(rows * p.parts * top));
    return p;
}

// A launch has fewer than 2^32 threads, at most kWide for a row: more rows take several launches (never of parts, which few rows have).
constexpr int64_t kRowsPerLaunch = 1 << 23;
Logits rows_from(Logits q, int64_t row, int64_t rows, int dtype) {
    q.z = static_cast<const char*>(q.z) + row * q.ld * (dtype == PCM_F32 ? 4 : 2);
    q.tokens = static_cast<const char*>(q.tokens) + row * (q.token_type == PCM_TOKEN_U8 ? 1 : q.token_type == PCM_TOKEN_I32 ? 4 : 8);
    if (q.allowed != nullptr) q.allowed += row * q.allowed_ld;
    q.rows = std::min(rows - row, kRowsPerLaunch);
    return q;
}
template <class P>
P* from(P* p, int64_t i) { return p == nullptr ? nullptr : p + i; }

constexpr int64_t kMaxRows = 0x7fffffff;
constexpr int kMaxVocabulary = 1 << 30;
constexpr float kLeastTemperature = 0x1p-126f;       // the least normal one: log2 e / temperature is finite

// The checks that both directions share.
int check_logits(const void* logits, int64_t ld, int dtype, const void* tokens, int token_type, const uint8_t* allowed, int64_t allowed_ld,
                 int64_t rows, int V, float temperature) {
    if (rows < 0 || V < 1 || ld < V || (dtype != PCM_F32 && dtype != PCM_BF16) ||
        (token_type != PCM_TOKEN_U8 && token_type != PCM_TOKEN_I32 && token_type != PCM_TOKEN_I64) ||
        (allowed != nullptr && allowed_ld != 0 && allowed_ld < V) || !(temperature >= kLeastTemperature) || temperature == __builtin_huge_valf())
        return PCM_EINVAL;
    if (rows == 0) return PCM_OK;
    const uintptr_t token_size = token_type == PCM_TOKEN_U8 ? 1 : token_type == PCM_TOKEN_I32 ? 4 : 8;
    if (!logits || !tokens || (reinterpret_cast<uintptr_t>(logits) & (dtype == PCM_F32 ? 3u : 1u)) != 0 ||
        (reinterpret_cast<uintptr_t>(tokens) & (token_size - 1)) != 0)
        return PCM_EINVAL;
    return rows > kMaxRows || V > kMaxVocabulary ? PCM_EUNSUPPORTED : PCM_OK;
}
bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

}  // namespace
}  // namespace pcm

using namespace pcm;

extern "C" {

PCM_API size_t pcm_token_logprobs_workspace_bytes(int64_t rows, int V, int top) {
    if (rows < 1 || rows > kMaxRows || V < 1 || V > kMaxVocabulary || top < 0 || top > kTopMost) return 0;
    Carver c(nullptr);
    carve_parts(c, rows, V, top);
    return c.used();
}

PCM_API int pcm_token_logprobs(const void* logits, int64_t logits_ld, int dtype, const void* tokens, int token_type,
                               const uint8_t* allowed, int64_t allowed_ld, int64_t rows, int V, float temperature, int top,
                               float* logp, float* lse, float* entropy, int32_t* top_ids, float* top_logp, void* workspace,
                               size_t workspace_bytes, void* stream) {
    const int rc = check_logits(logits, logits_ld, dtype, tokens, token_type, allowed, allowed_ld, rows, V, temperature);
    if (rc == PCM_EINVAL || top < 0 || top > kTopMost) return PCM_EINVAL;
    if (rows == 0) return PCM_OK;
    if (!logp || !lse || misaligned4(logp) || misaligned4(lse) || misaligned4(entropy)) return PCM_EINVAL;
    if (top > 0 && (!top_ids || !top_logp || misaligned4(top_ids) || misaligned4(top_logp))) return PCM_EINVAL;
    if (rc != PCM_OK) return rc;
    if (!workspace_ok(workspace, workspace_bytes, pcm_token_logprobs_workspace_bytes(rows, V, top))) return PCM_EWORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const Logits q{logits, logits_ld, allowed, allowed_ld, tokens, token_type, rows, V, temperature, 1.f / temperature};
    Carver c(workspace);
    const RowParts p = carve_parts(c, rows, V, top);
    StageTimer t(ST_TOKEN_LOGPROBS, s);
    for (int64_t row = 0; row < rows; row += kRowsPerLaunch) {
        const Logits some = rows_from(q, row, rows, dtype);
        const LogprobsOut to{logp + row, lse + row, from(entropy, row), top, from(top_ids, row * top), from(top_logp, row * top)};
        if (dtype == PCM_F32) launch_forward<float>(some, to, p, s);
        else launch_forward<uint16_t>(some, to, p, s);
    }
    return launch_status();
}

PCM_API int pcm_token_logprobs_backward(const void* logits, int64_t logits_ld, int dtype, const void* tokens, int token_type,
                                        const uint8_t* allowed, int64_t allowed_ld, int64_t rows, int V, float temperature,
                                        const float* lse, const float* dlogp, const float* entropy, const float* dentropy,
                                        void* dlogits, int64_t dlogits_ld, void* stream) {
    const int rc = check_logits(logits, logits_ld, dtype, tokens, token_type, allowed, allowed_ld, rows, V, temperature);
    if (rc == PCM_EINVAL || dlogits_ld < V || (entropy == nullptr) != (dentropy == nullptr)) return PCM_EINVAL;
    if (rows == 0) return PCM_OK;
    if (!lse || !dlogp || !dlogits || misaligned4(lse) || misaligned4(dlogp) || misaligned4(entropy) || misaligned4(dentropy) ||
        (reinterpret_cast<uintptr_t>(dlogits) & (dtype == PCM_F32 ? 3u : 1u)) != 0)
        return PCM_EINVAL;
    if (rc != PCM_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const Logits q{logits, logits_ld, allowed, allowed_ld, tokens, token_type, rows, V, temperature, 1.f / temperature};
    StageTimer t(ST_TOKEN_LOGPROBS_GRAD, s);
    for (int64_t row = 0; row < rows; row += kRowsPerLaunch) {
        const Logits some = rows_from(q, row, rows, dtype);
        const LogprobsGradient b{lse + row, dlogp + row, from(entropy, row), from(dentropy, row),
                                 static_cast<char*>(dlogits) + row * dlogits_ld * (dtype == PCM_F32 ? 4 : 2), dlogits_ld};
        if (dtype == PCM_F32) launch_backward<float>(some, b, s);
        else launch_backward<uint16_t>(some, b, s);
    }
    return launch_status();
}

}  // extern "C"
