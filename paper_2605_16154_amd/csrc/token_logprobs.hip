// Log-probabilities of given tokens, entropy and the likeliest alternatives from rows of logits, and their gradient.
//
// With x = logit / temperature over the allowed tokens of a row: lse = log sum e^x, log p(token) = x_token - lse,
// entropy = lse - sum p x, and the `top` tokens of the largest logits (of equal ones the lower index).  One pass over the row:
// every lane keeps s = sum 2^a and t = sum 2^a a with a = (x - r) log2 e, relative to a logit r that it has met, so that s is at
// least one; r moves only when a logit is so far above it that s could overflow.  All sums are fp32.
//
// Gradient: d logit_j = ([j = token] d_logp - p_j (d_logp + d_entropy (log p_j + entropy))) / temperature, from lse and entropy as
// the forward pass left them: every logit is read once and its gradient written once.
#include "common.h"

namespace pcm {
namespace {

constexpr int kThreads = 256;
constexpr int kTopMost = 64;                 // one list entry per lane
constexpr float kLog2E = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

__device__ inline float infinity() { return __builtin_huge_valf(); }

struct Logits {
    const void* z;
    int64_t ld;
    const uint8_t* allowed;      // or null
    int64_t allowed_ld;          // 0: the same tokens for every row
    const void* tokens;
    int token_type;
    int64_t rows;
    int V;
    float inv_t;
};

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

__device__ inline void load_eight(const float* p, float (&z)[8]) {
    const f32x4_any a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { z[e] = a[e]; z[4 + e] = b[e]; }
}
__device__ inline void load_eight(const uint16_t* p, float (&z)[8]) {
    const u16x8_any a = *reinterpret_cast<const u16x8_any*>(p);
#pragma unroll
    for (int e = 0; e < 8; ++e) z[e] = to_float<uint16_t>(a[e]);
}
template <class T, bool kMask>
__device__ inline uint32_t load_chunk(const T* row, const uint8_t* allowed, int j, int V, float (&z)[8]) {
    uint32_t ok = 0xFF;
    if (j + 8 <= V) {
        load_eight(row + j, z);
        if (kMask) {
            const uint64_t m = *reinterpret_cast<const u64_any*>(allowed + j);
            ok = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) ok |= (uint32_t)((m >> (8 * e) & 0xFF) != 0) << e;
        }
    } else {
        ok = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool in = j + e < V && (!kMask || allowed[j + e] != 0);
            z[e] = in ? to_float<T>(row[j + e]) : -infinity();
            ok |= (uint32_t)in << e;
        }
        return ok;
    }
    if (kMask)
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = (ok >> e & 1) ? z[e] : -infinity();
    return ok;
}

// What has been seen of a row: r the reference (a logit; -inf: none yet), s = sum 2^a, t = sum 2^a a, a = (z - r) c.  (z c - r c in one
// instruction would save one of about ten, but r c rounds, and it overflows at logits of the lowest fp32 value.)
struct Sums {
    float r, s, t;
};
// How far above the reference a logit may be, in powers of two: 2^17 such terms still fit.
constexpr float kHeadroom = 64.f;

template <bool kEntropy>
__device__ __forceinline__ void add_chunk(Sums& a, const float (&z)[8], float c) {
    const float r = a.r == -infinity() ? 0.f : a.r;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = (z[e] - r) * c;
        const float p = __builtin_amdgcn_exp2f(x);
        a.s += p;
        if (kEntropy) a.t = __builtin_fmaf(p, fmaxf(x, -300.f), a.t);       // 0 * -inf would be NaN; 2^-300 is zero
    }
}
__device__ __forceinline__ float chunk_max(const float (&z)[8]) {
    return fmaxf(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])), fmaxf(fmaxf(z[4], z[5]), fmaxf(z[6], z[7])));
}
// A chunk whose largest logit is far above the reference: it becomes the reference.
__device__ __forceinline__ void move_reference(Sums& a, float to, float c) {
    if (a.r != -infinity()) {
        const float d = (a.r - to) * c, f = __builtin_amdgcn_exp2f(d);
        a.t = f * (a.t + fmaxf(d, -300.f) * a.s);
        a.s *= f;
    }
    a.r = to;
}
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, float c) {
    const float r = fmaxf(a.r, b.r);
    auto moved = [&](const Sums& x) {
        if (x.r == -infinity()) return Sums{r, x.s, x.t};            // both are zero, or NaN
        const float d = (x.r - r) * c, f = __builtin_amdgcn_exp2f(d);
        return Sums{r, f * x.s, f * (x.t + fmaxf(d, -300.f) * x.s)};
    };
    const Sums ma = moved(a), mb = moved(b);
    return Sums{r, ma.s + mb.s, ma.t + mb.t};
}

// The largest logits met by a wavefront, lane i holding the i-th of them; of equal ones the lower index first.
struct TopList {
    float z;
    int id;
    int count;                   // the same in every lane
    __device__ void clear() { z = -infinity(); id = -1; count = 0; }
    __device__ float last_z(int k) const { return __shfl(z, k - 1, 64); }
    // z, id: the same in every lane
    __device__ void insert(float nz, int nid, int k) {
        const int lane = threadIdx.x & 63;
        const bool before = lane < count && (z > nz || (z == nz && id < nid));
        const int at = __popcll(__ballot(before));
        if (at >= k) return;
        const float uz = __shfl_up(z, 1, 64);
        const int uid = __shfl_up(id, 1, 64);
        if (lane > at) { z = uz; id = uid; }
        if (lane == at) { z = nz; id = nid; }
        count = min(count + 1, k);
    }
    // Every lane's own value, where it has one: those that belong into the list.
    __device__ void offer(bool have, float nz, int nid, int k) {
        const float last = last_z(k);            // (by all lanes: a shuffle does not read from lanes that are switched off)
        uint64_t todo = __ballot(have && !(nz != nz) && (count < k || nz >= last));
        while (todo != 0) {
            const int from = __builtin_ctzll(todo);
            todo &= todo - 1;
            insert(__shfl(nz, from, 64), __shfl(nid, from, 64), k);
        }
    }
};

struct ForwardOut {
    float *logp, *lse, *entropy;     // entropy: or null
    int top;
    int32_t* top_ids;
    float* top_logp;
};

// A workgroup per row.
template <class T, bool kMask, bool kEntropy>
__global__ __launch_bounds__(kThreads) void token_logprobs_rows(Logits q, ForwardOut o) {
    constexpr int kWaves = kThreads / 64;
    __shared__ Sums wave_sums[kWaves];
    __shared__ float list_z[kWaves][kTopMost];
    __shared__ int list_id[kWaves][kTopMost];
    const int64_t row = blockIdx.x;
    const T* z_row = static_cast<const T*>(q.z) + row * q.ld;
    const uint8_t* allowed = kMask ? q.allowed + row * q.allowed_ld : nullptr;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const float c = q.inv_t * kLog2E;
    Sums a{-infinity(), 0.f, 0.f};
    TopList list;
    list.clear();
    for (int j0 = 0; j0 < q.V; j0 += kThreads * 8) {
        const int j = j0 + (int)threadIdx.x * 8;
        float z[8];
        const uint32_t ok = load_chunk<T, kMask>(z_row, allowed, j, q.V, z);
        const float most = chunk_max(z);
        if (most > a.r + kHeadroom / c) move_reference(a, most, c);
        add_chunk<kEntropy>(a, z, c);
        if (o.top > 0 && (list.count < o.top || __any(most > list.last_z(o.top)))) {
#pragma unroll
            for (int e = 0; e < 8; ++e) list.offer(ok >> e & 1, z[e], j + e, o.top);
        }
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        const Sums b{__shfl_xor(a.r, d, 64), __shfl_xor(a.s, d, 64), __shfl_xor(a.t, d, 64)};
        a = join(a, b, c);
    }
    if (lane == 0) wave_sums[wave] = a;
    if (o.top > 0) {
        list_z[wave][lane] = list.z;
        list_id[wave][lane] = list.id;
    }
    __syncthreads();
    if (wave != 0) return;
    Sums all = wave_sums[0];
    for (int w = 1; w < kWaves; ++w) all = join(all, wave_sums[w], c);
    const bool empty = all.s == 0.f;                     // nothing allowed, or only logits of -inf
    const float log2_s = __builtin_amdgcn_logf(all.s);
    auto logp_of = [&](float z) { return empty ? -infinity() : (z - all.r) * q.inv_t - kLn2 * log2_s; };
    if (lane == 0) {
        const int token = token_of(q, row);
        float logp = 0.f;
        if (token >= 0) logp = kMask && allowed[token] == 0 ? -infinity() : logp_of(to_float<T>(z_row[token]));
        o.logp[row] = logp;
        o.lse[row] = empty ? -infinity() : all.r * q.inv_t + kLn2 * log2_s;
        if (kEntropy) o.entropy[row] = empty ? 0.f : kLn2 * (log2_s - all.t / all.s);
    }
    if (o.top > 0) {
        for (int w = 1; w < kWaves; ++w) list.offer(list_id[w][lane] >= 0, list_z[w][lane], list_id[w][lane], o.top);
        if (lane < o.top) {
            o.top_ids[row * o.top + lane] = lane < list.count ? list.id : -1;
            o.top_logp[row * o.top + lane] = lane < list.count ? logp_of(list.z) : -infinity();
        }
    }
}

struct BackwardArgs {
    const float *lse, *dlogp, *entropy, *dentropy;       // the last two: both or none
    void* dz;
    int64_t dz_ld;
};

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

// A workgroup per row.
template <class T, bool kMask>
__global__ __launch_bounds__(kThreads) void token_logprobs_gradient(Logits q, BackwardArgs b) {
    const int64_t row = blockIdx.x;
    const T* z_row = static_cast<const T*>(q.z) + row * q.ld;
    T* dz_row = static_cast<T*>(b.dz) + row * b.dz_ld;
    const uint8_t* allowed = kMask ? q.allowed + row * q.allowed_ld : nullptr;
    const float lse = b.lse[row];
    const bool empty = lse == -infinity();
    const int token = empty ? -1 : token_of(q, row);
    const float dlogp = token < 0 ? 0.f : b.dlogp[row] * q.inv_t;
    float along = 0.f, scale = -dlogp;                   // g = p (scale + along a), a = log2 p
    if (b.dentropy != nullptr) {
        const float dh = b.dentropy[row] * q.inv_t;
        along = -dh * kLn2;
        scale -= dh * b.entropy[row];
    }
    for (int j = (int)threadIdx.x * 8; j < q.V; j += kThreads * 8) {
        float z[8], g[8];
        const uint32_t ok = load_chunk<T, kMask>(z_row, allowed, j, q.V, z);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float a = __builtin_fmaf(z[e], q.inv_t, -lse) * kLog2E;
            const float p = __builtin_amdgcn_exp2f(a);
            g[e] = empty || (kMask && !(ok >> e & 1)) ? 0.f : p * __builtin_fmaf(along, fmaxf(a, -300.f), scale);
            if (j + e == token && (ok >> e & 1)) g[e] += dlogp;
        }
        store_chunk<T>(dz_row, j, q.V, g);
    }
}

template <class T, bool kMask>
void launch_forward(const Logits& q, const ForwardOut& o, hipStream_t s) {
    if (o.entropy != nullptr) token_logprobs_rows<T, kMask, true><<<(unsigned)q.rows, kThreads, 0, s>>>(q, o);
    else token_logprobs_rows<T, kMask, false><<<(unsigned)q.rows, kThreads, 0, s>>>(q, o);
}
template <class T>
void launch_forward(const Logits& q, const ForwardOut& o, hipStream_t s) {
    if (q.allowed != nullptr) launch_forward<T, true>(q, o, s);
    else launch_forward<T, false>(q, o, s);
}
template <class T>
void launch_backward(const Logits& q, const BackwardArgs& b, hipStream_t s) {
    if (q.allowed != nullptr) token_logprobs_gradient<T, true><<<(unsigned)q.rows, kThreads, 0, s>>>(q, b);
    else token_logprobs_gradient<T, false><<<(unsigned)q.rows, kThreads, 0, s>>>(q, b);
}

constexpr int64_t kMaxRows = 0x7fffffff;

// The checks that both directions share.
int check_logits(const void* logits, int64_t ld, int dtype, const void* tokens, int token_type, const uint8_t* allowed, int64_t allowed_ld,
                 int64_t rows, int V, float temperature) {
    if (rows < 0 || V < 1 || ld < V || (dtype != PCM_F32 && dtype != PCM_BF16) ||
        (token_type != PCM_TOKEN_U8 && token_type != PCM_TOKEN_I32 && token_type != PCM_TOKEN_I64) ||
        (allowed != nullptr && allowed_ld != 0 && allowed_ld < V) || !(temperature > 0.f) || !(1.f / temperature < __builtin_huge_valf()) ||
        temperature == __builtin_huge_valf())
        return PCM_EINVAL;
    if (rows == 0) return PCM_OK;
    const uintptr_t token_size = token_type == PCM_TOKEN_U8 ? 1 : token_type == PCM_TOKEN_I32 ? 4 : 8;
    if (!logits || !tokens || (reinterpret_cast<uintptr_t>(logits) & (dtype == PCM_F32 ? 3u : 1u)) != 0 ||
        (reinterpret_cast<uintptr_t>(tokens) & (token_size - 1)) != 0)
        return PCM_EINVAL;
    return rows > kMaxRows ? PCM_EUNSUPPORTED : PCM_OK;
}
bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

}  // namespace
}  // namespace pcm

using namespace pcm;

extern "C" {

PCM_API size_t pcm_token_logprobs_workspace_bytes(int64_t rows, int V, int top) {
    (void)rows; (void)V; (void)top;
    return 0;
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
    const Logits q{logits, logits_ld, allowed, allowed_ld, tokens, token_type, rows, V, 1.f / temperature};
    const ForwardOut o{logp, lse, entropy, top, top_ids, top_logp};
    StageTimer t(ST_TOKEN_LOGPROBS, s);
    if (dtype == PCM_F32) launch_forward<float>(q, o, s);
    else launch_forward<uint16_t>(q, o, s);
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
    const Logits q{logits, logits_ld, allowed, allowed_ld, tokens, token_type, rows, V, 1.f / temperature};
    const BackwardArgs b{lse, dlogp, entropy, dentropy, dlogits, dlogits_ld};
    StageTimer t(ST_TOKEN_LOGPROBS_GRAD, s);
    if (dtype == PCM_F32) launch_backward<float>(q, b, s);
    else launch_backward<uint16_t>(q, b, s);
    return launch_status();
}

}  // extern "C"
