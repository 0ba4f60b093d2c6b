// Orthogonalised updates: the Newton-Schulz iteration on a stack of matrices, and the optimizer step that applies it.
//
// X_0 = G / |G|_F (so no singular value exceeds one), then ns_steps times X <- P X with P = a I + b A + c A^2, A = X X^T, which
// takes every singular value s to a s + b s^3 + c s^5: what is not zero moves into [0.68, 1.21] and stays there, and the
// singular vectors are left alone.  With m the shorter side of the matrix A and P are m x m.
//
// Launches: the squares of the matrix (in 64 bits, and the momentum where there is one), the matrix divided by its norm
// in both orientations as pairs (pairs.h), then three products per step; the last one writes the result or the weights.
// Matrices of a call share the launches as long as they are small.
#include <algorithm>
#include <utility>

#include "gemm_pairs.h"
#include "orthogonalise.h"

namespace pcm {
namespace {

constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr int kMaxNsSteps = 10;
constexpr int kMaxSide = 1 << 20, kMaxShortSide = 1 << 15;
// Powers of two of the pairs: entries are at most 1.5 in X, A and B = A P (their largest singular value is), 3.5 in P and 3.5^3 in Q.
constexpr float kScaleX = 16384.f, kScaleA = 16384.f, kScaleP = 4096.f, kScaleB = 8192.f, kScaleQ = 1024.f;

constexpr int kCopyTile = 64, kCopyThreads = 256;
constexpr int kMaxParts = 1024;

// Four columns of a row of what is to be orthogonalised, from column c on; zero beyond the matrix.  write: the momentum is
// brought up to date first.
template <bool kWrite>
__device__ __forceinline__ f32x4 update_values(const UpdateMatrix& q, int r, int c) {
    f32x4 u = {0.f, 0.f, 0.f, 0.f};
    if (r >= q.rows || c >= q.cols) return u;
    const int64_t at = (int64_t)r * q.ld + c;
    const int n = min(4, q.cols - c);
    if (q.bf16) {
        const uint16_t* p = static_cast<const uint16_t*>(q.in) + at;
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (t < n) u[t] = __builtin_bit_cast(float, (uint32_t)p[t] << 16);
        return u;
    }
    const float* p = static_cast<const float*>(q.in) + at;
    f32x4 g = u;
    if (n == 4) g = *reinterpret_cast<const f32x4_any*>(p);
    else
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (t < n) g[t] = p[t];
    if (q.momentum == nullptr) return g;
    float* pm = q.momentum + at;
    f32x4 m = u;
    if (n == 4) m = *reinterpret_cast<const f32x4_any*>(pm);
    else
#pragma unroll
        for (int t = 0; t < 4; ++t)
            if (t < n) m[t] = pm[t];
    if (kWrite) {
#pragma unroll
        for (int t = 0; t < 4; ++t) m[t] = q.mu * m[t] + g[t];
        if (n == 4) *reinterpret_cast<f32x4_any*>(pm) = m;
        else
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t < n) pm[t] = m[t];
    }
    if (q.nesterov)
#pragma unroll
        for (int t = 0; t < 4; ++t) u[t] = g[t] + q.mu * m[t];
    else u = m;
    return u;
}

__device__ inline double workgroup_sum(double x, double* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    double total = 0.0;
#pragma unroll
    for (int w = 0; w < kCopyThreads / 64; ++w) total += lds[w];
    return total;
}

// Sums of squares in 64 bits (squares of large fp32 values leave the fp32 range), one per workgroup; the momentum is brought up to date on the way.
// Bound by memory: 4096 x 11008 fp32 37 us (4.9 TB/s).
__global__ __launch_bounds__(kCopyThreads) void update_squares(UpdateMatrices list) {
    __shared__ double lds[kCopyThreads / 64];
    int k = 0;
    while (k + 1 < list.n && (int)blockIdx.x >= list.m[k + 1].first_part) ++k;
    const UpdateMatrix& q = list.m[k];
    const int part = blockIdx.x - q.first_part;
    double sq = 0.0;
    for (int tile = part; tile < q.tiles; tile += q.parts) {
        const int r0 = tile / q.tiles_c * kCopyTile, c0 = tile % q.tiles_c * kCopyTile;
#pragma unroll
        for (int pass = 0; pass < 4; ++pass) {
            const f32x4 u = update_values<true>(q, r0 + pass * 16 + (threadIdx.x >> 4), c0 + (threadIdx.x & 15) * 4);
#pragma unroll
            for (int t = 0; t < 4; ++t) sq += (double)u[t] * (double)u[t];
        }
    }
    const double total = workgroup_sum(sq, lds);
    if (threadIdx.x == 0) q.partial[part] = total;
}

// The matrix divided by its norm, as pairs in both orientations: a tile of 64 x 64, 8 fragments in each.  Every workgroup adds up the sums of squares
// in the same order.  Bound by memory: 4096 x 11008 fp32 88 us (180 MB read, 361 written: 6.1 TB/s).
__global__ __launch_bounds__(kCopyThreads) void update_to_pairs(UpdateMatrices list) {
    __shared__ double lds[kCopyThreads / 64];
    __shared__ float tile[kCopyTile][kCopyTile + 1];
    int k = 0;
    while (k + 1 < list.n && (int)blockIdx.x >= list.m[k + 1].first_tile) ++k;
    const UpdateMatrix& q = list.m[k];
    const int number = blockIdx.x - q.first_tile;
    const int r0 = number / q.tiles_c * kCopyTile, c0 = number % q.tiles_c * kCopyTile;
    double sq = 0.0;
    for (int i = threadIdx.x; i < q.parts; i += kCopyThreads) sq += q.partial[i];
    const double norm = sqrt(workgroup_sum(sq, lds));
    // a matrix of zeros stays one; one that holds an infinity or a NaN becomes NaN throughout
    const double scale = norm > 0.0 ? (norm < __builtin_huge_val() ? (double)kScaleX / norm : __builtin_nan("")) : (norm == 0.0 ? 0.0 : norm);
#pragma unroll
    for (int pass = 0; pass < 4; ++pass) {
        const int r = pass * 16 + (threadIdx.x >> 4), c = (threadIdx.x & 15) * 4;
        const f32x4 u = update_values<false>(q, r0 + r, c0 + c);
#pragma unroll
        for (int t = 0; t < 4; ++t) tile[r][c + t] = (float)((double)u[t] * scale);
    }
    __syncthreads();
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, row = lane & 15;
    const int rows16 = pad32(q.rows) / 16, cols16 = pad32(q.cols) / 16;
    f16* const by_row = q.tall ? q.Xt : q.X;          // rows of the matrix as rows of the operand
    f16* const by_col = q.tall ? q.X : q.Xt;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int fr = r0 / 16 + wave, fc = c0 / 32 + h;
        if (fr < rows16 && fc * 2 < cols16) {
            f16x8 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f16 a, b;
                split_pair(tile[wave * 16 + row][h * 32 + e / 4 * 16 + 4 * g + e % 4], a, b);
                hi[e] = a; lo[e] = b;
            }
            f16* at = by_row + pair_fragment(fr, fc, rows16) + lane * 8;
            *reinterpret_cast<f16x8*>(at) = hi;
            *reinterpret_cast<f16x8*>(at + kPairPart) = lo;
        }
        const int tr = c0 / 16 + wave, tc = r0 / 32 + h;
        if (tr < cols16 && tc * 2 < rows16) {
            f16x8 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f16 a, b;
                split_pair(tile[h * 32 + e / 4 * 16 + 4 * g + e % 4][wave * 16 + row], a, b);
                hi[e] = a; lo[e] = b;
            }
            f16* at = by_col + pair_fragment(tr, tc, cols16) + lane * 8;
            *reinterpret_cast<f16x8*>(at) = hi;
            *reinterpret_cast<f16x8*>(at + kPairPart) = lo;
        }
    }
}

// A matrix of the call: where it comes from, and what becomes of it.
struct Task {
    UpdateMatrix in;
    int result;                  // PairResult
    void* out;
    uint16_t* lowp;
    int64_t out_ld;
    float decay, rate;
};

struct TaskBuffers {
    double* partial;
    f16 *X, *Xt, *Xt2, *A, *B, *P, *Q, *Q2;
};

int short_side(int rows, int cols) { return rows < cols ? rows : cols; }
int long_side(int rows, int cols) { return rows < cols ? cols : rows; }
int tiles_of(int rows, int cols) { return ceil_div(rows, kCopyTile) * ceil_div(cols, kCopyTile); }

TaskBuffers carve_task(Carver& c, int rows, int cols) {
    const int m = short_side(rows, cols), n = long_side(rows, cols);
    TaskBuffers b{};
    b.partial = c.take<double>((size_t)(tiles_of(rows, cols) < kMaxParts ? tiles_of(rows, cols) : kMaxParts));
    b.X = c.take<f16>(pair_values(m, n));
    b.Xt = c.take<f16>(pair_values(m, n));
    b.Xt2 = c.take<f16>(pair_values(m, n));
    b.A = c.take<f16>(pair_values(m, m));
    b.B = c.take<f16>(pair_values(m, m));
    b.P = c.take<f16>(pair_values(m, m));
    b.Q = c.take<f16>(pair_values(m, m));
    b.Q2 = c.take<f16>(pair_values(m, m));
    c.take<f16>(pair_values(n, 32 * kPairStepsBeyond));       // read, never used
    return b;
}
size_t task_bytes(int rows, int cols) {
    Carver c(nullptr);
    carve_task(c, rows, cols);
    return c.used();
}
// Matrices share launches while their buffers come to less than this (one alone may be larger): a bound on the workspace, which time pays for.  1 MB
// (one by one) / 64 MB / 256 MB / 1 GB: 8 of 256 x 1024 fp32 826 / 154 / 154 / 154 us, 8 of 1001 x 2815 1815 / 1815 / 1217 / 1115, 8 of 2048 x 5504
// 7411 / 7411 / 7414 / 6131, 4 of 4096 x 11008 18.5 ms whatever it is.
constexpr size_t kGroupBytes = (size_t)256 << 20;

bool shape_ok(int rows, int cols) { return rows >= 1 && cols >= 1; }
bool shape_supported(int rows, int cols) { return long_side(rows, cols) <= kMaxSide && short_side(rows, cols) <= kMaxShortSide; }

PairJob product(const f16* A, const f16* B, int m, int n, int k) {
    PairJob p{};
    p.A = A;
    p.B = B;
    p.m_frags = pad32(m) / 16;
    p.n_frags = pad32(n) / 16;
    p.steps = pad32(k) / 32;
    p.result = kPairs;
    return p;
}
PairJob symmetric_product(const f16* A, const f16* B, int m, int k, f16* C, float alpha) {
    PairJob p = product(A, B, m, m, k);
    p.symmetric = 1;
    p.C = p.Ct = C;
    p.alpha = alpha;
    return p;
}

// The products of ns_steps steps, in segments of at most `segment`: `launch` gets the jobs of one launch after the other.  A segment of one
// is the step as it is written, X <- P X.  In a longer one X stands still: every P is a polynomial of A = X X^T, so Q = P_k .. P_1 is gathered
// from m x m products and A goes on as A <- P A P, and at its end X <- Q X; all of them are symmetric.  In place of the two products over
// the long side that a step costs this has three m x m ones (A P, (A P) P, P Q).
template <class Launch>
void iterate(const Task* tasks, TaskBuffers* buf, int n, int ns_steps, int segment, f32x4* parts, Launch launch) {
    PairJobs jobs{};
    jobs.parts = parts;
    auto each = [&](auto f) {
        for (int i = 0; i < n; ++i) f(tasks[i], buf[i], short_side(tasks[i].in.rows, tasks[i].in.cols), long_side(tasks[i].in.rows, tasks[i].in.cols));
    };
    auto add = [&](const PairJob& p) { jobs.job[jobs.n++] = p; };
    auto go = [&] {
        launch(jobs);
        jobs.n = 0;
    };
    for (int done = 0; done < ns_steps;) {
        const int length = ns_steps - done < segment ? ns_steps - done : segment;
        done += length;
        each([&](const Task&, TaskBuffers& b, int m, int len) { add(symmetric_product(b.X, b.X, m, len, b.A, kScaleA / (kScaleX * kScaleX))); });
        go();
        for (int k = 0; k < length; ++k) {
            // P = a I + b A + c A^2; the first is what the segment has gathered so far
            each([&](const Task&, TaskBuffers& b, int m, int) {
                PairJob p = symmetric_product(b.A, b.A, m, m, k == 0 ? b.Q : b.P, kNsC * kScaleP / (kScaleA * kScaleA));
                p.D = b.A;
                p.beta = kNsB * kScaleP / kScaleA;
                p.gamma = kNsA * kScaleP;
                add(p);
            });
            go();
            const bool more = k + 1 < length;
            each([&](const Task&, TaskBuffers& b, int m, int) {
                if (more) add(symmetric_product(b.A, k == 0 ? b.Q : b.P, m, m, b.B, kScaleB / (kScaleA * kScaleP)));
                if (k == 0) return;
                add(symmetric_product(b.P, b.Q, m, m, b.Q2, kScaleQ / (kScaleP * (k == 1 ? kScaleP : kScaleQ))));
                std::swap(b.Q, b.Q2);
            });
            if (jobs.n > 0) go();
            if (!more) break;
            each([&](const Task&, TaskBuffers& b, int m, int) { add(symmetric_product(b.B, k == 0 ? b.Q : b.P, m, m, b.A, kScaleA / (kScaleB * kScaleP))); });
            go();
        }
        const float scale_q = length == 1 ? kScaleP : kScaleQ;
        each([&](const Task& k, TaskBuffers& b, int m, int len) {
            if (done < ns_steps) {
                PairJob p = product(b.Q, b.Xt, m, len, m);
                p.C = b.X;
                p.Ct = b.Xt2;
                p.alpha = 1.f / scale_q;
                std::swap(b.Xt, b.Xt2);
                add(p);
                return;
            }
            // in the orientation of the result
            PairJob p = k.in.tall ? product(b.Xt, b.Q, len, m, m) : product(b.Q, b.Xt, m, len, m);
            p.result = k.result;
            p.alpha = 1.f / (scale_q * kScaleX);
            p.out = k.out;
            p.lowp = k.lowp;
            p.ld = k.out_ld;
            p.rows = k.in.rows;
            p.cols = k.in.cols;
            p.decay = k.decay;
            p.rate = k.rate;
            add(p);
        });
        go();
    }
}
// Longer segments save time where the long side is long or the matrix large; but what is off in A in the directions that the matrix hardly
// has grows by 3.4445^2 a step within a segment, where in X it grows by 3.4445.  Errors on matrices like gradients in relation to those of
// fp32 products, segments of 1 / 2 / 3: short side 28 0.6 / 0.7 / 7.3, 63 0.9 / 1.1 / 5.2, 101 0.7 / 1.0 / 2.5, 195 0.5 / 0.8 / 1.6, 288 0.6 /
// 1.1 / 1.0, 651 0.5 / 0.7 / 0.8, 1164 0.5 / 0.6 / 0.7 (all five steps in one spoil the result).  So segments of three are for short sides from
// kLongSegmentSide on, where they save more than a twentieth.
constexpr int kSegment = 3, kLongSegmentSide = 256;
constexpr double kSegmentGain = 0.95;

int run_group(Task* tasks, int n, int ns_steps, void* workspace, hipStream_t s) {
    UpdateMatrices list{};
    TaskBuffers buf[kOrthGroup];
    list.n = n;
    Carver c(workspace);
    f32x4* const sums = c.take<f32x4>(kPairPartsBytes / sizeof(f32x4));
    int parts = 0, tiles = 0;
    for (int i = 0; i < n; ++i) {
        UpdateMatrix& q = tasks[i].in;
        buf[i] = carve_task(c, q.rows, q.cols);
        q.tall = q.rows > q.cols;
        q.tiles_c = ceil_div(q.cols, kCopyTile);
        q.tiles = tiles_of(q.rows, q.cols);
        q.parts = q.tiles < kMaxParts ? q.tiles : kMaxParts;
        q.first_part = parts;
        q.first_tile = tiles;
        parts += q.parts;
        tiles += q.tiles;
        q.partial = buf[i].partial;
        q.X = buf[i].X;
        q.Xt = buf[i].Xt;
        list.m[i] = q;
    }
    {
        StageTimer t(ST_ORTH_PREPARE, s);
        update_squares<<<(unsigned)parts, kCopyThreads, 0, s>>>(list);
        update_to_pairs<<<(unsigned)tiles, kCopyThreads, 0, s>>>(list);
    }
    StageTimer t(ST_ORTH_PRODUCTS, s);
    auto estimate = [&](int segment) {
        TaskBuffers b[kOrthGroup];
        for (int i = 0; i < n; ++i) b[i] = buf[i];
        double us = 0.0;
        iterate(tasks, b, n, ns_steps, segment, sums, [&](PairJobs& jobs) { us += plan_pair_products(jobs).us; });
        return us;
    };
    int shortest = kMaxShortSide;
    for (int i = 0; i < n; ++i) shortest = std::min(shortest, short_side(tasks[i].in.rows, tasks[i].in.cols));
    const int segment = shortest >= kLongSegmentSide && estimate(kSegment) < kSegmentGain * estimate(1) ? kSegment : 1;
    iterate(tasks, buf, n, ns_steps, segment, sums, [&](PairJobs& jobs) { launch_pair_products(jobs, s); });
    return launch_status();
}

// How many of the tasks from `first` on go into one group; the bytes of their buffers.
template <class Shape>
int group_length(int first, int n, Shape shape, size_t& bytes) {
    int count = 0;
    bytes = 0;
    while (count < kOrthGroup && first + count < n) {
        int rows, cols;
        shape(first + count, rows, cols);
        const size_t more = task_bytes(rows, cols);
        if (count > 0 && bytes + more > kGroupBytes) break;
        bytes += more;
        ++count;
    }
    return count;
}
template <class Shape>
size_t groups_bytes(int n, Shape shape) {
    size_t most = 0;
    for (int first = 0; first < n;) {
        size_t bytes;
        first += group_length(first, n, shape, bytes);
        most = bytes > most ? bytes : most;
    }
    return most + kPairPartsBytes;
}

bool misaligned(const void* p, unsigned by) { return (reinterpret_cast<uintptr_t>(p) & (by - 1)) != 0; }

}  // namespace
}  // namespace pcm

using namespace pcm;

extern "C" {

PCM_API size_t pcm_orthogonalise_workspace_bytes(int batch, int rows, int cols) {
    if (batch < 1 || !shape_ok(rows, cols) || !shape_supported(rows, cols)) return 0;
    const int same = batch < kOrthGroup ? batch : kOrthGroup;        // every later group is as long or shorter
    return groups_bytes(same, [&](int, int& r, int& c) { r = rows; c = cols; });
}

PCM_API int pcm_orthogonalise(const void* update, int64_t update_ld, int64_t update_stride, void* out, int64_t out_ld, int64_t out_stride,
                              int batch, int rows, int cols, int dtype, int ns_steps, void* workspace, size_t workspace_bytes,
                              void* stream) {
    if (batch < 0 || !shape_ok(rows, cols) || ns_steps < 1 || ns_steps > kMaxNsSteps || update_ld < cols || out_ld < cols ||
        (dtype != PCM_F32 && dtype != PCM_BF16))
        return PCM_EINVAL;
    if (batch == 0) return PCM_OK;
    const unsigned size = dtype == PCM_F32 ? 4 : 2;
    if (!update || !out || misaligned(update, size) || misaligned(out, size)) return PCM_EINVAL;
    if (batch > 1 && (update_stride < 0 || out_stride < (int64_t)(rows - 1) * out_ld + cols)) return PCM_EINVAL;
    if (!shape_supported(rows, cols)) return PCM_EUNSUPPORTED;
    const size_t need = pcm_orthogonalise_workspace_bytes(batch, rows, cols);
    if (!workspace_ok(workspace, workspace_bytes, need)) return PCM_EWORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto shape = [&](int, int& r, int& c) { r = rows; c = cols; };
    for (int first = 0; first < batch;) {
        size_t bytes;
        const int n = group_length(first, batch, shape, bytes);
        Task tasks[kOrthGroup] = {};
        for (int i = 0; i < n; ++i) {
            Task& t = tasks[i];
            t.in.in = static_cast<const char*>(update) + (int64_t)(first + i) * update_stride * size;
            t.in.ld = update_ld;
            t.in.rows = rows;
            t.in.cols = cols;
            t.in.bf16 = dtype == PCM_BF16;
            t.result = dtype == PCM_F32 ? kOutF32 : kOutBf16;
            t.out = static_cast<char*>(out) + (int64_t)(first + i) * out_stride * size;
            t.out_ld = out_ld;
        }
        const int rc = run_group(tasks, n, ns_steps, workspace, s);
        if (rc != PCM_OK) return rc;
        first += n;
    }
    return PCM_OK;
}

PCM_API size_t pcm_muon_step_workspace_bytes(int n_tensors, const int* rows, const int* cols) {
    if (n_tensors < 1 || n_tensors > PCM_MAX_OPT_TENSORS || rows == nullptr || cols == nullptr) return 0;
    for (int i = 0; i < n_tensors; ++i)
        if (!shape_ok(rows[i], cols[i]) || !shape_supported(rows[i], cols[i])) return 0;
    return groups_bytes(n_tensors, [&](int i, int& r, int& c) { r = rows[i]; c = cols[i]; });
}

PCM_API int pcm_muon_step(int n_tensors, const int* rows, const int* cols, const float* const* grads, float* const* weights,
                          float* const* momentum, void* const* weights_bf16, double lr, double momentum_coef, int nesterov,
                          double weight_decay, int ns_steps, int scale_rule, void* workspace, size_t workspace_bytes, void* stream) {
    if (n_tensors < 1 || n_tensors > PCM_MAX_OPT_TENSORS || !rows || !cols || !grads || !weights || !momentum) return PCM_EINVAL;
    if (!(lr >= 0.0) || !(momentum_coef >= 0.0 && momentum_coef < 1.0) || !(weight_decay >= 0.0) || ns_steps < 1 || ns_steps > kMaxNsSteps ||
        (scale_rule != PCM_MUON_SCALE_SHAPE && scale_rule != PCM_MUON_SCALE_RMS))
        return PCM_EINVAL;
    for (int i = 0; i < n_tensors; ++i) {
        if (!shape_ok(rows[i], cols[i]) || !grads[i] || !weights[i] || !momentum[i]) return PCM_EINVAL;
        if (misaligned(grads[i], 4) || misaligned(weights[i], 4) || misaligned(momentum[i], 4) ||
            (weights_bf16 && misaligned(weights_bf16[i], 2)))
            return PCM_EINVAL;
    }
    for (int i = 0; i < n_tensors; ++i)
        if (!shape_supported(rows[i], cols[i])) return PCM_EUNSUPPORTED;
    if (!workspace_ok(workspace, workspace_bytes, pcm_muon_step_workspace_bytes(n_tensors, rows, cols))) return PCM_EWORKSPACE;
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto shape = [&](int i, int& r, int& c) { r = rows[i]; c = cols[i]; };
    for (int first = 0; first < n_tensors;) {
        size_t bytes;
        const int n = group_length(first, n_tensors, shape, bytes);
        Task tasks[kOrthGroup] = {};
        for (int i = 0; i < n; ++i) {
            const int j = first + i;
            const double m = rows[j], k = cols[j];
            const double scale = scale_rule == PCM_MUON_SCALE_SHAPE ? sqrt(k > m ? k / m : 1.0) : 0.2 * sqrt(k > m ? k : m);
            Task& t = tasks[i];
            t.in.in = grads[j];
            t.in.momentum = momentum[j];
            t.in.mu = (float)momentum_coef;
            t.in.nesterov = nesterov != 0;
            t.in.ld = t.out_ld = cols[j];
            t.in.rows = rows[j];
            t.in.cols = cols[j];
            t.result = kOutWeights;
            t.out = weights[j];
            t.lowp = weights_bf16 ? static_cast<uint16_t*>(weights_bf16[j]) : nullptr;
            t.decay = (float)(1.0 - lr * weight_decay);
            t.rate = (float)(lr * scale);
        }
        const int rc = run_group(tasks, n, ns_steps, workspace, s);
        if (rc != PCM_OK) return rc;
        first += n;
    }
    return PCM_OK;
}

}  // extern "C"
