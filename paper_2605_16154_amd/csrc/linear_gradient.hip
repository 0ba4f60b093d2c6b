// Gradient of the log-probabilities through a vocabulary projection, in the hidden rows and in the projection.
//
// Piece by piece of the vocabulary:
//   z = h W of the piece; the epilogue makes dz of it (log p = z / temperature - lse is known) and writes that, the only matrix of rows x vocabulary
//       there is, in bf16 (fp32: as a pair of fp16)
//   dhidden += dz W^T, over the piece
//   dW of the piece = h^T dz, over all rows at once, so that it is written once and rounded once
// Six operations per row, value of a row and token, all on the matrix cores.  4096 rows of 4096 -> 131072, bf16: 3.19 + 2.75 + 3.16 ms, 1.38 / 1.60 / 1.39 PFLOP/s,
// the matrix pipes 74 / 88 / 74 % busy under the power cap: a step of the main loop takes 2,235 cycles of 2,048 that the products need, at 1.5 to 1.75 GHz.
// dz is written and read twice since dhidden sums over the vocabulary and dW over the rows.
#include "linear_epilogues.h"

#include <type_traits>

namespace pcm {
namespace {

// ---- sums of parts --------------------------------------------------------------------------------------

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
#pragma unroll 16
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
// small one 0.46 (see tile_for); parts are written and read at 4.8 TB/s, in at most 256 MB.
constexpr int kMostParts = 128;
struct ProductPlan {
    int kW, parts, cost;             // parts; what one costs, in eighths of a step
    ProductPlan() : kW(kSmallTile), parts(1), cost(1) {}
    ProductPlan(int M, int N, int steps) {
        double best = 1e30;
        const int most = (int)std::min<int64_t>({kMostParts, std::max(1, steps / 8), std::max<int64_t>(1, ((int64_t)64 << 20) / ((int64_t)M * N))});
        for (const int tile : {kLargeTile, kSmallTile}) {
            if (M % (32 * tile) != 0) continue;
            const double step = tile == kLargeTile ? 0.94 : 0.46;
            const int tiles = ceil_div(M, 32 * tile) * ceil_div(N, 32 * tile), each = 1 + (int)(8 * 2.0 * M * N * 4.0 / 4.8e6 / step);
            const int n = parts_for(tiles, steps, most, each);
            const double time = step * (((tiles * n + 255) / 256) * (ceil_div(steps, n) + 10) + (n > 1 ? n * each / 8.0 + 14 : 0));
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
    int rows;                        // of the products that have them
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
    b.rows = rows <= 128 ? 128 : b.slots.padded;
    b.dh = ProductPlan(b.rows, (int)h.ld, b.dh_steps);
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
void logit_gradient(const BackwardPlan& b, const WeightSource& src, const WeightOperand& w, int first, int columns, float c, hipStream_t s) {
    BoundedProblem<kThirds> p = slot_product<kThirds>(b.slots, kRowsAreM);
    p.M = b.rows;
    set_a(p, b.slots.h, b.slots.h_low, b.slots.d64);
    set_b<kLayW>(p, w.w, w.low, w.ld, columns, src.d);
    const LogitGradient gradient{b.slots.live, b.grads.of, b.slots.token, kThirds ? b.slots.h_unit : nullptr, kThirds ? b.copy.unit : nullptr, c, first, columns};
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
    p.M = b.rows;
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
        const WeightOperand w = weight_operand(src, b.copy, first, columns, s);
        if (src.layout == PCM_WEIGHT_OUT_IN) {
            logit_gradient<kThirds, kRowsByK>(b, src, w, first, columns, c, s);
            piece_gradients<kThirds, kKByRows>(b, src, w, first, columns, out, s);
        } else {
            logit_gradient<kThirds, kKByRows>(b, src, w, first, columns, c, s);
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
    return plan_backward(nullptr, (int)rows, weight_source(weight, weight_ld, dtype, weight_layout, d, V, true)).bytes;
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
    const WeightSource src = weight_source(weight, weight_ld, dtype, weight_layout, d, V, true);
    BackwardPlan b = plan_backward(workspace, (int)rows, src);
    if (!workspace_ok(workspace, workspace_bytes, b.bytes)) return PCM_EWORKSPACE;
    const LinearRows in{hidden, hidden_ld, tokens, token_type, (int)rows, d, V};
    const float inv_t = 1.f / temperature, c = inv_t * kLog2E;
    b.grads.lse = lse; b.grads.dlogp = dlogp; b.grads.entropy = entropy; b.grads.dentropy = dentropy;
    b.grads.inv_t = inv_t;
    if (!dweight) b.grads.w_h = nullptr;
    b.grads.dh = dhidden;
    b.grads.dh_ld = dhidden_ld;
    const BackwardOut out{dhidden, dhidden_ld, dweight, dweight_ld, dweight_dtype, accumulate};
    StageTimer t(ST_LINEAR_LOGPROBS_GRAD, s);
    prepare_operands(in, b.slots, &b.grads, src, b.copy, b.columns, s);
    if (dtype == PCM_F32) backward<true>(b, src, (int)rows, c, out, s);
    else backward<false>(b, src, (int)rows, c, out, s);
    return launch_status();
}

}  // extern "C"
