// Runs the host side of the log-probabilities through a projection and of the optimizer step over many tensors, as built in libpcm.so, on a
// HIP runtime of its own that launches nothing, so no GPU is needed or touched.  Every launch is looked at as the library issues it: what its kernels
// read and write has to lie inside the buffers that the call was given, with a workspace as long as the library's own query says, its
// grid has to cover its work, and what a launch writes may not be what it reads elsewhere.  A kernel that is not known here is a failure.
//
//   linear_path bounds   sweeps sizes and options and checks every launch
//   linear_path errors   lets each launch of a call fail in turn: the call has to return PCM_EHIP
#include <cxxabi.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "adamw_many.h"
#include "linear_epilogues.h"
#include "pcm.h"

using namespace pcm;

namespace {

struct Region {
    const char* what;
    uintptr_t begin, end;
};
std::vector<Region> regions;                           // what the call may touch
std::map<const void*, std::string>& kernel_names() {   // by host stub; the library registers its kernels before main
    static std::map<const void*, std::string> names;
    return names;
}
std::string call;                                      // the call under way
int failures = 0, launches = 0, calls = 0, products = 0, pairs = 0, in_parts = 0, pieces = 0;
int fail_at = -1;                                      // the launch that fails, or -1
bool check_bounds = false;
hipError_t last_error = hipSuccess;

void fail(const char* kernel, const char* text) {
    const std::string name = kernel;
    if (++failures <= 20) printf("%s\n  %s: %s\n", call.c_str(), name.substr(0, name.find('(', name.rfind('>') == std::string::npos ? 0 : 25)).c_str(), text);
}
void* buffer(const char* what, size_t bytes, size_t shift = 0) {
    const uintptr_t begin = (regions.empty() ? (uintptr_t)1 << 40 : (regions.back().end + (1u << 20)) / 4096 * 4096) + shift;
    regions.push_back(Region{what, begin, begin + bytes});
    return reinterpret_cast<void*>(begin);
}
struct Span {
    const char* what;
    uintptr_t begin, end;
    bool written;
};
std::vector<Span> spans;                               // of the launch under way
const char* kernel = "";
void touches(const char* what, const void* p, int64_t bytes, bool written) {
    if (bytes <= 0) return;
    const uintptr_t begin = (uintptr_t)p;
    spans.push_back(Span{what, begin, begin + (uintptr_t)bytes, written});
    for (const Region& r : regions)
        if (begin >= r.begin && begin + (uintptr_t)bytes <= r.end) return;
    char text[200];
    snprintf(text, sizeof text, "%s, %lld bytes, is not inside a buffer", what, (long long)bytes);
    fail(kernel, text);
}
void touches_rows(const char* what, const void* p, int64_t rows, int64_t columns, int64_t ld, int64_t size, bool written) {
    if (rows > 0 && columns > 0) touches(what, p, ((rows - 1) * ld + columns) * size, written);
}
// Matrices with room between their rows may lie in one another's gaps only where that is said.
void check_overlaps() {
    for (size_t a = 0; a < spans.size(); ++a)
        for (size_t b = 0; b < a; ++b) {
            const Span &p = spans[a], &q = spans[b];
            if (!(p.written || q.written) || strcmp(p.what, q.what) == 0 || p.end <= q.begin || q.end <= p.begin) continue;
            char text[200];
            snprintf(text, sizeof text, "%s and %s share memory", p.what, q.what);
            fail(kernel, text);
        }
}

// ---- the projection ------------------------------------------------------------------------------

bool has(const std::string& name, const char* what) { return name.find(what) != std::string::npos; }
void look_at_rows(const LinearRows& in, int size) {
    touches_rows("hidden", in.hidden, in.rows, in.d, in.ld, size, false);
    touches("tokens", in.tokens, (int64_t)in.rows * (in.token_type == PCM_TOKEN_U8 ? 1 : in.token_type == PCM_TOKEN_I32 ? 4 : 8), false);
}
void look_at_parts(const PartSums& p, bool written) { touches("parts of rows", p.of, p.ld * p.parts * 16, written); }

// tile: rows and columns of it.  What of B is read ends with whole pieces of 16 bytes.
template <bool kThirds>
void look_at_product(const BoundedProblem<kThirds>& p, int lay_a, int lay_b, int tile, int64_t blocks, bool exact) {
    ++products;
    if (p.M % tile || p.N % tile || p.K1 % kTileK || p.M <= 0 || p.N <= 0 || p.N < p.N_real || p.N - p.N_real >= tile || p.K1 < p.K_real || p.K1 - p.K_real >= kTileK)
        fail(kernel, "sizes that are no whole tiles");
    if (p.lda % 8 || p.ldb % 8 || ((uintptr_t)p.A | (uintptr_t)p.B) % 16) fail(kernel, "operands that are no whole pieces");
    if ((lay_b == kRowsByK ? p.K_real : p.N_real) % 8) fail(kernel, "rows of B that are no whole pieces");
    // offsets inside a step of a tile are 32 bits
    if (255 * p.lda * 2 > 0xffffffffLL || 255 * p.ldb * 2 > 0xffffffffLL) fail(kernel, "rows too far apart");
    if (p.kept_max < 0 || p.rows_per_kept != 1 || p.splits < 1) fail(kernel, "rows or parts that make no sense");
    touches("live", p.kept, 4, false);
    const bf16 *a[] = {p.A, p.A2, p.A3}, *b[] = {p.B, p.B2, p.B3};
    for (int segment = 0; segment < (kThirds ? 3 : 1); ++segment) {
        touches_rows("A", a[segment], lay_a == kRowsByK ? p.M : p.K1, lay_a == kRowsByK ? p.K1 : p.M, p.lda, 2, false);
        touches_rows("B", b[segment], lay_b == kRowsByK ? p.N_real : p.K_real, lay_b == kRowsByK ? p.K_real : p.N_real, p.ldb, 2, false);
    }
    if (!kThirds && (p.A2 != p.A || p.B2 != p.B)) fail(kernel, "a segment that is not there");
    const int64_t tiles = (int64_t)(p.M / tile) * (p.N / tile);
    int64_t need = tiles * p.splits;
    if (p.part_cost > 0) {
        ++in_parts;
        need = 0;
        for (int rows = 1; rows <= p.kept_max; rows += kTileM) {
            const int n = std::min(p.M / tile, (rows + kTileM - 1) / kTileM * (kTileM / tile)) * (p.N / tile);
            need = std::max<int64_t>(need, (int64_t)part_workgroups(n) * parts_for(n, p.part_steps, p.splits, p.part_cost));
        }
    }
    if (exact ? blocks != need : blocks < need) fail(kernel, "a grid that does not fit the product");
}
void look_at_epilogue(const EpiRowStats& e, int M, int N, int tile) {
    const int first = e.first_part, last = first + ceil_div(e.columns, tile / 2);
    if (last > e.out.parts) fail(kernel, "more parts than there is room for");
    look_at_parts(e.out, true);
    if (e.out.ld < M) fail(kernel, "more rows than there is room for");
    touches("logits of tokens", e.token_z, (int64_t)M * 4, true);
    touches("tokens of slots", e.token, (int64_t)M * 4, false);
    if (e.h_unit) touches("units", e.h_unit, (int64_t)M * 4, false), touches("unit of W", e.w_unit, 4, false);
    if (e.columns > N) fail(kernel, "more columns than the product has");
}
void look_at_gradient(const LogitGradient& g, int M) {
    touches("gradients of slots", g.of, (int64_t)M * sizeof(SlotGradient), false);
    touches("tokens of slots", g.token, (int64_t)M * 4, false);
    if (g.h_unit) touches("units", g.h_unit, (int64_t)M * 4, false), touches("unit of W", g.w_unit, 4, false);
}
void look_at_epilogue(const EpiLogitGradient& e, int M, int N, int) {
    look_at_gradient(e.gradient, M);
    touches_rows("dz", e.dz, M, N, e.ld, 2, true);
}
void look_at_epilogue(const EpiLogitGradientPairs& e, int M, int N, int) {
    look_at_gradient(e.gradient, M);
    touches_rows("dz", e.hi, M, N, e.ld, 2, true);
    touches_rows("dz, low parts", e.lo, M, N, e.ld, 2, true);
}
int rows_of_call = 0, splits_of_product = 1;
template <class T>
void look_at_epilogue(const EpiHidden<T>& e, int M, int N, int) {
    touches("the number of parts", e.parts.used, 4, true);
    if (e.parts.of != nullptr) {
        if (e.parts.ld < N) fail(kernel, "parts narrower than the product");
        touches("parts of dhidden", e.parts.of, ((splits_of_product - 1) * e.parts.part + (int64_t)(M - 1) * e.parts.ld + N) * 4, true);
    } else if (splits_of_product != 1 || !e.whole) {
        fail(kernel, "parts without room");
    }
    if (e.whole) {
        touches_rows("dhidden", e.out, rows_of_call, e.cols, e.ld, sizeof(T), true);
        touches("rows of slots", e.row_of, (int64_t)rows_of_call * 4, false);
    }
    if (e.z_shift) touches("shifts", e.z_shift, (int64_t)M * 4, false), touches("unit of W", e.w_unit, 4, false);
}
template <class T>
void look_at_epilogue(const EpiStoreAnywhere<T>& e, int M, int N, int) {
    if (e.rows > M || e.cols > N) fail(kernel, "a result larger than the product");
    touches_rows("dweight", e.C, e.rows, e.cols, e.ldc, sizeof(T), true);
}
void look_at_epilogue(const EpiStoreF32& e, int M, int N, int) {
    if (e.ldc < N) fail(kernel, "parts narrower than the product");
    touches("parts of dweight", e.C, ((splits_of_product - 1) * e.split_stride + (int64_t)(M - 1) * e.ldc + N) * 4, true);
}
template <class E, bool kThirds>
void look_at_tile(void* problem, void* epilogue, int lay_a, int lay_b, int tile, int64_t blocks, bool exact) {
    const auto& p = *static_cast<BoundedProblem<kThirds>*>(problem);
    splits_of_product = p.splits;
    look_at_product(p, lay_a, lay_b, tile, blocks, exact);
    look_at_epilogue(*static_cast<E*>(epilogue), p.M, p.N, tile);
}
// The product that a name begins at `at` with "<problem, epilogue, layouts ..": dispatch by its epilogue.
void look_at_named(const std::string& e, bool thirds, void* problem, void* epilogue, int lay_a, int lay_b, int tile, int64_t blocks, bool exact) {
#define PCM_CASE(text, type)                                                                                                           \
    if (e == text) {                                                                                                                   \
        if (thirds) return look_at_tile<type, true>(problem, epilogue, lay_a, lay_b, tile, blocks, exact);                             \
        return look_at_tile<type, false>(problem, epilogue, lay_a, lay_b, tile, blocks, exact);                                        \
    }
    PCM_CASE("EpiRowStats", EpiRowStats)
    PCM_CASE("EpiLogitGradient", EpiLogitGradient)
    PCM_CASE("EpiLogitGradientPairs", EpiLogitGradientPairs)
    PCM_CASE("EpiHidden<float>", EpiHidden<float>)
    PCM_CASE("EpiHidden<unsigned short>", EpiHidden<uint16_t>)
    PCM_CASE("EpiStoreAnywhere<float>", EpiStoreAnywhere<float>)
    PCM_CASE("EpiStoreAnywhere<unsigned short>", EpiStoreAnywhere<uint16_t>)
    PCM_CASE("EpiStoreF32", EpiStoreF32)
#undef PCM_CASE
    fail(kernel, "an epilogue that this program does not know");
}
std::string without_spaces(std::string name) {
    for (const char* drop : {"pcm::", "(anonymous namespace)::"})
        for (size_t at; (at = name.find(drop)) != std::string::npos;) name.erase(at, strlen(drop));
    return name;
}
// "a, b<c, d>, e" -> its parts
std::vector<std::string> arguments(const std::string& list) {
    std::vector<std::string> out(1);
    int depth = 0;
    for (char c : list) {
        if (c == '<') ++depth;
        if (c == '>') --depth;
        if (c == ',' && depth == 0) out.emplace_back();
        else if (c != ' ' || !out.back().empty()) out.back() += c;
    }
    for (std::string& x : out)
        while (!x.empty() && x.back() == ' ') x.pop_back();
    return out;
}
std::string inside_angles(const std::string& name) {
    const size_t begin = name.find('<');
    int depth = 0;
    for (size_t i = begin; i < name.size(); ++i) {
        if (name[i] == '<') ++depth;
        if (name[i] == '>' && --depth == 0) return name.substr(begin + 1, i - begin - 1);
    }
    return "";
}
void look_at_grads(const SlotGradients& g, const Slots& s, int rows) {
    for (const float* p : {g.lse, g.dlogp, g.entropy, g.dentropy})
        if (p != nullptr) touches("a value per row", p, (int64_t)rows * 4, false);
    touches("gradients of slots", g.of, (int64_t)s.padded * sizeof(SlotGradient), true);
}
void look_at_slots(const Slots& s, int rows, bool thirds, bool units) {
    const int64_t h = (int64_t)s.padded * s.d64 * 2;
    if (s.padded < rows || s.padded % kTileM || s.d64 % kTileK) fail(kernel, "slots that do not hold the rows");
    touches("slots of rows", s.slot_of, (int64_t)rows * 4, true);
    touches("rows of slots", s.row_of, (int64_t)s.padded * 4, true);
    touches("tokens of slots", s.token, (int64_t)s.padded * 4, true);
    if (!units) return;
    touches("h", s.h, h, true);
    if (thirds) touches("h, low parts", s.h_low, h, true), touches("units", s.h_unit, (int64_t)s.padded * 4, true);
}

void look_at_split(const RowSplit& s, int rows, int64_t cols, int each) {
    if (s.lanes < 0 || s.lanes > 8 || ((int64_t)each * s.chunks << s.lanes) < cols || (int64_t)s.blocks / s.chunks * (256 >> s.lanes) < rows || s.blocks % s.chunks)
        fail(kernel, "a split that does not cover the rows");
}
void look_at_piece(const WeightPiece& p, bool floats, int64_t blocks) {
    if (p.w == nullptr) {
        if (blocks != 0 || floats) fail(kernel, "a copy of nothing");
        return;
    }
    ++pieces;
    touches_rows("weight", p.w, p.rows, p.cols, p.ld, floats ? 4 : 2, false);
    touches("the copy", p.to, p.rows * p.ld_to * 2, true);
    if (floats) {
        touches("the copy, low parts", p.low, p.rows * p.ld_to * 2, true);
        touches("unit of W", p.unit, 4, true);
        touches("largest values", p.absmax, (int64_t)p.absmax_parts * 4, false);
    }
    look_at_split(p.split, p.rows, p.ld_to, 8);
    if (p.ld_to < p.cols || p.ld_to % 8 || blocks != p.split.blocks) fail(kernel, "a grid that does not fit the copy");
}
void look_at_launch(const std::string& raw, void** args, dim3 grid) {
    std::string name = without_spaces(raw);
    const size_t ends = name.find('<') < name.find('(') ? name.find(inside_angles(name)) + inside_angles(name).size() + 1 : name.find('(');
    name = name.substr(0, ends);                       // without the types of its arguments
    const int64_t threads = (int64_t)grid.x * 256;
    if (has(name, "gemm_bounded_pair<")) {
        ++pairs;
        const std::vector<std::string> jobs = arguments(inside_angles(name));
        const int first = *static_cast<int*>(args[2]);
        if (first % kNumXcd || first <= 0 || first >= (int)grid.x) fail(kernel, "workgroups that do not follow one another");
        for (int job = 0; job < 2; ++job) {
            const std::vector<std::string> a = arguments(inside_angles(jobs[job]));      // SlotProduct<thirds, layout, layout, epilogue>
            look_at_named(a[3], a[0] == "true", args[job ? 3 : 0], args[job ? 4 : 1], atoi(a[1].c_str()), atoi(a[2].c_str()), 32 * kSmallTile,
                          job ? grid.x - first : first, job == 1);
        }
    } else if (has(name, "gemm_bounded<")) {
        const std::vector<std::string> a = arguments(inside_angles(name));               // problem, epilogue, layouts, kW, slots
        look_at_named(a[1], has(a[0], "true"), args[0], args[1], atoi(a[2].c_str()), atoi(a[3].c_str()), 32 * atoi(a[4].c_str()), grid.x, true);
    } else if (has(name, "linear_counts")) {
        const LinearRows& in = *static_cast<LinearRows*>(args[0]);
        touches("tokens", in.tokens, (int64_t)in.rows * (in.token_type == PCM_TOKEN_U8 ? 1 : in.token_type == PCM_TOKEN_I32 ? 4 : 8), false);
        touches("counts", *static_cast<int32_t**>(args[1]), (int64_t)grid.x * 4, true);
        if ((int64_t)grid.x * kCountRows < in.rows) fail(kernel, "a grid that does not fit the rows");
    } else if (has(name, "linear_slots")) {
        const LinearRows& in = *static_cast<LinearRows*>(args[0]);
        const Slots& s = *static_cast<Slots*>(args[1]);
        touches("live", s.live, 4, true);
        touches("shares of the exponent", s.mosts, kMosts * kMostPitch * 4, true);
        look_at_slots(s, in.rows, false, false);
        if (s.counts) touches("counts", s.counts, (int64_t)grid.x * 4, false);
        if ((int64_t)grid.x * kCountRows < in.rows) fail(kernel, "a grid that does not fit the rows");
    } else if (has(name, "linear_gather<") || has(name, "linear_weigh")) {
        const LinearRows& in = *static_cast<LinearRows*>(args[0]);
        const Slots& s = *static_cast<Slots*>(args[1]);
        const SlotGradients& g = *static_cast<SlotGradients*>(args[2]);
        const int rows_blocks = *static_cast<int*>(args[3]);
        const bool weighs = has(name, "linear_weigh"), thirds = has(name, "float") || weighs;
        look_at_rows(in, thirds ? 4 : 2);
        touches("live", s.live, 4, !weighs);
        if (weighs) {
            touches("weighted h", g.w_h, (int64_t)s.padded * s.d64 * 2, true);
            touches("weighted h, low parts", g.w_h_low, (int64_t)s.padded * s.d64 * 2, true);
            touches("shifts", g.z_shift, (int64_t)s.padded * 4, false);
            touches("exponents", g.exponent, (int64_t)s.padded * 4, false);
            touches("the exponent", s.most, 4, true);
            if (s.counts) touches("shares of the exponent", s.mosts, kMosts * kMostPitch * 4, false);
            look_at_piece(*static_cast<WeightPiece*>(args[4]), true, grid.x - rows_blocks);
        } else {
            look_at_slots(s, in.rows, thirds, true);
            if (g.of) look_at_grads(g, s, in.rows);
            if (g.of && thirds) touches("shifts", g.z_shift, (int64_t)s.padded * 4, true), touches("exponents", g.exponent, (int64_t)s.padded * 4, true);
            if (g.of && thirds && s.counts) touches("shares of the exponent", s.mosts, kMosts * kMostPitch * 4, true);
            if (g.dh) touches_rows("dhidden", g.dh, in.rows, in.d, g.dh_ld, thirds ? 4 : 2, true);
            rows_of_call = in.rows;
            if (has(name, "true") != (s.counts == nullptr)) fail(kernel, "a list in the wrong place");
            if (thirds) {
                const WeightAbsmax& a = *static_cast<WeightAbsmax*>(args[4]);
                touches_rows("weight", a.w, a.rows, a.cols, a.ld, 4, false);
                touches("largest values", a.out, (int64_t)a.parts * 4, true);
                look_at_split(a.split, a.rows, ((int64_t)a.cols + 3) / 4, 4);
                if (a.parts < 1 || a.parts > kAbsmaxParts || a.parts != (int)grid.x - rows_blocks) fail(kernel, "a grid that does not fit the weight");
            } else {
                look_at_piece(*static_cast<WeightPiece*>(args[5]), false, grid.x - rows_blocks);
            }
        }
        if ((int64_t)rows_blocks * 4 < in.rows + kTileM) fail(kernel, "a grid that does not fit the rows");
    } else if (has(name, "linear_copy<")) {
        look_at_piece(*static_cast<WeightPiece*>(args[0]), has(name, "float"), grid.x);
    } else if (has(name, "few_rows<")) {
        const LinearRows& in = *static_cast<LinearRows*>(args[0]);
        const PartSums& p = *static_cast<PartSums*>(args[3]);
        const bool floats = has(name, "float"), by_token = has(name, ", 1>");
        look_at_rows(in, floats ? 4 : 2);
        touches_rows("weight", *static_cast<void**>(args[1]), by_token ? in.V : in.d, by_token ? in.d : in.V, *static_cast<int64_t*>(args[2]), floats ? 4 : 2, false);
        look_at_parts(p, true);
        touches("logits of tokens", *static_cast<float**>(args[4]), (int64_t)in.rows * 4, true);
        const int groups = *static_cast<int*>(args[6]), blocks = groups == 1 ? (int)grid.x : (int)grid.x / groups;
        if (groups * kFewRows < in.rows || p.ld < in.rows || p.parts > blocks || (int64_t)p.parts * (by_token || floats ? 64 : 128) < in.V || (groups > 1 && blocks % kNumXcd) ||
            grid.x % groups)
            fail(kernel, "a grid that does not fit the rows and columns");
    } else if (has(name, "linear_join<")) {
        const LinearRows& in = *static_cast<LinearRows*>(args[0]);
        const int32_t* slot_of = *static_cast<int32_t**>(args[1]);
        look_at_parts(*static_cast<PartSums*>(args[2]), false);
        if (slot_of) touches("slots of rows", slot_of, (int64_t)in.rows * 4, false);
        const RowResults& o = *static_cast<RowResults*>(args[5]);
        touches("logp", o.logp, (int64_t)in.rows * 4, true);
        touches("lse", o.lse, (int64_t)in.rows * 4, true);
        if (o.entropy) touches("entropy", o.entropy, (int64_t)in.rows * 4, true);
        if ((int64_t)grid.x * (has(name, "<4>") ? 4 : 1) < in.rows) fail(kernel, "a grid that does not fit the rows");
    } else if (has(name, "linear_sum_parts<")) {
        const PartSum& q = *static_cast<PartSum*>(args[0]);
        const int64_t size = has(name, "float") ? 4 : 2;
        touches_rows(q.slot_of ? "dhidden" : "dweight", *static_cast<void**>(args[1]), q.rows, q.cols, *static_cast<int64_t*>(args[2]), size, true);
        if (q.slot_of) touches("slots of rows", q.slot_of, (int64_t)q.rows * 4, false), touches("the number of parts", q.used, 4, false);
        else if (q.n > 0) touches("parts of dweight", q.parts, ((q.n - 1) * q.part + (q.rows - 1) * q.ld + round_up(q.cols, 4)) * 4, false);
        if (q.slot_of || q.n > 0) if (q.ld < round_up(q.cols, 4) || q.ld % 4) fail(kernel, "parts narrower than what is read");
        if ((int64_t)grid.x * 1024 < q.cols || ((int64_t)(grid.y - 1) * 65535 + grid.z) * q.rows_each < q.rows) fail(kernel, "a grid that does not fit the result");
    } else if (has(name, "many_sumsq")) {
        touches("the plan", *static_cast<void**>(args[0]), *static_cast<int64_t*>(args[1]) * (int64_t)sizeof(AdamwChunk), false);
        touches("partial sums", *static_cast<void**>(args[2]), (int64_t)grid.x * 8, true);
    } else if (has(name, "many_update<")) {
        const ManyStep& s = *static_cast<ManyStep*>(args[0]);
        touches("the plan", s.chunks, s.n * (int64_t)sizeof(AdamwChunk), false);
        if (s.elements) touches("the state", s.state, has(name, "<32") ? s.elements * 8 : s.elements * 2 + s.elements / kManyBlock * 2, true);
        if (s.parts) touches("partial sums", s.partial, (int64_t)s.parts * 8, false);
        if (s.norm_out) touches("norm", s.norm_out, 4, true);
        if (s.parts > 1024) fail(kernel, "more partial sums than are added up");
    } else if (has(name, "many_states<")) {
        const int64_t E = *static_cast<int64_t*>(args[1]), size = has(name, "true") ? 2 : 4;
        touches("the state", *static_cast<void**>(args[0]), E * 2 + E / kManyBlock * 2, false);
        touches("m", *static_cast<void**>(args[2]), E * size, true);
        touches("v", *static_cast<void**>(args[3]), E * size, true);
    } else {
        fail(kernel, "a launch that this program does not know");
    }
    if (threads <= 0) fail(kernel, "an empty grid");
}

}  // namespace

// ---- the runtime -------------------------------------------------------------------------------
extern "C" {
struct CallConfiguration { dim3 grid, block; size_t shared; hipStream_t stream; };
static CallConfiguration configuration;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, hipStream_t stream) {
    configuration = CallConfiguration{grid, block, shared, stream};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, hipStream_t* stream) {
    *grid = configuration.grid; *block = configuration.block; *shared = configuration.shared; *stream = configuration.stream;
    return hipSuccess;
}
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void* stub, char*, const char* name, unsigned, void*, void*, dim3*, dim3*, int*) {
    int status = 0;
    char* const text = abi::__cxa_demangle(name, nullptr, nullptr, &status);
    kernel_names()[stub] = text ? text : name;
    free(text);
}
void __hipRegisterVar(void**, void*, char*, char*, int, size_t, int, int) {}
hipError_t hipLaunchKernel(const void* stub, dim3 grid, dim3 block, void** args, size_t, hipStream_t) {
    if (launches++ == fail_at) return last_error = hipErrorLaunchFailure;
    if (check_bounds) {
        const std::string& name = kernel_names()[stub];
        kernel = name.c_str();
        if (grid.x == 0 || grid.y == 0 || grid.z == 0 || grid.y > 65535 || grid.z > 65535 || block.x * block.y * block.z > 1024 || (uint64_t)grid.x * block.x >> 32)
            fail(kernel, "an empty or too large grid");
        spans.clear();
        look_at_launch(name, args, grid);
        check_overlaps();
    }
    return hipSuccess;
}
hipError_t hipGetLastError() {
    const hipError_t e = last_error;
    last_error = hipSuccess;
    return e;
}
hipError_t hipGetDevice(int* device) { *device = 0; return hipSuccess; }
hipError_t hipGetSymbolAddress(void**, const void*) { return hipErrorInvalidSymbol; }
hipError_t hipEventCreate(hipEvent_t*) { return hipErrorInvalidValue; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipErrorInvalidValue; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipErrorInvalidValue; }
hipError_t hipEventElapsedTime(float*, hipEvent_t, hipEvent_t) { return hipErrorInvalidValue; }
}

namespace {

void begin(const std::string& text) {
    call = text;
    regions.clear();
    launches = 0;
    last_error = hipSuccess;
    ++calls;
}
void expect(int rc, int want) {
    if (rc == want) return;
    char text[60];
    snprintf(text, sizeof text, "returned %d, not %d", rc, want);
    fail("the call", text);
}

struct Linear {
    int64_t rows;
    int d, V, dtype, layout, token_type, pad, shift;       // shift: bytes that the weight lies off a multiple of 16
    bool entropy;
    int dw_dtype, want;                                    // want: 1 dhidden, 2 dweight, 3 both
    std::string text(const char* what) const {
        char t[200];
        snprintf(t, sizeof t, "%s, %lld rows of %d -> %d, type %d, layout %d, pad %d, shift %d, entropy %d, dweight %d, want %d", what, (long long)rows, d, V, dtype, layout,
                 pad, shift, entropy, dw_dtype, want);
        return t;
    }
    int64_t size() const { return dtype == PCM_F32 ? 4 : 2; }
    int64_t ld() const { return (layout ? d : V) + pad; }
    int64_t matrix(int64_t rows_, int64_t cols, int64_t ld_) const { return (rows_ - 1) * ld_ + cols; }
    void* weight(const char* what, int64_t each, int shift_) const { return buffer(what, (layout ? matrix(V, d, ld()) : matrix(d, V, ld())) * each, shift_); }
};
int forward(const Linear& c) {
    begin(c.text("log-probabilities"));
    void* h = buffer("hidden", c.matrix(c.rows, c.d, c.d + c.pad) * c.size());
    void* w = c.weight("weight", c.size(), c.shift);
    void* tokens = buffer("tokens", c.rows * (c.token_type == PCM_TOKEN_U8 ? 1 : c.token_type == PCM_TOKEN_I32 ? 4 : 8));
    float *logp = (float*)buffer("logp", c.rows * 4), *lse = (float*)buffer("lse", c.rows * 4), *entropy = c.entropy ? (float*)buffer("entropy", c.rows * 4) : nullptr;
    const size_t bytes = pcm_linear_logprobs_workspace_bytes(c.rows, c.d, c.V, c.dtype, c.layout, w, c.ld());
    if (bytes == 0 && c.rows <= 1 << 24) fail("the query", "no workspace");
    void* ws = buffer("workspace", bytes);
    return pcm_linear_logprobs(h, c.d + c.pad, w, c.ld(), c.layout, c.dtype, tokens, c.token_type, c.rows, c.d, c.V, 0.7f, logp, lse, entropy, ws, bytes, nullptr);
}
int backward(const Linear& c) {
    begin(c.text("gradient"));
    void* h = buffer("hidden", c.matrix(c.rows, c.d, c.d + c.pad) * c.size());
    void* w = c.weight("weight", c.size(), c.shift);
    void* tokens = buffer("tokens", c.rows * (c.token_type == PCM_TOKEN_U8 ? 1 : c.token_type == PCM_TOKEN_I32 ? 4 : 8));
    float *lse = (float*)buffer("lse", c.rows * 4), *dlogp = (float*)buffer("dlogp", c.rows * 4);
    float *entropy = c.entropy ? (float*)buffer("entropy", c.rows * 4) : nullptr, *dentropy = c.entropy ? (float*)buffer("dentropy", c.rows * 4) : nullptr;
    void* dh = c.want & 1 ? buffer("dhidden", c.matrix(c.rows, c.d, c.d + c.pad) * c.size(), c.size()) : nullptr;
    void* dw = c.want & 2 ? c.weight("dweight", c.dw_dtype == PCM_F32 ? 4 : 2, c.dw_dtype == PCM_F32 ? 4 : 2) : nullptr;
    const size_t bytes = pcm_linear_logprobs_backward_workspace_bytes(c.rows, c.d, c.V, c.dtype, c.layout, w, c.ld());
    if (bytes == 0 && c.rows <= 1 << 24) fail("the query", "no workspace");
    void* ws = buffer("workspace", bytes);
    return pcm_linear_logprobs_backward(h, c.d + c.pad, w, c.ld(), c.layout, c.dtype, tokens, c.token_type, c.rows, c.d, c.V, 0.7f, lse, dlogp, entropy, dentropy, dh,
                                        c.d + c.pad, dw, c.ld(), c.dw_dtype, 0, ws, bytes, nullptr);
}
int optimizer(const std::vector<int64_t>& numel, int bits, bool clip, bool states) {
    begin("optimizer step");
    pcm_adamw_many_layout l;
    expect(pcm_adamw_many_describe((int)numel.size(), numel.data(), bits, &l), PCM_OK);
    void* plan = buffer("plan", l.plan_bytes);
    void* state = buffer("state", l.state_bytes);
    if (states) return pcm_adamw_many_states(&l, state, PCM_BF16, buffer("m", l.elements * 2), buffer("v", l.elements * 2), nullptr);
    const size_t bytes = pcm_adamw_many_step_workspace_bytes(&l);
    void* ws = buffer("workspace", bytes);
    float* norm = clip ? (float*)buffer("norm", 4) : nullptr;
    return pcm_adamw_many_step(plan, &l, state, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, clip ? 1.0 : __builtin_huge_val(), 1, norm, clip ? ws : nullptr, clip ? bytes : 0, nullptr);
}

void bounds() {
    check_bounds = true;
    const int sides[] = {1, 2, 7, 8, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513, 1000, 1536, 4096};
    const int vocabularies[] = {1, 2, 7, 8, 64, 65, 128, 129, 255, 256, 257, 1000, 1024, 5000, 32003, 50021, 131072};
    int turn = 0;
    for (int64_t rows : {1, 2, 15, 16, 17, 64, 127, 128, 129, 255, 256, 257, 777, 1111, 4096, 4097, 43008})
        for (int d : sides)
            for (int V : vocabularies)
                for (int dtype : {PCM_F32, PCM_BF16})
                    for (int layout = 0; layout < 2; ++layout) {
                        ++turn;
                        const Linear c{rows, d, V, dtype, layout, turn % 3, (int)(turn / 3 % 4 == 0 ? 0 : turn / 3 % 4 == 1 ? 1 : 8), turn % 5 == 0 ? (dtype == PCM_F32 ? 4 : 2) : 0,
                                       turn % 2 == 0, dtype == PCM_F32 || turn % 3 == 0 ? PCM_F32 : PCM_BF16, turn % 4 == 0 ? 1 : turn % 4 == 1 ? 2 : 3};
                        expect(forward(c), PCM_OK);
                        expect(backward(c), PCM_OK);
                    }
    // rows of the weight far apart
    for (int layout = 0; layout < 2; ++layout)
        for (int pad : {(1 << 22), (1 << 23) - 1000 - 8, (1 << 23) - 1000, 1 << 27})
            for (int dtype : {PCM_F32, PCM_BF16}) {
                const Linear c{300, 1000, 1000, dtype, layout, 1, pad, 0, true, dtype, 3};
                expect(forward(c), PCM_OK);
                expect(backward(c), PCM_OK);
            }
    // the largest sizes, and many pieces
    for (int layout = 0; layout < 2; ++layout)
        for (int dtype : {PCM_F32, PCM_BF16})
            for (const Linear& c : {Linear{1 << 24, 64, 1 << 14, dtype, layout, 1, 0, 0, true, PCM_F32, 3}, Linear{300, 1 << 16, 1 << 16, dtype, layout, 1, 1, 0, true, PCM_F32, 3},
                                    Linear{300, 256, 1 << 22, dtype, layout, 1, 0, 0, true, PCM_F32, 3}, Linear{3, 256, 1 << 22, dtype, layout, 1, 3, 0, true, PCM_F32, 3},
                                    Linear{1 << 20, 512, 50021, dtype, layout, 2, 0, 0, false, PCM_F32, 3}}) {
                expect(forward(c), PCM_OK);
                expect(backward(c), PCM_OK);
            }
    expect(backward({(1 << 24) + 1, 64, 64, PCM_BF16, 0, 1, 0, 0, true, PCM_BF16, 3}), PCM_EUNSUPPORTED);
    for (int bits : {8, 32})
        for (bool clip : {false, true}) {
            std::vector<int64_t> numel;
            for (int64_t n : {1, 0, 127, 128, 129, 2048, 2049, 100000, 30000000}) {
                numel.push_back(n);
                expect(optimizer(numel, bits, clip, false), PCM_OK);
                if (bits == 8) expect(optimizer(numel, bits, clip, true), PCM_OK);
            }
            expect(optimizer({(int64_t)1 << 41}, bits, clip, false), PCM_OK);
            expect(optimizer({0, 0}, bits, clip, false), PCM_OK);
        }
}

template <class F>
void each_launch_fails(F f) {
    fail_at = -1;
    expect(f(), PCM_OK);
    const int n = launches;
    for (fail_at = 0; fail_at < n; ++fail_at) expect(f(), PCM_EHIP);
    fail_at = -1;
}
void errors() {
    for (int dtype : {PCM_F32, PCM_BF16})
        for (int layout = 0; layout < 2; ++layout)
            for (int64_t rows : {5, 300, 5000})
                for (int pad : {0, 1}) {
                    const Linear c{rows, 200, 5000, dtype, layout, 1, pad, 0, true, dtype, 3};
                    each_launch_fails([&] { return forward(c); });
                    each_launch_fails([&] { return backward(c); });
                }
    each_launch_fails([] { return optimizer({1000, 5, 100000}, 32, true, false); });
    each_launch_fails([] { return optimizer({1000, 5, 100000}, 8, false, false); });
    each_launch_fails([] { return optimizer({1000, 5, 100000}, 8, false, true); });
}

}  // namespace

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "bounds") bounds();
    else if (what == "errors") errors();
    else return 2;
    if (what == "bounds" && (products == 0 || pairs == 0 || in_parts == 0 || pieces == 0)) fail("the sweep", "a kind of launch did not occur");
    printf("%d calls, %d products (%d in parts by the rows, %d pairs), %d copies, %d failures\n", calls, products, in_parts, pairs, pieces, failures);
    return failures ? 1 : 0;
}
