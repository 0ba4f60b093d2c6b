// Runs the host side of the operators on logits and on updates, as built in libpcm.so, on a HIP runtime of its own that launches
// nothing, so no GPU is needed or touched.  Every launch is looked at as the library issues it: what its kernels read and write has to lie
// inside the buffers that the call was given, with a workspace as long as the library's own query says, and what a launch writes may not
// be what it reads elsewhere.  A kernel that is not known here is a failure.
//
//   operators_path bounds   sweeps sizes and options and checks every launch
//   operators_path errors   lets each launch of a call fail in turn: the call has to return PCM_EHIP
#include <cxxabi.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <map>
#include <string>
#include <vector>

#include "gemm_pairs.h"
#include "orthogonalise.h"
#include "pcm.h"
#include "token_logprobs.h"

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
int failures = 0, launches = 0, calls = 0, products = 0, in_parts = 0;
int64_t rows_seen = 0;                                 // of the logits of a call
int fail_at = -1;                                      // the launch that fails, or -1
bool check_bounds = false;
hipError_t last_error = hipSuccess;

void fail(const char* kernel, const char* text) {
    if (++failures <= 20) printf("%s\n  %s: %s\n", call.c_str(), kernel, text);
}
void* buffer(const char* what, size_t bytes) {
    const uintptr_t begin = regions.empty() ? (uintptr_t)1 << 40 : (regions.back().end + (1u << 20)) / 4096 * 4096;
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
bool inside(uintptr_t begin, uintptr_t end) {
    for (const Region& r : regions)
        if (begin >= r.begin && end <= r.end) return true;
    return false;
}
void touches(const char* what, const void* p, size_t bytes, bool written, size_t beyond = 0) {
    if (bytes == 0) return;
    const uintptr_t begin = (uintptr_t)p;
    spans.push_back(Span{what, begin, begin + bytes, written});
    if (inside(begin, begin + bytes + beyond)) return;
    char text[200];
    snprintf(text, sizeof text, "%s, %zu bytes and %zu beyond them, is not inside a buffer", what, bytes, beyond);
    fail(kernel, text);
}
void touches_rows(const char* what, const void* p, int64_t rows, int64_t columns, int64_t ld, size_t size, bool written) {
    if (rows > 0) touches(what, p, (size_t)((rows - 1) * ld + columns) * size, written);
}
void check_overlaps() {
    for (size_t a = 0; a < spans.size(); ++a)
        for (size_t b = 0; b < a; ++b) {
            const Span &p = spans[a], &q = spans[b];
            if (!(p.written || q.written) || (p.begin == q.begin && p.end == q.end && strcmp(p.what, q.what) == 0) || p.end <= q.begin || q.end <= p.begin) continue;
            char text[200];
            snprintf(text, sizeof text, "%s and %s share memory", p.what, q.what);
            fail(kernel, text);
        }
}

// ---- products: kW from the name, any list of jobs (a longer list begins like a shorter one but for the count behind it)
size_t pairs_bytes(int frags, int64_t steps) { return (size_t)pair_fragment(0, steps, frags) * 2; }
void look_at_job(const PairJob& p, int kW, bool final) {
    ++products;
    if (p.m_frags < 2 || p.n_frags < 2 || p.m_frags % 2 || p.n_frags % 2 || p.steps < 1) fail(kernel, "sizes that are no multiples of 32");
    if (p.tiles_m * 2 * kW < p.m_frags || p.tiles_n * 2 * kW < p.n_frags || (p.tiles_m - 1) * 2 * kW >= p.m_frags || (p.tiles_n - 1) * 2 * kW >= p.n_frags)
        fail(kernel, "tiles that do not fit the result");
    if (p.symmetric && p.m_frags != p.n_frags) fail(kernel, "a symmetric result that is not square");
    if ((p.result != kPairs) != final) fail(kernel, "results and pairs in one launch");
    touches("A", p.A, pairs_bytes(p.m_frags, p.steps), false, pairs_bytes(p.m_frags, kPairStepsBeyond));
    touches("B", p.B, pairs_bytes(p.n_frags, p.steps), false, pairs_bytes(p.n_frags, kPairStepsBeyond));
    if (!final) {
        touches("C", p.C, pairs_bytes(p.m_frags, p.n_frags / 2), true);
        if (p.Ct != nullptr && p.Ct != p.C) touches("C transposed", p.Ct, pairs_bytes(p.n_frags, p.m_frags / 2), true);
        if (p.D != nullptr) touches("D", p.D, pairs_bytes(p.m_frags, p.n_frags / 2), false);
        return;
    }
    const size_t size = p.result == kOutBf16 ? 2 : 4;
    if (p.rows > p.m_frags * 16 || p.cols > p.n_frags * 16) fail(kernel, "a result larger than the product");
    touches_rows("the result", p.out, p.rows, p.cols, p.ld, size, true);
    if (p.result == kOutWeights && p.lowp != nullptr) touches_rows("the bf16 copy", p.lowp, p.rows, p.cols, p.ld, 2, true);
}
template <int kMax>
void look_at_products(const std::string& name, int kW, bool final, void** args, dim3 grid) {
    const PairJobList<kMax>& list = *static_cast<PairJobList<kMax>*>(args[0]);
    if (list.n < 1 || list.n > kMax) return fail(kernel, "a list longer than its argument");
    int blocks = 0;
    const int splits = list.job[0].splits;
    for (int i = 0; i < list.n; ++i) {
        const PairJob& p = list.job[i];
        if (p.first != blocks || p.first_part != blocks) fail(kernel, "workgroups that do not follow one another");
        if (p.splits != splits || splits < 1 || splits > p.steps || (splits > 1 && (kW != kPairPartTile || final))) fail(kernel, "parts that do not fit");
        blocks += (p.tiles() * splits + 7) / 8 * 8;
        look_at_job(p, kW, final);
    }
    if (splits > 1) {
        if (blocks > kPairParts) fail(kernel, "more parts than their buffer has");
        touches("parts", list.parts, (size_t)blocks * 64 * 64 * 4, true);
        in_parts += list.n;
    }
    if ((int)grid.x != blocks) fail(kernel, "a grid that does not fit the jobs");
}
template <int kMax>
void look_at_join(void** args, dim3 grid) {
    const PairJobList<kMax>& list = *static_cast<PairJobList<kMax>*>(args[0]);
    int tiles = 0;
    for (int i = 0; i < list.n; ++i) {
        const PairJob& p = list.job[i];
        if (p.first != tiles) fail(kernel, "workgroups that do not follow one another");
        tiles += p.tiles();
        touches("parts", list.parts + (int64_t)p.first_part * 1024, (size_t)p.tiles() * p.splits * 64 * 64 * 4, false);
        touches("C", p.C, pairs_bytes(p.m_frags, p.n_frags / 2), true);
        if (p.Ct != nullptr && p.Ct != p.C) touches("C transposed", p.Ct, pairs_bytes(p.n_frags, p.m_frags / 2), true);
        if (p.D != nullptr) touches("D", p.D, pairs_bytes(p.m_frags, p.n_frags / 2), false);
    }
    if ((int)grid.x != tiles) fail(kernel, "a grid that does not fit the jobs");
}
void look_at_matrices(bool squares, void** args, dim3 grid) {
    const UpdateMatrices& list = *static_cast<UpdateMatrices*>(args[0]);
    int blocks = 0;
    for (int i = 0; i < list.n; ++i) {
        const UpdateMatrix& q = list.m[i];
        const int64_t tiles = (int64_t)((q.rows + 63) / 64) * ((q.cols + 63) / 64);
        if (q.tiles != tiles || q.tiles_c != (q.cols + 63) / 64 || q.parts < 1 || q.parts > q.tiles) fail(kernel, "tiles that do not fit the matrix");
        if ((squares ? q.first_part : q.first_tile) != blocks) fail(kernel, "workgroups that do not follow one another");
        blocks += squares ? q.parts : q.tiles;
        touches_rows("the update", q.in, q.rows, q.cols, q.ld, q.bf16 ? 2 : 4, false);
        if (q.momentum != nullptr) touches_rows("the momentum", q.momentum, q.rows, q.cols, q.ld, 4, squares);
        touches("sums", q.partial, (size_t)q.parts * 8, squares);
        if (squares) continue;
        const int m = q.rows < q.cols ? q.rows : q.cols, n = q.rows < q.cols ? q.cols : q.rows;
        touches("X", q.X, pair_values(m, n) * 2, true);
        touches("X transposed", q.Xt, pair_values(m, n) * 2, true);
    }
    if ((int)grid.x != blocks) fail(kernel, "a grid that does not fit the matrices");
}

// ---- logits
void look_at_logits(const Logits& q, size_t size) {
    touches_rows("logits", q.z, q.rows, q.V, q.ld, size, false);
    touches("tokens", q.tokens, (size_t)q.rows * (q.token_type == PCM_TOKEN_U8 ? 1 : q.token_type == PCM_TOKEN_I32 ? 4 : 8), false);
    if (q.allowed != nullptr) touches_rows("the mask", q.allowed, q.allowed_ld ? q.rows : 1, q.V, q.allowed_ld ? q.allowed_ld : q.V, 1, false);
}
void look_at_outputs(const Logits& q, const LogprobsOut& o) {
    touches("logp", o.logp, (size_t)q.rows * 4, true);
    touches("lse", o.lse, (size_t)q.rows * 4, true);
    if (o.entropy != nullptr) touches("entropy", o.entropy, (size_t)q.rows * 4, true);
    if (o.top > 0) {
        touches("top_ids", o.top_ids, (size_t)q.rows * o.top * 4, true);
        touches("top_logp", o.top_logp, (size_t)q.rows * o.top * 4, true);
    }
}
void look_at_parts(const Logits& q, const LogprobsOut& o, const RowParts& p, bool written) {
    touches("sums", p.sums, (size_t)q.rows * p.parts * sizeof(RowSums), written);
    touches("keys", p.keys, (size_t)q.rows * p.parts * o.top * 8, written);
}
void look_at_launch(const std::string& name, void** args, dim3 grid) {
    auto has = [&](const char* text) { return name.find(text) != std::string::npos; };
    const size_t size = has("<float") ? 4 : 2;
    auto number = [&](size_t from) { return atoi(name.c_str() + from); };
    if (has("pair_product<")) {
        const size_t at = name.find("pair_product<") + 13, comma = name.find(',', at), last = name.find(',', comma + 1);
        const int kW = number(at), kMax = number(last + 1);
        const bool final = name.compare(comma + 2, 4, "true") == 0;
        if (kMax == kFewPairJobs) look_at_products<kFewPairJobs>(name, kW, final, args, grid);
        else if (kMax == kMaxPairJobs) look_at_products<kMaxPairJobs>(name, kW, final, args, grid);
        else fail(kernel, "an unknown list");
    } else if (has("pair_join<")) {
        const int kMax = number(name.find("pair_join<") + 10);
        if (kMax == kFewPairJobs) look_at_join<kFewPairJobs>(args, grid);
        else if (kMax == kMaxPairJobs) look_at_join<kMaxPairJobs>(args, grid);
        else fail(kernel, "an unknown list");
    } else if (has("update_squares")) {
        look_at_matrices(true, args, grid);
    } else if (has("update_to_pairs")) {
        look_at_matrices(false, args, grid);
    } else if (has("token_logprobs_parts<") || has("token_logprobs_join<")) {
        const Logits& q = *static_cast<Logits*>(args[0]);
        const LogprobsOut& o = *static_cast<LogprobsOut*>(args[1]);
        const RowParts& p = *static_cast<RowParts*>(args[2]);
        const bool joins = has("join<");
        look_at_logits(q, size);
        if (p.parts > 1) look_at_parts(q, o, p, !joins);
        if (joins || p.parts == 1) look_at_outputs(q, o);
        if (!joins) rows_seen += q.rows;
        if ((int64_t)grid.x != q.rows * (joins ? 1 : p.parts)) fail(kernel, "a grid that does not fit the rows");
        if (!joins && (int64_t)p.parts * 2048 > q.V + 2048 && p.parts > 1) fail(kernel, "more parts than the row has");
    } else if (has("token_logprobs_narrow<")) {
        const Logits& q = *static_cast<Logits*>(args[0]);
        const int lanes = number(name.rfind(", ", name.find('>')) + 2);
        look_at_logits(q, size);
        look_at_outputs(q, *static_cast<LogprobsOut*>(args[1]));
        rows_seen += q.rows;
        if (q.V > 16 * lanes) fail(kernel, "a row that its lanes do not hold");
        if ((int64_t)grid.x * (256 / lanes) < q.rows) fail(kernel, "a grid that does not fit the rows");
    } else if (has("token_logprobs_gradient<")) {
        const Logits& q = *static_cast<Logits*>(args[0]);
        const LogprobsGradient& b = *static_cast<LogprobsGradient*>(args[1]);
        const int lanes = number(name.rfind(", ", name.find('>')) + 2), parts = *static_cast<int*>(args[2]);
        look_at_logits(q, size);
        rows_seen += q.rows;
        for (const float* p : {b.lse, b.dlogp, b.entropy, b.dentropy})
            if (p != nullptr) touches("a value per row", p, (size_t)q.rows * 4, false);
        touches_rows(b.dz == q.z ? "logits" : "the gradient", b.dz, q.rows, q.V, b.dz_ld, size, true);
        if ((int64_t)grid.x < (q.rows + 256 / lanes - 1) / (256 / lanes) * parts) fail(kernel, "a grid that does not fit the rows");
    } else {
        fail(kernel, "a launch that this program does not know");
    }
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
        if (grid.x == 0 || grid.y != 1 || grid.z != 1 || block.x * block.y * block.z > 1024 || (uint64_t)grid.x * block.x >> 32)
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

void begin(const char* text) {
    call = text;
    regions.clear();
    launches = 0;
    rows_seen = 0;
    last_error = hipSuccess;
    ++calls;
}

struct RowsCall {
    int64_t rows;
    int V, dtype, token_type, mask, top;               // mask: 0 none, 1 [V], 2 [rows, V]
    bool entropy;
    int pad;
};
int forward(const RowsCall& c) {
    char text[200];
    snprintf(text, sizeof text, "log-probabilities, %lld rows of %d (+%d), type %d, tokens %d, mask %d, top %d, entropy %d", (long long)c.rows, c.V, c.pad, c.dtype,
             c.token_type, c.mask, c.top, c.entropy);
    begin(text);
    const size_t size = c.dtype == PCM_F32 ? 4 : 2, token = c.token_type == PCM_TOKEN_U8 ? 1 : c.token_type == PCM_TOKEN_I32 ? 4 : 8;
    const int64_t ld = c.V + c.pad;
    void* z = buffer("logits", ((c.rows - 1) * ld + c.V) * size);
    void* tokens = buffer("tokens", c.rows * token);
    uint8_t* mask = c.mask ? (uint8_t*)buffer("mask", c.mask == 1 ? c.V : (c.rows - 1) * ld + c.V) : nullptr;
    float *logp = (float*)buffer("logp", c.rows * 4), *lse = (float*)buffer("lse", c.rows * 4);
    float* entropy = c.entropy ? (float*)buffer("entropy", c.rows * 4) : nullptr;
    int32_t* ids = c.top ? (int32_t*)buffer("ids", c.rows * c.top * 4) : nullptr;
    float* best = c.top ? (float*)buffer("top_logp", c.rows * c.top * 4) : nullptr;
    const size_t bytes = pcm_token_logprobs_workspace_bytes(c.rows, c.V, c.top);
    void* ws = bytes ? buffer("workspace", bytes) : nullptr;
    return pcm_token_logprobs(z, ld, c.dtype, tokens, c.token_type, mask, c.mask == 2 ? ld : 0, c.rows, c.V, 0.7f, c.top, logp, lse, entropy, ids, best, ws,
                              bytes, nullptr);
}
int backward(const RowsCall& c, bool in_place) {
    char text[200];
    snprintf(text, sizeof text, "gradient, %lld rows of %d (+%d), type %d, mask %d, entropy %d", (long long)c.rows, c.V, c.pad, c.dtype, c.mask, c.entropy);
    begin(text);
    const size_t size = c.dtype == PCM_F32 ? 4 : 2;
    const int64_t ld = c.V + c.pad;
    void* z = buffer("logits", ((c.rows - 1) * ld + c.V) * size);
    void* tokens = buffer("tokens", c.rows * 4);
    uint8_t* mask = c.mask ? (uint8_t*)buffer("mask", c.mask == 1 ? c.V : (c.rows - 1) * ld + c.V) : nullptr;
    float *lse = (float*)buffer("lse", c.rows * 4), *dlogp = (float*)buffer("dlogp", c.rows * 4);
    float *entropy = c.entropy ? (float*)buffer("entropy", c.rows * 4) : nullptr, *dentropy = c.entropy ? (float*)buffer("dentropy", c.rows * 4) : nullptr;
    void* dz = in_place ? z : buffer("gradient", ((c.rows - 1) * ld + c.V) * size);
    return pcm_token_logprobs_backward(z, ld, c.dtype, tokens, PCM_TOKEN_I32, mask, c.mask == 2 ? ld : 0, c.rows, c.V, 1.f, lse, dlogp, entropy, dentropy, dz, ld,
                                       nullptr);
}
int orthogonalise(int batch, int rows, int cols, int dtype, int steps, int pad) {
    char text[200];
    snprintf(text, sizeof text, "orthogonalise %d of %d x %d (+%d), type %d, %d steps", batch, rows, cols, pad, dtype, steps);
    begin(text);
    const size_t size = dtype == PCM_F32 ? 4 : 2;
    const int64_t ld = cols + pad, stride = rows * ld + 3;
    void* in = buffer("update", ((batch - 1) * stride + (rows - 1) * ld + cols) * size);
    void* out = buffer("out", ((batch - 1) * stride + (rows - 1) * ld + cols) * size);
    const size_t bytes = pcm_orthogonalise_workspace_bytes(batch, rows, cols);
    void* ws = buffer("workspace", bytes);
    return pcm_orthogonalise(in, ld, stride, out, ld, stride, batch, rows, cols, dtype, steps, ws, bytes, nullptr);
}
int muon(const std::vector<std::pair<int, int>>& shapes, bool lowp) {
    std::string text = "Muon step of";
    for (const auto& s : shapes) text += " " + std::to_string(s.first) + " x " + std::to_string(s.second);
    begin(text.c_str());
    int rows[8], cols[8];
    const float* g[8];
    float *w[8], *m[8];
    void* b[8];
    const int n = (int)shapes.size();
    for (int i = 0; i < n; ++i) {
        rows[i] = shapes[i].first;
        cols[i] = shapes[i].second;
        const size_t count = (size_t)rows[i] * cols[i];
        g[i] = (const float*)buffer("gradient", count * 4);
        w[i] = (float*)buffer("weights", count * 4);
        m[i] = (float*)buffer("momentum", count * 4);
        b[i] = lowp && i % 3 != 1 ? buffer("bf16 weights", count * 2) : nullptr;
    }
    const size_t bytes = pcm_muon_step_workspace_bytes(n, rows, cols);
    void* ws = buffer("workspace", bytes);
    return pcm_muon_step(n, rows, cols, g, w, m, lowp ? b : nullptr, 0.02, 0.95, 1, 0.01, 5, PCM_MUON_SCALE_SHAPE, ws, bytes, nullptr);
}
void expect(int rc, int want) {
    if (rc == want) return;
    char text[60];
    snprintf(text, sizeof text, "returned %d, not %d", rc, want);
    fail("the call", text);
}

const int kSides[] = {1, 2, 15, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 193, 255, 257, 300, 511, 513, 1000, 1025, 2049, 4096, 4097, 5504, 11008, 40000};
void bounds() {
    check_bounds = true;
    for (int rows : kSides)
        for (int cols : kSides) {
            if ((int64_t)rows * cols > (int64_t)4097 * 40000) continue;
            for (int steps : {1, 2, 3, 4, 5, 7, 10}) expect(orthogonalise(1, rows, cols, PCM_F32, steps, 0), PCM_OK);
            expect(orthogonalise(3, rows, cols, PCM_BF16, 5, 7), PCM_OK);
            expect(orthogonalise(19, rows, cols, PCM_F32, 5, 1), PCM_OK);
            expect(muon({{rows, cols}, {cols, rows}, {rows, cols}, {64, 64}, {rows, 1}}, true), PCM_OK);
        }
    expect(muon({{4096, 11008}, {4096, 11008}, {11008, 4096}, {4096, 256}}, true), PCM_OK);
    expect(muon({{256, 1024}, {256, 1024}, {1024, 256}, {256, 256}, {1, 1}, {7, 9}, {100, 3}, {64, 128}}, false), PCM_OK);
    expect(orthogonalise(1, 1 << 15, 1 << 15, PCM_F32, 5, 0), PCM_OK);
    expect(orthogonalise(1, 1 << 20, 3, PCM_F32, 5, 0), PCM_OK);
    for (int64_t rows : {1, 2, 7, 8, 63, 64, 100, 777, 2047, 2049, 4096, 43008, 3000000})
        for (int V : {1, 2, 7, 8, 9, 63, 64, 65, 128, 129, 255, 256, 257, 512, 513, 1023, 1024, 1025, 4095, 4096, 4097, 8191, 8192, 32003, 65536, 131072, 1 << 24}) {
            if (rows * V > (int64_t)1 << 32) continue;
            for (int mask = 0; mask < 3; ++mask)
                for (int top : {0, 1, 20, 64}) {
                    const RowsCall c{rows, V, top % 2 ? PCM_F32 : PCM_BF16, (int)(rows + V + top) % 3, mask, top, (rows + mask) % 2 == 0, top};
                    expect(forward(c), PCM_OK);
                    expect(backward(c, top == 0), PCM_OK);
                }
        }
    for (int64_t rows : {(int64_t)8388607, (int64_t)8388609, (int64_t)70000001, (int64_t)0x7fffffff})    // launches of less than 2^32 threads
        for (int V : {1, 2, 300, 2000, 5000})
            for (int top : {0, 1}) {
                const RowsCall c{rows, V, top ? PCM_F32 : PCM_BF16, V % 3, V % 2 ? 2 : 1, top, true, top};
                expect(forward(c), PCM_OK);
                if (rows_seen != rows) fail("the call", "not every row once");
                expect(backward(c, top == 0), PCM_OK);
                if (rows_seen != rows) fail("the call", "not every row once");
            }
    expect(forward({2, 1 << 30, PCM_BF16, PCM_TOKEN_I64, 1, 5, true, 0}), PCM_OK);
    expect(backward({2, 1 << 30, PCM_BF16, PCM_TOKEN_I64, 1, 5, true, 0}, false), PCM_OK);
    expect(forward({2, (1 << 30) + 1, PCM_BF16, PCM_TOKEN_I64, 1, 0, true, 0}), PCM_EUNSUPPORTED);
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
    for (int top : {0, 3})
        for (int V : {100, 3000, 100000}) {
            each_launch_fails([&] { return forward({5, V, PCM_F32, PCM_TOKEN_I32, 0, top, true, 0}); });
            each_launch_fails([&] { return backward({5, V, PCM_F32, PCM_TOKEN_I32, 0, top, true, 0}, false); });
        }
    each_launch_fails([] { return orthogonalise(1, 100, 300, PCM_F32, 5, 0); });
    each_launch_fails([] { return orthogonalise(20, 300, 100, PCM_BF16, 4, 0); });
    each_launch_fails([] { return orthogonalise(2, 4096, 11008, PCM_F32, 5, 0); });
    each_launch_fails([] { return muon({{256, 1024}, {1024, 256}, {4096, 4096}, {4096, 11008}}, true); });
}

}  // namespace

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "bounds") bounds();
    else if (what == "errors") errors();
    else return 2;
    if (what == "bounds" && in_parts == 0) fail("products", "none was done in parts");
    printf("%d calls, %d products, %d of them in parts, %d failures\n", calls, products, in_parts, failures);
    return failures == 0 ? 0 : 1;
}
