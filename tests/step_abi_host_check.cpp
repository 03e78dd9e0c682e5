// Driver for the sanitized build of the rotation's, the windows' and the gradient operators' host code
// (tests/test_step_abi_sanitized.py): the lists that launches get, and refusals,
// with launchers that only look at what they are given.
#include "../include/normpre.h"
#include "../paper_2609_36692_amd/csrc/np_grads.h"
#include "../paper_2609_36692_amd/csrc/np_rope.h"

#include <cstdio>
#include <limits>
#include <string>
#include <vector>

static int g_failures = 0;
static std::string g_error;

#define EXPECT(got, want)                                                                              \
    do {                                                                                               \
        const long long g_ = (long long)(got), w_ = (long long)(want);                                 \
        if (g_ != w_) {                                                                                \
            std::printf("line %d: %s is %lld, expected %lld (%s)\n", __LINE__, #got, g_, w_, g_error.c_str()); \
            ++g_failures;                                                                              \
        }                                                                                              \
    } while (0)

// What the launches of a call covered.
static long long g_squares, g_scaled, g_partials, g_total_of, g_launches;
static double* g_work;

namespace np {
int set_thread_error(int code, const char* msg) { g_error = msg; return code; }

static long long elements(const GradList& l, int blocks, uint32_t chunk) {
    EXPECT(l.count >= 1 && l.count <= kGradList, 1);
    EXPECT(l.first[0], 0);
    long long n = 0;
    for (int i = 0; i < l.count; ++i) {
        const uint32_t size = l.size[i] & (kGradInBf16 - 1);
        EXPECT(size >= 1 && size <= kGradMost, 1);
        EXPECT(l.first[i + 1] - l.first[i], (size + chunk - 1) / chunk);
        n += size;
    }
    EXPECT(blocks >= 1 && blocks <= kGradBlocks && (uint32_t)blocks <= l.first[l.count], 1);
    ++g_launches;
    return n;
}
hipError_t launch_grad_small(const GradList& l, double, float*, bool scale, hipStream_t) {
    const long long n = elements(l, 1, kGradSmallChunk);
    EXPECT(l.first[l.count] <= kGradSmallChunks, 1);
    g_squares += n;
    if (scale) g_scaled += n;
    g_total_of = g_partials;
    return hipSuccess;
}
hipError_t launch_grad_squares(const GradList& l, int blocks, double* partial, hipStream_t) {
    g_squares += elements(l, blocks, kGradChunk);
    EXPECT(partial - g_work, kGradHead + g_partials);    // one block's behind the other's
    g_partials += blocks;
    EXPECT(g_partials <= kGradPartials, 1);
    return hipSuccess;
}
hipError_t launch_grad_total(double* work, int partials, double, float*, hipStream_t) {
    EXPECT(work == g_work, 1);
    g_total_of = partials;
    return hipSuccess;
}
hipError_t launch_grad_scale(const GradList& l, int blocks, const double*, hipStream_t) {
    g_scaled += elements(l, blocks, kGradScaleChunk);
    return hipSuccess;
}

int64_t rope_workspace(DType, const RopeArgs& a) { return rope_sums(a) ? 100 : 0; }
hipError_t launch_rope(DType, const RopeArgs& a, bool backward, hipStream_t) {
    ++g_launches;
    EXPECT(a.partial != nullptr, backward && rope_sums(a));
    return a.tokens == 77 ? hipErrorInvalidValue : hipSuccess;
}

int attention_splits(int64_t, int) { return 2; }
int window_splits(DType, const AttnArgs&) { return 2; }
int64_t attention_workspace(const AttnArgs& a) { return 2 * (int64_t)a.heads * a.tokens + 1; }
hipError_t launch_window_forward(DType, const AttnArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_window_backward(DType, const AttnArgs& a, hipStream_t) {
    ++g_launches;
    EXPECT((reinterpret_cast<uintptr_t>(a.first_keys) - reinterpret_cast<uintptr_t>(a.lse2)) % 16, 0);
    return hipErrorInvalidValue;
}
}  // namespace np

static void window_calls(char* mem) {
    const int64_t huge = std::numeric_limits<int64_t>::max();
    // Plans, into buffers of exactly their size.
    for (const std::vector<int64_t>& lens : {std::vector<int64_t>{}, {0}, {1}, {128, 129, 0, 4000}, std::vector<int64_t>(999, 3), {100000}})
        for (int64_t window : {(int64_t)1, (int64_t)100, (int64_t)3999, huge})
            for (int64_t sinks : {(int64_t)0, (int64_t)1, (int64_t)130, huge}) {
                normpre_window w{window, sinks, -1, -1};
                int64_t n = -1;
                EXPECT(normpre_window_attention_plan_sizes((int64_t)lens.size(), lens.data(), &w, &n), NORMPRE_OK);
                const int64_t size = 8 * n + 8 * w.sink_tiles + 4 * w.sink_pieces;
                std::vector<int32_t> plan(size);
                EXPECT(normpre_window_attention_plan((int64_t)lens.size(), lens.data(), &w, plan.data(), size), NORMPRE_OK);
                EXPECT(normpre_window_attention_plan((int64_t)lens.size(), lens.data(), &w, plan.data(), size - 1), NORMPRE_ERR_INVALID_ARG);
            }
    int64_t n = 0, bad[2] = {huge, huge}, long_one[1] = {std::numeric_limits<int32_t>::max()};
    normpre_window w{1, huge, 0, 0};
    EXPECT(normpre_window_attention_plan_sizes(2, bad, &w, &n), NORMPRE_ERR_UNSUPPORTED);
    EXPECT(normpre_window_attention_plan_sizes(1, long_one, &w, &n), NORMPRE_OK);
    EXPECT(w.sink_pieces <= w.sink_tiles + 512, 1);

    normpre_attention a{};
    a.dtype = NORMPRE_DTYPE_BF16;
    a.heads = 4;
    a.kv_heads = 2;
    a.head_dim = 64;
    a.causal = 1;
    a.scale = 1.f;
    a.tokens = 300;
    a.plan = reinterpret_cast<int32_t*>(mem);
    a.num_tiles = 3;
    a.q = a.out = a.dout = a.dq = {mem, 256, 64};
    a.k = a.v = a.dk = a.dv = {mem, 128, 64};
    a.lse = reinterpret_cast<float*>(mem);
    a.workspace = mem;
    w = {5, 1, 1, 1};
    g_launches = 0;
    EXPECT(normpre_window_attention_workspace(&a, &w, &a.workspace_bytes), NORMPRE_OK);
    EXPECT(a.workspace_bytes, 4 * ((2 * 4 * 300 + 1 + 3) / 4 * 4 + 2 * 2 * 2 * 2 * 32 * 64));
    EXPECT(normpre_window_attention_forward(&a, &w, nullptr), NORMPRE_OK);
    EXPECT(normpre_window_attention_backward(&a, &w, nullptr), NORMPRE_ERR_HIP);
    EXPECT(g_launches, 2);
    for (const normpre_window& x : {normpre_window{huge, huge, huge, huge}, {-huge, 0, 0, 0}, {1, -huge, 0, 0}, {1, 1, -huge, 0},
                                    {1, 1, 1, huge}, {1, 1, 1, -huge}}) {
        EXPECT(normpre_window_attention_backward(&a, &x, nullptr), NORMPRE_ERR_INVALID_ARG);
        EXPECT(normpre_window_attention_workspace(&a, &x, &n), NORMPRE_ERR_INVALID_ARG);
    }
    normpre_attention b = a;
    b.tokens = b.num_tiles = std::numeric_limits<int32_t>::max();
    b.heads = b.kv_heads = 1;
    EXPECT(normpre_window_attention_forward(&b, &w, nullptr), NORMPRE_ERR_UNSUPPORTED);
    b.num_tiles = huge;
    EXPECT(normpre_window_attention_forward(&b, &w, nullptr), NORMPRE_ERR_INVALID_ARG);
    EXPECT(g_launches, 2);
}

static void rope_calls(char* mem) {
    const int64_t huge = std::numeric_limits<int64_t>::max();
    const int32_t most = std::numeric_limits<int32_t>::max(), least = std::numeric_limits<int32_t>::min();
    float* f = reinterpret_cast<float*>(mem);
    normpre_qk_rope a{};
    a.dtype = NORMPRE_DTYPE_BF16;
    a.heads = 4;
    a.kv_heads = 2;
    a.head_dim = 64;
    a.pairs = 32;
    a.norm = 1;
    a.num_axes = 1;
    a.position_bytes = 8;
    a.tokens = 100;
    a.freqs = reinterpret_cast<double*>(mem);
    a.positions = a.q_weight = a.k_weight = mem;
    a.q = a.q_out = a.dq = {mem, 256, 64};
    a.k = a.k_out = a.dk = {mem, 128, 64};
    a.dq_weight = a.dk_weight = f;
    a.workspace = mem;
    g_launches = 0;
    EXPECT(normpre_qk_rope_workspace(&a, &a.workspace_bytes), NORMPRE_OK);
    EXPECT(a.workspace_bytes, 400);
    EXPECT(normpre_qk_rope_forward(&a, nullptr), NORMPRE_OK);
    EXPECT(normpre_qk_rope_backward(&a, nullptr), NORMPRE_OK);
    EXPECT(g_launches, 2);
    normpre_qk_rope b = a;
    b.workspace_bytes = 399;
    EXPECT(normpre_qk_rope_backward(&b, nullptr), NORMPRE_ERR_INVALID_ARG);
    b.dq_weight = b.dk_weight = nullptr;
    b.workspace = nullptr;
    EXPECT(normpre_qk_rope_backward(&b, nullptr), NORMPRE_OK);
    b = a;
    b.tokens = 0;                                    // zero weight gradients
    EXPECT(normpre_qk_rope_forward(&b, nullptr), NORMPRE_OK);
    EXPECT(g_launches, 3);
    EXPECT(normpre_qk_rope_backward(&b, nullptr), NORMPRE_OK);
    EXPECT(g_launches, 4);
    b.tokens = 77;
    EXPECT(normpre_qk_rope_forward(&b, nullptr), NORMPRE_ERR_HIP);
    b = a;
    b.tokens = huge;
    EXPECT(normpre_qk_rope_forward(&b, nullptr), NORMPRE_ERR_UNSUPPORTED);
    b = a;
    b.heads = most;
    EXPECT(normpre_qk_rope_workspace(&b, &b.workspace_bytes), NORMPRE_ERR_UNSUPPORTED);
    for (int32_t n : {least, -1, 33, most}) {
        b = a;
        b.pairs = n;
        EXPECT(normpre_qk_rope_forward(&b, nullptr), NORMPRE_ERR_INVALID_ARG);
    }
    b = a;
    b.tokens = most;
    b.heads = b.kv_heads = np::kRopeMaxHeads;
    b.q_out = {mem, int64_t(1) << 40, int64_t(1) << 40};
    EXPECT(normpre_qk_rope_forward(&b, nullptr), NORMPRE_ERR_INVALID_ARG);
    b.q_out = {mem, huge, 64};
    EXPECT(normpre_qk_rope_forward(&b, nullptr), NORMPRE_ERR_UNSUPPORTED);
}

static void reset() { g_squares = g_scaled = g_partials = g_launches = 0; g_total_of = -1; }

int main() {
    const int64_t huge = std::numeric_limits<int64_t>::max();
    alignas(16) static char mem[64];
    char* const far = reinterpret_cast<char*>(uintptr_t(1) << 44);
    float* norm = reinterpret_cast<float*>(mem);
    g_work = reinterpret_cast<double*>(mem + 16);
    const int64_t ws = NORMPRE_GRAD_WORKSPACE_BYTES;

    // Tensors of one element, of several pieces, of none; more than a launch holds.
    for (int64_t count : {0, 1, 3, 40, 60, 151, 152, 153, 5000, 1 << 20}) {
        std::vector<normpre_grad> g(count);
        long long all = 0;
        char* at = far;
        for (int64_t i = 0; i < count; ++i) {
            const int64_t n = i == 3 && count != 40 ? (int64_t(1) << 32) + 5 : i % 7 == 5 ? 0 : i % 100 + 1;
            g[i] = {at, at, n, (int)(i % 2), (int)(i % 2)};
            at += 4 * n;
            all += n;
        }
        reset();
        EXPECT(normpre_grad_norm(count, g.data(), norm, g_work, ws, nullptr), NORMPRE_OK);
        EXPECT(g_squares, all);
        EXPECT(g_total_of, g_partials);
        EXPECT(g_scaled, 0);
        reset();
        EXPECT(normpre_grad_clip(count, g.data(), 1.0, norm, g_work, ws, nullptr), NORMPRE_OK);
        EXPECT(g_squares, all);
        EXPECT(g_scaled, all);
        for (auto& x : g) x.out = nullptr;
        reset();
        EXPECT(normpre_grad_norm(count, g.data(), norm, g_work, ws, nullptr), NORMPRE_OK);
    }
    reset();
    EXPECT(normpre_grad_norm(0, nullptr, norm, g_work, ws, nullptr), NORMPRE_OK);
    EXPECT(g_total_of, 0);
    // The largest call that is taken: 2^40 elements in all.
    std::vector<normpre_grad> g(1 << 20, normpre_grad{far, nullptr, 1, 0, 0});
    g[0].count = (int64_t(1) << 40) - (1 << 20) + 1;
    reset();
    EXPECT(normpre_grad_norm(1 << 20, g.data(), norm, g_work, ws, nullptr), NORMPRE_OK);
    ++g[0].count;
    reset();
    EXPECT(normpre_grad_norm(1 << 20, g.data(), norm, g_work, ws, nullptr), NORMPRE_ERR_UNSUPPORTED);
    g[0].count = huge;
    EXPECT(normpre_grad_norm(1 << 20, g.data(), norm, g_work, ws, nullptr), NORMPRE_ERR_UNSUPPORTED);
    EXPECT(normpre_grad_norm(huge, g.data(), norm, g_work, ws, nullptr), NORMPRE_ERR_UNSUPPORTED);
    EXPECT(normpre_grad_norm(-huge, g.data(), norm, g_work, ws, nullptr), NORMPRE_ERR_INVALID_ARG);
    g[0].count = -huge;
    EXPECT(normpre_grad_norm(2, g.data(), norm, g_work, ws, nullptr), NORMPRE_ERR_INVALID_ARG);
    EXPECT(g_launches, 0);
    rope_calls(mem);
    window_calls(mem);

    std::printf("%d failure(s)\n", g_failures);
    return g_failures != 0;
}
