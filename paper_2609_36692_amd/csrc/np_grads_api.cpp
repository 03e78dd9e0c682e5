// Host side of the gradient norm and clipping of the C ABI (include/normpre.h):
// argument checks, the lists of tensors that each launch works on.
#include "np_checks.h"
#include "np_grads.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

using namespace np;

namespace {

static_assert(kGradWorkspace == NORMPRE_GRAD_WORKSPACE_BYTES, "the header's size");
constexpr int64_t kMaxGrads = int64_t(1) << 20;
constexpr int64_t kMaxGradElements = int64_t(1) << 40;

int check_grads(int64_t num, const normpre_grad* g, bool scale) {
    if (num < 0) return bad("the number of gradients is negative");
    if (num > kMaxGrads) return fail(NORMPRE_ERR_UNSUPPORTED, "more than 2^20 gradients");
    if (num > 0 && !g) return bad("the list of gradients is null");
    int64_t all = 0;
    for (int64_t i = 0; i < num; ++i) {
        const normpre_grad& x = g[i];
        const long long at = i;
        if (!known(x.dtype)) return fail(NORMPRE_ERR_INVALID_ARG, "gradient %lld has an unknown dtype", at);
        if (x.count < 0) return fail(NORMPRE_ERR_INVALID_ARG, "gradient %lld has a negative size", at);
        if (x.count > kMaxGradElements - all) return fail(NORMPRE_ERR_UNSUPPORTED, "more than 2^40 elements");
        all += x.count;
        if (x.count && (!x.grad || !on(x.grad, size_of(x.dtype))))
            return fail(NORMPRE_ERR_INVALID_ARG, "gradient %lld is null or misaligned", at);
        if (!scale) continue;
        if (!known(x.out_dtype)) return fail(NORMPRE_ERR_INVALID_ARG, "output %lld has an unknown dtype", at);
        if (x.count && (!x.out || !on(x.out, size_of(x.out_dtype))))
            return fail(NORMPRE_ERR_INVALID_ARG, "output %lld is null or misaligned", at);
    }
    return NORMPRE_OK;
}

// Outputs lie apart from each other and from every gradient, but for a gradient that
// is scaled in place.
int check_apart(int64_t num, const normpre_grad* g) {
    struct Range { uintptr_t from, to; int64_t index; };
    std::vector<Range> outs;
    outs.reserve((size_t)num);
    for (int64_t i = 0; i < num; ++i)
        if (g[i].count) {
            const uintptr_t p = reinterpret_cast<uintptr_t>(g[i].out);
            outs.push_back({p, p + (uintptr_t)(g[i].count * size_of(g[i].out_dtype)), i});
        }
    std::sort(outs.begin(), outs.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
    for (size_t i = 1; i < outs.size(); ++i)
        if (outs[i].from < outs[i - 1].to)
            return fail(NORMPRE_ERR_INVALID_ARG, "outputs %lld and %lld overlap", (long long)outs[i - 1].index,
                        (long long)outs[i].index);
    for (int64_t i = 0; i < num; ++i) {
        if (!g[i].count) continue;
        const uintptr_t from = reinterpret_cast<uintptr_t>(g[i].grad), to = from + (uintptr_t)(g[i].count * size_of(g[i].dtype));
        // Outputs that end behind `from`, in their order: the first decides.
        auto o = std::partition_point(outs.begin(), outs.end(), [&](const Range& r) { return r.to <= from; });
        if (o == outs.end() || o->from >= to) continue;
        if (o->index != i || o->from != from || g[i].dtype != g[i].out_dtype)
            return fail(NORMPRE_ERR_INVALID_ARG, "gradient %lld overlaps output %lld", (long long)i, (long long)o->index);
    }
    return NORMPRE_OK;
}

// f(list) for every launch's list of tensors; the number of launches (at most
// 2^40 / 2^29 + 2^20 pieces of tensors: fewer than there are partial sums).
template <class F>
int64_t lists(int64_t num, const normpre_grad* g, bool scale, uint32_t chunk, F f) {
    GradList l;
    int64_t launches = 0;
    l.count = 0;
    l.first[0] = 0;
    auto flush = [&] {
        if (l.count == 0) return;
        ++launches;
        f(l);
        l.count = 0;
    };
    for (int64_t i = 0; i < num; ++i)
        for (int64_t at = 0; at < g[i].count; at += kGradMost) {
            const uint32_t n = (uint32_t)std::min<int64_t>(g[i].count - at, kGradMost);
            const int k = l.count++;
            l.size[k] = n | (g[i].dtype == NORMPRE_DTYPE_BF16 ? kGradInBf16 : 0) |
                        (g[i].out_dtype == NORMPRE_DTYPE_BF16 ? kGradOutBf16 : 0);
            l.in[k] = static_cast<const char*>(g[i].grad) + at * size_of(g[i].dtype);
            l.out[k] = scale ? static_cast<char*>(g[i].out) + at * size_of(g[i].out_dtype) : nullptr;
            l.first[k + 1] = l.first[k] + (n + chunk - 1) / chunk;
            if (l.count == kGradList) flush();
        }
    flush();
    return launches;
}

int grads(int64_t num, const normpre_grad* g, bool scale, double max_norm, float* norm, void* workspace,
          int64_t workspace_bytes, hipStream_t stream) {
    NP_CHECK(check_grads(num, g, scale));
    if (scale && !(max_norm >= 0.0)) return bad("max_norm is negative or NaN");
    if (!norm || !on(norm, 4)) return bad("norm is null or misaligned");
    if (!workspace || !on(workspace, 16) || workspace_bytes < kGradWorkspace)
        return bad("workspace is null, misaligned or too small");
    if (scale) try {
        NP_CHECK(check_apart(num, g));
    } catch (const std::bad_alloc&) {
        return fail(NORMPRE_ERR_OOM, "no memory to check the gradients");
    }
    if (!scale) max_norm = INFINITY;
    // Few elements: one launch of one block instead of three.
    int64_t few = 0;
    bool some = false;
    for (int64_t i = 0; i < num && few <= kGradSmallChunks; ++i) {
        few += std::min<int64_t>((g[i].count + kGradSmallChunk - 1) / kGradSmallChunk, kGradSmallChunks + 1);
        some |= g[i].count > 0;
    }
    if (few <= kGradSmallChunks && some) {
        hipError_t e = hipSuccess;
        lists(num, g, scale, kGradSmallChunk, [&](const GradList& l) { e = launch_grad_small(l, max_norm, norm, scale, stream); });
        return launched(e);
    }
    double* work = static_cast<double*>(workspace);
    // Blocks of a launch: all of them hold a partial sum.
    const int64_t launches = lists(num, g, scale, kGradChunk, [](const GradList&) {});
    const int most = (int)std::min<int64_t>(kGradBlocks, kGradPartials / std::max<int64_t>(launches, 1));
    auto blocks = [&](const GradList& l) { return (int)std::min<int64_t>(l.first[l.count], most); };
    int partials = 0;
    hipError_t e = hipSuccess;
    lists(num, g, scale, kGradChunk, [&](const GradList& l) {
        if (e != hipSuccess) return;
        e = launch_grad_squares(l, blocks(l), work + kGradHead + partials, stream);
        partials += blocks(l);
    });
    if (e == hipSuccess) e = launch_grad_total(work, partials, max_norm, norm, stream);
    if (scale)
        lists(num, g, scale, kGradScaleChunk, [&](const GradList& l) {
            if (e == hipSuccess) e = launch_grad_scale(l, blocks(l), work, stream);
        });
    return launched(e);
}

}  // namespace

extern "C" {

int normpre_grad_norm(int64_t num_grads, const normpre_grad* list, float* norm, void* workspace,
                      int64_t workspace_bytes, void* stream) {
    return grads(num_grads, list, false, 0.0, norm, workspace, workspace_bytes, (hipStream_t)stream);
}

int normpre_grad_clip(int64_t num_grads, const normpre_grad* list, double max_norm, float* norm, void* workspace,
                      int64_t workspace_bytes, void* stream) {
    return grads(num_grads, list, true, max_norm, norm, workspace, workspace_bytes, (hipStream_t)stream);
}

}  // extern "C"
