// Host side of the training-step operators of the C ABI (include/normpre.h):
// argument checks, the plan of a packed batch, and the calls of the kernels'
// launchers.  Nothing here keeps state or computes results on the host.
#include "np_checks.h"

#include <algorithm>
#include <cstring>
#include <new>
#include <vector>

using namespace np;

namespace {

// ----------------------------------------------------------- attention ---
// The sizes alone, with what the backward pass makes of them.
AttnArgs sizes(const normpre_attention* a) {
    AttnArgs k = attention_sizes(a);
    k.splits = attention_splits(a->num_tiles, a->kv_heads);
    return k;
}

int attention(const normpre_attention* a, bool backward, void* stream) {
    NP_CHECK(check_attention(a, backward));
    if (a->tokens == 0) return NORMPRE_OK;
    AttnArgs k = sizes(a);
    attention_operands(a, backward, k);
    const DType dt = (DType)a->dtype;
    if (!backward) return launched(launch_attention_forward(dt, k, (hipStream_t)stream));
    float* ws = static_cast<float*>(a->workspace);
    if (!ws || !on(ws, 16) || a->workspace_bytes < 4 * attention_workspace(k))
        return bad("workspace is null, misaligned or too small");
    attention_parts(ws, k);
    return launched(launch_attention_backward(dt, k, (hipStream_t)stream));
}

// --------------------------------------------------------- checkpoints ---
int check_matrix(int dtype, int64_t rows, int64_t cols) {
    if (!known(dtype)) return fail(NORMPRE_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    if (rows < 0 || cols < 1)
        return fail(NORMPRE_ERR_INVALID_ARG, "bad shape %lld x %lld", (long long)rows, (long long)cols);
    if (cols > kMaxElements || rows > kMaxElements / ckpt_pitch(cols))
        return fail(NORMPRE_ERR_UNSUPPORTED, "more than 2^34 elements");
    return NORMPRE_OK;
}

int check_rows(const char* name, const void* p, int64_t ld, int64_t cols, int64_t elt) {
    if (!p || !on(p, elt)) return fail(NORMPRE_ERR_INVALID_ARG, "%s is null or misaligned", name);
    if (ld < cols) return fail(NORMPRE_ERR_INVALID_ARG, "row stride of %s is smaller than a row", name);
    if (ld > kMaxStride) return fail(NORMPRE_ERR_UNSUPPORTED, "row stride of %s exceeds 2^40", name);
    return NORMPRE_OK;
}

int check_held(const char* name, const int8_t* codes, const int8_t* exps) {
    if (!codes || !exps || !on(codes, 16))
        return fail(NORMPRE_ERR_INVALID_ARG, "checkpoint of %s is null or not 16-byte aligned", name);
    return NORMPRE_OK;
}

}  // namespace

extern "C" {

int normpre_attention_plan_tiles(int64_t num_seqs, const int64_t* lens, int64_t* num_tiles) {
    if (!num_tiles) return bad("num_tiles is null");
    int64_t tiles, tokens;
    NP_CHECK(count_tiles(num_seqs, lens, tiles, tokens));
    *num_tiles = tiles;
    return NORMPRE_OK;
}

int normpre_attention_plan(int64_t num_seqs, const int64_t* lens, int causal, int32_t* plan, int64_t capacity) {
    int64_t n, tokens;
    NP_CHECK(count_tiles(num_seqs, lens, n, tokens));
    if (causal != 0 && causal != 1) return bad("causal is neither 0 nor 1");
    if (capacity < 8 * n) return bad("the plan does not fit");
    if (n == 0) return NORMPRE_OK;
    if (!plan) return bad("plan is null");
    try {
        // Rows that the other side streams past one tile: queries of a causal
        // tile see the keys up to its end, keys are seen by the queries from
        // its start on.
        struct Item { AttnTile t; int64_t work; };
        std::vector<Item> items((size_t)n);
        for (int side = 0; side < 2; ++side) {
            size_t at = 0;
            int64_t start = 0;
            for (int64_t i = 0; i < num_seqs; ++i) {
                const int64_t len = lens[i];
                for (int64_t k = 0; k * kAttnRows < len; ++k) {
                    const int64_t seen = !causal ? len
                                         : side == 0 ? std::min(len, (k + 1) * kAttnRows)
                                                     : len - k * kAttnRows;
                    items[at++] = {{(int32_t)start, (int32_t)len, (int32_t)k, 0}, seen};
                }
                start += len;
            }
            std::stable_sort(items.begin(), items.end(),
                             [](const Item& x, const Item& y) { return x.work > y.work; });
            for (size_t i = 0; i < items.size(); ++i)
                std::memcpy(plan + 4 * (side * (size_t)n + i), &items[i].t, sizeof(AttnTile));
        }
    } catch (const std::bad_alloc&) {
        return fail(NORMPRE_ERR_OOM, "no memory for the plan");
    }
    return NORMPRE_OK;
}

int normpre_attention_workspace(const normpre_attention* a, int64_t* bytes) {
    if (!bytes) return bad("bytes is null");
    NP_CHECK(check_attention_sizes(a));
    *bytes = 4 * attention_workspace(sizes(a));
    return NORMPRE_OK;
}

int normpre_attention_forward(const normpre_attention* a, void* stream) { return attention(a, false, stream); }

int normpre_attention_backward(const normpre_attention* a, void* stream) { return attention(a, true, stream); }

int normpre_checkpoint_pack(int act, int dtype, int64_t rows, int64_t cols, const void* u, int64_t ld_u,
                            const void* up, int64_t ld_up, void* h, int64_t ld_h, int8_t* u_codes, int8_t* u_exps,
                            int8_t* up_codes, int8_t* up_exps, int8_t* h_codes, int8_t* h_exps, void* stream) {
    if (act < NORMPRE_ACT_NONE || act > NORMPRE_ACT_SWIGLU)
        return fail(NORMPRE_ERR_INVALID_ARG, "unknown activation %d", act);
    NP_CHECK(check_matrix(dtype, rows, cols));
    if (rows == 0) return NORMPRE_OK;
    const int64_t e = size_of(dtype);
    CkptPackArgs a{};
    a.rows = rows;
    a.cols = cols;
    NP_CHECK(check_rows("u", u, ld_u, cols, e));
    NP_CHECK(check_held("u", u_codes, u_exps));
    a.u = u;
    a.ld_u = ld_u;
    a.cu = {u_codes, u_exps};
    if (act == NORMPRE_ACT_SWIGLU) {
        NP_CHECK(check_rows("up", up, ld_up, cols, e));
        NP_CHECK(check_held("up", up_codes, up_exps));
        a.up = up;
        a.ld_up = ld_up;
        a.cup = {up_codes, up_exps};
    }
    if (act != NORMPRE_ACT_NONE) {
        NP_CHECK(check_rows("h", h, ld_h, cols, e));
        NP_CHECK(check_held("h", h_codes, h_exps));
        a.h = h;
        a.ld_h = ld_h;
        a.ch = {h_codes, h_exps};
    }
    return launched(launch_ckpt_pack((DType)dtype, (Act)act, a, (hipStream_t)stream));
}

int normpre_checkpoint_unpack(int dtype, int64_t rows, int64_t cols, const int8_t* codes, const int8_t* exps,
                              void* out, int64_t ld_out, void* stream) {
    NP_CHECK(check_matrix(dtype, rows, cols));
    if (rows == 0) return NORMPRE_OK;
    NP_CHECK(check_held("x", codes, exps));
    NP_CHECK(check_rows("out", out, ld_out, cols, size_of(dtype)));
    const CkptUnpackArgs a{rows, cols, {codes, exps}, out, ld_out};
    return launched(launch_ckpt_unpack((DType)dtype, a, (hipStream_t)stream));
}

int normpre_checkpoint_act_grad(int act, int dtype, int64_t rows, int64_t cols, const void* dh, int64_t ld_dh,
                                const int8_t* u_codes, const int8_t* u_exps, const int8_t* up_codes,
                                const int8_t* up_exps, void* du, int64_t ld_du, void* dup, int64_t ld_dup,
                                void* stream) {
    if (act != NORMPRE_ACT_GELU && act != NORMPRE_ACT_SWIGLU)
        return fail(NORMPRE_ERR_INVALID_ARG, "no gradient of activation %d", act);
    NP_CHECK(check_matrix(dtype, rows, cols));
    if (rows == 0) return NORMPRE_OK;
    const int64_t e = size_of(dtype);
    CkptGradArgs a{};
    a.rows = rows;
    a.cols = cols;
    NP_CHECK(check_rows("dh", dh, ld_dh, cols, e));
    NP_CHECK(check_held("u", u_codes, u_exps));
    NP_CHECK(check_rows("du", du, ld_du, cols, e));
    a.dh = dh;
    a.ld_dh = ld_dh;
    a.cu = {u_codes, u_exps};
    a.du = du;
    a.ld_du = ld_du;
    if (act == NORMPRE_ACT_SWIGLU) {
        NP_CHECK(check_held("up", up_codes, up_exps));
        NP_CHECK(check_rows("dup", dup, ld_dup, cols, e));
        a.cup = {up_codes, up_exps};
        a.dup = dup;
        a.ld_dup = ld_dup;
    }
    return launched(launch_ckpt_act_grad((DType)dtype, (Act)act, a, (hipStream_t)stream));
}

static int check_weight(int dtype, int64_t tokens, int64_t inner, int64_t outer) {
    NP_CHECK(check_matrix(dtype, tokens, inner));
    NP_CHECK(check_matrix(dtype, tokens, outer));
    NP_CHECK(check_matrix(dtype, inner, outer));
    if (tokens > kMaxTokens || inner > kMaxFeatures || outer > kMaxFeatures)
        return fail(NORMPRE_ERR_UNSUPPORTED, "2^31 tokens or more, or more than 2^29 features");
    return NORMPRE_OK;
}

int normpre_checkpoint_weight_grad_workspace(int dtype, int64_t tokens, int64_t inner, int64_t outer,
                                             int64_t* bytes) {
    if (!bytes) return bad("bytes is null");
    NP_CHECK(check_weight(dtype, tokens, inner, outer));
    const int n = wgrad_splits((DType)dtype, tokens, inner, outer);
    *bytes = n > 1 ? 4 * inner * outer * n : 0;
    return NORMPRE_OK;
}

int normpre_checkpoint_weight_grad(int dtype, int layout, int accumulate, int64_t tokens, int64_t inner,
                                   int64_t outer, const int8_t* codes, const int8_t* exps, const void* dy,
                                   int64_t ld_dy, float* dw, int64_t ld_dw, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
    if (layout != NORMPRE_WEIGHT_INNER_OUTER && layout != NORMPRE_WEIGHT_OUTER_INNER)
        return fail(NORMPRE_ERR_INVALID_ARG, "unknown layout %d", layout);
    if (accumulate != 0 && accumulate != 1) return bad("accumulate is neither 0 nor 1");
    NP_CHECK(check_weight(dtype, tokens, inner, outer));
    if (tokens > 0) {
        NP_CHECK(check_held("x", codes, exps));
        NP_CHECK(check_rows("dy", dy, ld_dy, outer, size_of(dtype)));
    }
    const bool oi = layout == NORMPRE_WEIGHT_OUTER_INNER;
    NP_CHECK(check_rows("dw", dw, ld_dw, oi ? inner : outer, 4));
    WgradArgs a{};
    a.tokens = tokens;
    a.inner = inner;
    a.outer = outer;
    a.x = {codes, exps};
    a.dy = dy;
    a.ld_dy = ld_dy;
    a.dw = dw;
    a.ld_dw = ld_dw;
    a.oi = oi;
    a.accumulate = accumulate;
    a.splits = wgrad_splits((DType)dtype, tokens, inner, outer);
    if (a.splits > 1) {
        if (!workspace || !on(workspace, 16) || workspace_bytes < 4 * inner * outer * a.splits)
            return bad("workspace is null, misaligned or too small");
        a.partial = static_cast<float*>(workspace);
    }
    return launched(launch_wgrad((DType)dtype, a, (hipStream_t)stream));
}

}  // extern "C"
