// Host side of the training-step operators of the C ABI (include/normpre.h):
// argument checks, the plan of a packed batch, and the calls of the kernels'
// launchers.  Nothing here keeps state or computes results on the host.
#include "../../include/normpre.h"
#include "np_internal.h"
#include "np_train.h"

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>
#include <vector>

using namespace np;

namespace {

constexpr int64_t kMaxTokens = INT32_MAX;
constexpr int64_t kMaxStride = int64_t(1) << 40;
// A launch holds fewer than 2^32 threads a dimension: blocks of up to 512, and
// eight elements a thread.
constexpr int64_t kMaxElements = int64_t(1) << 34;
constexpr int64_t kMaxBlocks = (int64_t(1) << 23) - 1;
constexpr int64_t kMaxFeatures = int64_t(1) << 29;

int fail(int code, const char* f, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, f);
    vsnprintf(buf, sizeof buf, f, ap);
    va_end(ap);
    return set_thread_error(code, buf);
}

int bad(const char* what) { return fail(NORMPRE_ERR_INVALID_ARG, "%s", what); }

int launched(hipError_t e) {
    return e == hipSuccess ? NORMPRE_OK : fail(NORMPRE_ERR_HIP, "launch: %s", hipGetErrorString(e));
}

bool known(int dtype) { return dtype == NORMPRE_DTYPE_F32 || dtype == NORMPRE_DTYPE_BF16; }
int64_t size_of(int dtype) { return dtype == NORMPRE_DTYPE_BF16 ? 2 : 4; }
bool on(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

// ----------------------------------------------------------- attention ---
// Number of tiles of 128 rows and of tokens; false: error set.
int count(int64_t num_seqs, const int64_t* lens, int64_t& tiles, int64_t& tokens) {
    if (num_seqs < 0) return bad("num_seqs < 0");
    if (num_seqs > 0 && !lens) return bad("lens is null");
    tiles = tokens = 0;
    for (int64_t i = 0; i < num_seqs; ++i) {
        if (lens[i] < 0) return fail(NORMPRE_ERR_INVALID_ARG, "sequence %lld has a negative length", (long long)i);
        if (lens[i] > kMaxTokens - tokens) return fail(NORMPRE_ERR_UNSUPPORTED, "2^31 tokens or more");
        tokens += lens[i];
        tiles += (lens[i] + kAttnRows - 1) / kAttnRows;
    }
    return NORMPRE_OK;
}

int check_operand(const char* name, const normpre_heads& o, int64_t tokens, int64_t heads, int64_t dim, int64_t elt,
                  bool written) {
    if (!o.data) return fail(NORMPRE_ERR_INVALID_ARG, "%s is null", name);
    if (!on(o.data, elt)) return fail(NORMPRE_ERR_INVALID_ARG, "%s is not aligned to its elements", name);
    if (o.token_stride < 0 || o.head_stride < 0) return fail(NORMPRE_ERR_INVALID_ARG, "%s has a negative stride", name);
    if (o.token_stride > kMaxStride || o.head_stride > kMaxStride)
        return fail(NORMPRE_ERR_UNSUPPORTED, "a stride of %s exceeds 2^40", name);
    if (written) {
        // Rows of one token side by side, or rows of one head (a stride that
        // is never taken does not matter).  heads < 2^23 and strides to 2^40 keep the
        // first product within 64 bits, 2^31 tokens would not the second.
        const int64_t t = tokens > 1 ? o.token_stride : 0, h = heads > 1 ? o.head_stride : 0;
        const bool by_token = (heads == 1 || h >= dim) && (tokens == 1 || t >= (heads - 1) * h + dim);
        const bool by_head = (tokens == 1 || t >= dim) && (heads == 1 || (h >= dim && (tokens == 1 || (h - dim) / (tokens - 1) >= t)));
        if (!by_token && !by_head) return fail(NORMPRE_ERR_INVALID_ARG, "rows of %s overlap", name);
    }
    return NORMPRE_OK;
}

AttnOperand operand(const normpre_heads& o) { return {o.data, o.token_stride, o.head_stride}; }

int check_sizes(const normpre_attention* a) {
    if (!a) return bad("the argument block is null");
    if (!known(a->dtype)) return fail(NORMPRE_ERR_INVALID_ARG, "unknown dtype %d", a->dtype);
    if (a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads)
        return fail(NORMPRE_ERR_INVALID_ARG, "%d heads over %d key heads", a->heads, a->kv_heads);
    if (a->head_dim < 1) return fail(NORMPRE_ERR_INVALID_ARG, "head_dim %d < 1", a->head_dim);
    if (a->head_dim > kAttnMaxDim)
        return fail(NORMPRE_ERR_UNSUPPORTED, "head_dim %d exceeds %d", a->head_dim, kAttnMaxDim);
    if (a->causal != 0 && a->causal != 1) return bad("causal is neither 0 nor 1");
    if (!std::isfinite(a->scale)) return bad("scale must be finite");
    if (a->tokens < 0 || a->num_tiles < 0) return bad("tokens < 0 or num_tiles < 0");
    if (a->tokens > kMaxTokens) return fail(NORMPRE_ERR_UNSUPPORTED, "2^31 tokens or more");
    // Every token lies in one tile, and no tile is empty.
    if (a->num_tiles > a->tokens || a->num_tiles * kAttnRows < a->tokens)
        return fail(NORMPRE_ERR_INVALID_ARG, "%lld tiles cannot hold %lld tokens", (long long)a->num_tiles,
                    (long long)a->tokens);
    if (a->num_tiles * a->heads > kMaxBlocks) return fail(NORMPRE_ERR_UNSUPPORTED, "more than 2^23 - 1 blocks of 128 rows");
    return NORMPRE_OK;
}

// The sizes alone, with what the backward pass makes of them.
AttnArgs sizes(const normpre_attention* a) {
    AttnArgs k{};
    k.num_tiles = (int)a->num_tiles;
    k.tokens = a->tokens;
    k.heads = a->heads;
    k.kv_heads = a->kv_heads;
    k.dim = a->head_dim;
    k.splits = attention_splits(a->num_tiles, a->kv_heads);
    return k;
}

int attention(const normpre_attention* a, bool backward, void* stream) {
    const int sized = check_sizes(a);
    if (sized != NORMPRE_OK) return sized;
    if (a->tokens == 0) return NORMPRE_OK;
    if (!a->plan || !on(a->plan, 16)) return bad("plan is null or not 16-byte aligned");
    if (!a->lse || !on(a->lse, 4)) return bad("lse is null or misaligned");
    const int64_t t = a->tokens, hq = a->heads, hk = a->kv_heads, d = a->head_dim, e = size_of(a->dtype);
    int rc = NORMPRE_OK;
    auto operand_ok = [&](const char* n, const normpre_heads& o, int64_t h, bool w) {
        if (rc == NORMPRE_OK) rc = check_operand(n, o, t, h, d, e, w);
    };
    operand_ok("q", a->q, hq, false);
    operand_ok("k", a->k, hk, false);
    operand_ok("v", a->v, hk, false);
    operand_ok("out", a->out, hq, !backward);
    if (backward) {
        operand_ok("dout", a->dout, hq, false);
        operand_ok("dq", a->dq, hq, true);
        operand_ok("dk", a->dk, hk, true);
        operand_ok("dv", a->dv, hk, true);
    }
    if (rc != NORMPRE_OK) return rc;

    AttnArgs k = sizes(a);
    k.q = operand(a->q);
    k.k = operand(a->k);
    k.v = operand(a->v);
    k.out = operand(a->out);
    k.lse = a->lse;
    k.tiles = reinterpret_cast<const AttnTile*>(a->plan);
    k.causal = a->causal;
    k.scale = a->scale;
    const DType dt = (DType)a->dtype;
    if (!backward) return launched(launch_attention_forward(dt, k, (hipStream_t)stream));
    k.dout = operand(a->dout);
    k.dq = operand(a->dq);
    k.dk = operand(a->dk);
    k.dv = operand(a->dv);
    float* ws = static_cast<float*>(a->workspace);
    if (!ws || !on(ws, 16) || a->workspace_bytes < 4 * attention_workspace(k))
        return bad("workspace is null, misaligned or too small");
    const int64_t rows = (int64_t)a->heads * a->tokens;
    k.lse2 = ws;
    k.delta = ws + rows;
    k.partial = ws + (2 * rows + 3) / 4 * 4;
    k.odd = reinterpret_cast<uint32_t*>(k.partial);
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

#define NP_CHECK(call)                            \
    do {                                          \
        const int rc_ = (call);                   \
        if (rc_ != NORMPRE_OK) return rc_;        \
    } while (0)

}  // namespace

extern "C" {

int normpre_attention_plan_tiles(int64_t num_seqs, const int64_t* lens, int64_t* num_tiles) {
    if (!num_tiles) return bad("num_tiles is null");
    int64_t tiles, tokens;
    NP_CHECK(count(num_seqs, lens, tiles, tokens));
    *num_tiles = tiles;
    return NORMPRE_OK;
}

int normpre_attention_plan(int64_t num_seqs, const int64_t* lens, int causal, int32_t* plan, int64_t capacity) {
    int64_t n, tokens;
    NP_CHECK(count(num_seqs, lens, n, tokens));
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
    NP_CHECK(check_sizes(a));
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
