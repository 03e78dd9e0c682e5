// Argument checks that the host sides of the training-step operators share.
#pragma once

#include "../../include/normpre.h"
#include "np_internal.h"
#include "np_train.h"

#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

namespace np {
namespace {

constexpr int64_t kMaxTokens = INT32_MAX;
constexpr int64_t kMaxStride = int64_t(1) << 40;
// A launch holds fewer than 2^32 threads a dimension: blocks of up to 512, and
// eight elements a thread.
constexpr int64_t kMaxElements = int64_t(1) << 34;
constexpr int64_t kMaxBlocks = (int64_t(1) << 23) - 1;
constexpr int64_t kMaxFeatures = int64_t(1) << 29;

inline int fail(int code, const char* f, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, f);
    vsnprintf(buf, sizeof buf, f, ap);
    va_end(ap);
    return set_thread_error(code, buf);
}

inline int bad(const char* what) { return fail(NORMPRE_ERR_INVALID_ARG, "%s", what); }

inline int launched(hipError_t e) {
    return e == hipSuccess ? NORMPRE_OK : fail(NORMPRE_ERR_HIP, "launch: %s", hipGetErrorString(e));
}

inline bool known(int dtype) { return dtype == NORMPRE_DTYPE_F32 || dtype == NORMPRE_DTYPE_BF16; }
inline int64_t size_of(int dtype) { return dtype == NORMPRE_DTYPE_BF16 ? 2 : 4; }
inline bool on(const void* p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes == 0; }

inline int check_operand(const char* name, const normpre_heads& o, int64_t tokens, int64_t heads, int64_t dim, int64_t elt,
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

inline AttnOperand operand(const normpre_heads& o) { return {o.data, o.token_stride, o.head_stride}; }

#define NP_CHECK(call)                            \
    do {                                          \
        const int rc_ = (call);                   \
        if (rc_ != NORMPRE_OK) return rc_;        \
    } while (0)

// ----------------------------------------------------------- attention ---
// Number of tiles of 128 rows and of tokens.
inline int count_tiles(int64_t num_seqs, const int64_t* lens, int64_t& tiles, int64_t& tokens) {
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

inline int check_attention_sizes(const normpre_attention* a) {
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

inline AttnArgs attention_sizes(const normpre_attention* a) {
    AttnArgs k{};
    k.num_tiles = (int)a->num_tiles;
    k.tokens = a->tokens;
    k.heads = a->heads;
    k.kv_heads = a->kv_heads;
    k.dim = a->head_dim;
    return k;
}

// All but the workspace.
inline int check_attention(const normpre_attention* a, bool backward) {
    NP_CHECK(check_attention_sizes(a));
    if (a->tokens == 0) return NORMPRE_OK;
    if (!a->plan || !on(a->plan, 16)) return bad("plan is null or not 16-byte aligned");
    if (!a->lse || !on(a->lse, 4)) return bad("lse is null or misaligned");
    const int64_t t = a->tokens, hq = a->heads, hk = a->kv_heads, d = a->head_dim, e = size_of(a->dtype);
    NP_CHECK(check_operand("q", a->q, t, hq, d, e, false));
    NP_CHECK(check_operand("k", a->k, t, hk, d, e, false));
    NP_CHECK(check_operand("v", a->v, t, hk, d, e, false));
    NP_CHECK(check_operand("out", a->out, t, hq, d, e, !backward));
    if (backward) {
        NP_CHECK(check_operand("dout", a->dout, t, hq, d, e, false));
        NP_CHECK(check_operand("dq", a->dq, t, hq, d, e, true));
        NP_CHECK(check_operand("dk", a->dk, t, hk, d, e, true));
        NP_CHECK(check_operand("dv", a->dv, t, hk, d, e, true));
    }
    return NORMPRE_OK;
}

inline void attention_operands(const normpre_attention* a, bool backward, AttnArgs& k) {
    k.q = operand(a->q);
    k.k = operand(a->k);
    k.v = operand(a->v);
    k.out = operand(a->out);
    k.lse = a->lse;
    k.tiles = reinterpret_cast<const AttnTile*>(a->plan);
    k.causal = a->causal;
    k.scale = a->scale;
    if (!backward) return;
    k.dout = operand(a->dout);
    k.dq = operand(a->dq);
    k.dk = operand(a->dk);
    k.dv = operand(a->dv);
}

// The parts of a backward call's workspace.
inline void attention_parts(float* ws, AttnArgs& k) {
    const int64_t rows = (int64_t)k.heads * k.tokens;
    k.lse2 = ws;
    k.delta = ws + rows;
    k.partial = ws + (2 * rows + 3) / 4 * 4;
    k.odd = reinterpret_cast<uint32_t*>(k.partial);
}

}  // namespace
}  // namespace np
