// Host side of the norm and rotation of query and key heads of the C ABI
// (include/normpre.h): argument checks and the calls of the kernels' launchers.
#include "np_checks.h"
#include "np_rope.h"

#include <cmath>

using namespace np;

namespace {

int check_sizes(const normpre_qk_rope* a) {
    if (!a) return bad("the argument block is null");
    if (!known(a->dtype)) return fail(NORMPRE_ERR_INVALID_ARG, "unknown dtype %d", a->dtype);
    if (a->heads < 1 || a->kv_heads < 1) return fail(NORMPRE_ERR_INVALID_ARG, "%d and %d heads", a->heads, a->kv_heads);
    if (a->heads > kRopeMaxHeads || a->kv_heads > kRopeMaxHeads) return fail(NORMPRE_ERR_UNSUPPORTED, "more than 2^16 heads");
    if (a->head_dim < 1) return fail(NORMPRE_ERR_INVALID_ARG, "head_dim %d < 1", a->head_dim);
    if (a->head_dim > kRopeMaxDim) return fail(NORMPRE_ERR_UNSUPPORTED, "head_dim %d exceeds %d", a->head_dim, kRopeMaxDim);
    if (a->pairs < 0 || a->pairs > a->head_dim / 2)
        return fail(NORMPRE_ERR_INVALID_ARG, "%d pairs in heads of %d", a->pairs, a->head_dim);
    if (a->adjacent != 0 && a->adjacent != 1) return bad("adjacent is neither 0 nor 1");
    if (a->norm != 0 && a->norm != 1) return bad("norm is neither 0 nor 1");
    if (!(a->eps >= 0.0) || !std::isfinite(a->eps)) return bad("eps is negative or not finite");
    if (!known(a->weight_dtype)) return fail(NORMPRE_ERR_INVALID_ARG, "unknown weight_dtype %d", a->weight_dtype);
    if (a->tokens < 0) return bad("tokens < 0");
    if (a->tokens > kMaxTokens) return fail(NORMPRE_ERR_UNSUPPORTED, "2^31 tokens or more");
    return NORMPRE_OK;
}

RopeArgs sizes(const normpre_qk_rope* a) {
    RopeArgs k{};
    k.heads[0] = a->heads;
    k.heads[1] = a->kv_heads;
    k.dim = a->head_dim;
    k.inv_dim = 1.0 / a->head_dim;
    k.pairs = a->pairs;
    k.adjacent = a->adjacent;
    k.norm = a->norm;
    k.weight_bf16 = a->weight_dtype == NORMPRE_DTYPE_BF16;
    k.eps = a->eps;
    k.tokens = a->tokens;
    k.axis = a->pairs > 0 ? a->axes : nullptr;
    k.dw[0] = a->dq_weight;
    k.dw[1] = a->dk_weight;
    return k;
}

static_assert(4 * 2 * kRopeMostSums == 4096, "the header's bound");

int rope(const normpre_qk_rope* a, bool backward, void* stream) {
    NP_CHECK(check_sizes(a));
    RopeArgs k = sizes(a);
    if (!backward) k.dw[0] = k.dw[1] = nullptr;
    for (const float* dw : k.dw)
        if (dw && !on(dw, 4)) return bad("a weight gradient is misaligned");
    if (a->tokens == 0 && !(backward && rope_sums(k))) return NORMPRE_OK;
    const int64_t t = a->tokens, hq = a->heads, hk = a->kv_heads, d = a->head_dim, e = size_of(a->dtype);
    if (t > 0) {
        if (a->pairs > 0) {
            if (!a->freqs || !on(a->freqs, 8)) return bad("freqs is null or misaligned");
            if (a->axes && !on(a->axes, 4)) return bad("axes is misaligned");
            if (a->num_axes < 1) return bad("num_axes < 1");
            if (a->num_axes > kRopeMaxAxes) return fail(NORMPRE_ERR_UNSUPPORTED, "more than %d axes", kRopeMaxAxes);
            if (a->position_bytes != 4 && a->position_bytes != 8) return bad("positions have 4 or 8 bytes");
            if (!a->positions || !on(a->positions, a->position_bytes)) return bad("positions is null or misaligned");
            if (a->position_stride < 0) return bad("position_stride < 0");
            if (a->position_stride > kMaxStride) return fail(NORMPRE_ERR_UNSUPPORTED, "position_stride exceeds 2^40");
        }
        if (!backward || a->norm) {
            NP_CHECK(check_operand("q", a->q, t, hq, d, e, false));
            NP_CHECK(check_operand("k", a->k, t, hk, d, e, false));
        }
        NP_CHECK(check_operand("q_out", a->q_out, t, hq, d, e, !backward));
        NP_CHECK(check_operand("k_out", a->k_out, t, hk, d, e, !backward));
        if (backward) {
            NP_CHECK(check_operand("dq", a->dq, t, hq, d, e, true));
            NP_CHECK(check_operand("dk", a->dk, t, hk, d, e, true));
        }
        if (a->norm && (!on(a->q_weight, size_of(a->weight_dtype)) || !on(a->k_weight, size_of(a->weight_dtype))))
            return bad("a weight is misaligned");
    }
    k.x[0] = operand(a->q);
    k.x[1] = operand(a->k);
    k.y[0] = operand(backward ? a->dq : a->q_out);
    k.y[1] = operand(backward ? a->dk : a->k_out);
    if (backward) {
        k.g[0] = operand(a->q_out);
        k.g[1] = operand(a->k_out);
    }
    if (a->norm) {
        k.w[0] = a->q_weight;
        k.w[1] = a->k_weight;
    }
    k.freqs = a->freqs;
    k.axes = a->num_axes;
    k.positions = a->positions;
    k.positions_64 = a->position_bytes == 8;
    k.position_stride = a->position_stride;
    const DType dt = (DType)a->dtype;
    if (const int64_t need = backward ? 4 * rope_workspace(dt, k) : 0) {
        if (!a->workspace || !on(a->workspace, 16) || a->workspace_bytes < need)
            return bad("workspace is null, misaligned or too small");
        k.partial = static_cast<float*>(a->workspace);
    }
    return launched(launch_rope(dt, k, backward, (hipStream_t)stream));
}

}  // namespace

extern "C" {

int normpre_qk_rope_workspace(const normpre_qk_rope* a, int64_t* bytes) {
    if (!bytes) return bad("bytes is null");
    NP_CHECK(check_sizes(a));
    *bytes = 4 * rope_workspace((DType)a->dtype, sizes(a));
    return NORMPRE_OK;
}

int normpre_qk_rope_forward(const normpre_qk_rope* a, void* stream) { return rope(a, false, stream); }

int normpre_qk_rope_backward(const normpre_qk_rope* a, void* stream) { return rope(a, true, stream); }

}  // extern "C"
