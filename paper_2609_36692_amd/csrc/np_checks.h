// Argument checks that the host sides of the training-step operators share.
#pragma once

#include "../../include/normpre.h"
#include "np_internal.h"
#include "np_train.h"

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

}  // namespace
}  // namespace np
