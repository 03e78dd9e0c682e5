// Driver for the sanitized build of the training-step operators' host code
// (tests/test_train_abi_sanitized.py): plans of packed batches and every
// refusal, with launchers that only count their calls.
#include "../include/normpre.h"
#include "../paper_2609_36692_amd/csrc/np_train.h"

#include <cstdio>
#include <limits>
#include <string>
#include <vector>

static int g_launches = 0, g_failures = 0;
static std::string g_error;

namespace np {
int set_thread_error(int code, const char* msg) { g_error = msg; return code; }
hipError_t launch_attention_forward(DType, const AttnArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_attention_backward(DType, const AttnArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
int attention_splits(int64_t, int) { return 2; }
int64_t attention_workspace(const AttnArgs& a) { return 2 * (int64_t)a.heads * a.tokens; }
hipError_t launch_ckpt_pack(DType, Act, const CkptPackArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_ckpt_unpack(DType, const CkptUnpackArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_ckpt_act_grad(DType, Act, const CkptGradArgs&, hipStream_t) { ++g_launches; return hipSuccess; }
hipError_t launch_wgrad(DType, const WgradArgs&, hipStream_t) { ++g_launches; return hipErrorInvalidValue; }
int wgrad_splits(DType, int64_t tokens, int64_t, int64_t) { return tokens > 1000 ? 3 : 1; }
}  // namespace np

#define EXPECT(got, want)                                                                              \
    do {                                                                                               \
        const long long g_ = (long long)(got), w_ = (long long)(want);                                 \
        if (g_ != w_) {                                                                                \
            std::printf("line %d: %s is %lld, expected %lld (%s)\n", __LINE__, #got, g_, w_, g_error.c_str()); \
            ++g_failures;                                                                              \
        }                                                                                              \
    } while (0)

int main() {
    const int64_t huge = std::numeric_limits<int64_t>::max();
    // Plans: exactly the tiles counted, into a buffer of exactly that size.
    for (const std::vector<int64_t>& lens : {std::vector<int64_t>{}, {0}, {1}, {128, 129, 0, 4000}, std::vector<int64_t>(999, 3)}) {
        int64_t n = -1;
        EXPECT(normpre_attention_plan_tiles((int64_t)lens.size(), lens.data(), &n), NORMPRE_OK);
        std::vector<int32_t> plan(8 * n);
        for (int causal = 0; causal < 2; ++causal)
            EXPECT(normpre_attention_plan((int64_t)lens.size(), lens.data(), causal, plan.data(), 8 * n), NORMPRE_OK);
        if (n) EXPECT(normpre_attention_plan((int64_t)lens.size(), lens.data(), 1, plan.data(), 8 * n - 1), NORMPRE_ERR_INVALID_ARG);
    }
    int64_t n = 0, bad[2] = {huge, huge};
    EXPECT(normpre_attention_plan_tiles(2, bad, &n), NORMPRE_ERR_UNSUPPORTED);
    EXPECT(normpre_attention_plan_tiles(huge, nullptr, &n), NORMPRE_ERR_INVALID_ARG);

    alignas(16) static char mem[64];
    normpre_attention a{};
    a.dtype = NORMPRE_DTYPE_BF16;
    a.heads = 4;
    a.kv_heads = 2;
    a.head_dim = 64;
    a.causal = 1;
    a.scale = 1.f;
    a.tokens = 100;
    a.plan = reinterpret_cast<int32_t*>(mem);
    a.num_tiles = 1;
    a.q = a.out = a.dout = a.dq = {mem, 256, 64};
    a.k = a.v = a.dk = a.dv = {mem, 128, 64};
    a.lse = reinterpret_cast<float*>(mem);
    a.workspace = mem;
    EXPECT(normpre_attention_workspace(&a, &a.workspace_bytes), NORMPRE_OK);
    EXPECT(a.workspace_bytes, 4 * 2 * 4 * 100);
    EXPECT(normpre_attention_forward(&a, nullptr), NORMPRE_OK);
    EXPECT(normpre_attention_backward(&a, nullptr), NORMPRE_OK);
    EXPECT(g_launches, 2);
    EXPECT(normpre_attention_forward(nullptr, nullptr), NORMPRE_ERR_INVALID_ARG);
    normpre_attention b = a;
    b.q.token_stride = b.q.head_stride = huge;
    EXPECT(normpre_attention_forward(&b, nullptr), NORMPRE_ERR_UNSUPPORTED);
    b = a;
    b.out.token_stride = huge;
    EXPECT(normpre_attention_forward(&b, nullptr), NORMPRE_ERR_UNSUPPORTED);
    b = a;
    b.tokens = b.num_tiles = std::numeric_limits<int32_t>::max();
    b.heads = b.kv_heads = std::numeric_limits<int32_t>::max();
    EXPECT(normpre_attention_forward(&b, nullptr), NORMPRE_ERR_UNSUPPORTED);
    b = a;
    b.num_tiles = huge;
    EXPECT(normpre_attention_forward(&b, nullptr), NORMPRE_ERR_INVALID_ARG);
    b = a;
    b.heads = std::numeric_limits<int32_t>::min();
    EXPECT(normpre_attention_backward(&b, nullptr), NORMPRE_ERR_INVALID_ARG);
    EXPECT(g_launches, 2);

    int8_t* c = reinterpret_cast<int8_t*>(mem);
    EXPECT(normpre_checkpoint_pack(NORMPRE_ACT_SWIGLU, 1, 3, 70, mem, 70, mem, 70, mem, 70, c, c, c, c, c, c, nullptr), NORMPRE_OK);
    EXPECT(normpre_checkpoint_pack(NORMPRE_ACT_NONE, 0, 3, 70, mem, 70, nullptr, 0, nullptr, 0, c, c, nullptr, nullptr, nullptr, nullptr, nullptr), NORMPRE_OK);
    EXPECT(normpre_checkpoint_pack(NORMPRE_ACT_GELU, 1, huge, huge, mem, huge, mem, 70, mem, huge, c, c, c, c, c, c, nullptr), NORMPRE_ERR_UNSUPPORTED);
    EXPECT(normpre_checkpoint_pack(NORMPRE_ACT_GELU, 1, 3, huge - 1, mem, huge, mem, 70, mem, huge, c, c, c, c, c, c, nullptr), NORMPRE_ERR_UNSUPPORTED);
    EXPECT(normpre_checkpoint_unpack(1, 3, 70, c, c, mem, 70, nullptr), NORMPRE_OK);
    EXPECT(normpre_checkpoint_unpack(1, 3, 70, c + 1, c, mem, 70, nullptr), NORMPRE_ERR_INVALID_ARG);
    EXPECT(normpre_checkpoint_act_grad(NORMPRE_ACT_GELU, 1, 3, 70, mem, 70, c, c, nullptr, nullptr, mem, 70, nullptr, 0, nullptr), NORMPRE_OK);
    EXPECT(normpre_checkpoint_act_grad(NORMPRE_ACT_SWIGLU, 1, 3, 70, mem, 70, c, c, nullptr, nullptr, mem, 70, nullptr, 0, nullptr), NORMPRE_ERR_INVALID_ARG);
    EXPECT(g_launches, 6);
    int64_t bytes = -1;
    EXPECT(normpre_checkpoint_weight_grad_workspace(1, 2000, 64, 64, &bytes), NORMPRE_OK);
    EXPECT(bytes, 3 * 64 * 64 * 4);
    EXPECT(normpre_checkpoint_weight_grad_workspace(1, huge, huge, huge, &bytes), NORMPRE_ERR_UNSUPPORTED);
    // A launch that fails is reported.
    float* f = reinterpret_cast<float*>(mem);
    EXPECT(normpre_checkpoint_weight_grad(1, 0, 0, 10, 64, 64, c, c, mem, 64, f, 64, nullptr, 0, nullptr), NORMPRE_ERR_HIP);
    EXPECT(normpre_checkpoint_weight_grad(1, 1, 1, 2000, 64, 64, c, c, mem, 64, f, 64, mem, bytes, nullptr), NORMPRE_ERR_HIP);
    EXPECT(normpre_checkpoint_weight_grad(1, 1, 1, 2000, 64, 64, c, c, mem, 64, f, 64, mem, 100, nullptr), NORMPRE_ERR_INVALID_ARG);
    std::printf("%d failure(s)\n", g_failures);
    return g_failures != 0;
}
