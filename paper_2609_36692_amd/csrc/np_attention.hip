// Packed attention, causal or full: which form of the passes (np_attn_passes.h) a call
// takes.
#include "np_attn_passes.h"

namespace np {
namespace {

// -------------------------------------------------------------- launches ---
template <class T, int DP, bool VEC>
hipError_t run(const AttnArgs& a, bool backward, hipStream_t s) {
    // Few blocks: their waves share the keys, so that a block's chain of tiles is
    // half as long, and up to 192 (fp32: 448) of 128 rows they are cut in two.
    // Many blocks: one team, whose blocks run out of step, so that one's softmax
    // meets the other's products.  Forward us of (4, 1), (4, 2), (2, 2):
    //   bf16, heads of 64, blocks of 128 rows 96: 19.5 15.6 12.6, 192: 19.9 16.3 15.1,
    //     288: 20.6 16.5 16.9, 384: 20.9 17.7 18.3, 576: 22.6 26.6 26.2, 960: 31.6 40.5 40.2
    //   bf16, 128: 256: 47.0 39.0 42.1, 512: 55.4 49.3 84.5, 768: 68.0 78.8 130
    //   fp32, 64, (4, 1) and (2, 2): 96: 62 44, 384: 66 54, 768: 86 99, 1536: 159 187
    //   fp32, 128: 128: 127 73, 256: 263 158, 512: 275 297, 1024: 402 593
    // Rows that do not start on 16 bytes take (4, 1) whatever the batch, so that two
    // more forms of each pass need not be built.  Forward us of aligned rows, of others
    // and of others by the rule above: bf16 heads of 64, 1024 tokens of 12 heads 13 30
    // 22, 4 x 1024 20 37 31; fp32 42 62 43, 57 67 55; bf16 128, 2 x 1024 of 16/8 24 47 41.
    const int64_t blocks = (int64_t)a.num_tiles * a.heads;
    constexpr bool small = sizeof(T) == 2;
    if (!VEC || blocks > (small ? 512 : 448)) query_pass<T, DP, VEC, 4, 1, false>(a, backward, s);
    else if (small && blocks > 192) {
        if constexpr (small) query_pass<T, DP, true, 4, 2, false>(a, backward, s);
    } else query_pass<T, DP, true, 2, 2, false>(a, backward, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !backward) return e;
    // bf16 heads of 128: with v's rows in LDS two blocks fit a CU instead of one,
    // for more LDS reads and half tiles.  us with them there / in registers: packed
    // 16418 tokens (1032 blocks) 827 / 873, 16 x 2048 (2048) 1146 / 1254, 4 x 8192
    // (2048) 3890 / 4195; 4 x 2048 (512) 338 / 295, 2 x 2048 (256) 222 / 183.
    const dim3 keys((unsigned)a.num_tiles * a.kv_heads, a.splits);
    constexpr bool can_hold = VEC && sizeof(T) == 2 && DP == 128;
    if (can_hold && (int64_t)a.num_tiles * a.kv_heads >= 1024)
        attn_dkv_kernel<T, DP, VEC, can_hold, false><<<keys, kThreads, 0, s>>>(a);
    else attn_dkv_kernel<T, DP, VEC, false, false><<<keys, kThreads, 0, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.splits == 1) attn_odd_keys_kernel<T, DP, VEC, false><<<keys, kThreads, 0, s>>>(a);
    else attn_join_kernel<T, DP, false><<<dim3((unsigned)a.num_tiles * a.kv_heads, DP / 8), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t dispatch(const AttnArgs& a, bool backward, hipStream_t s) {
    const bool vec = whole_rows<T>(a, backward);
    if (a.dim <= 64) return vec ? run<T, 64, true>(a, backward, s) : run<T, 64, false>(a, backward, s);
    return vec ? run<T, 128, true>(a, backward, s) : run<T, 128, false>(a, backward, s);
}

}  // namespace

// Shares of the queries in the dk/dv pass: enough blocks for two on every CU, at
// most 4, since the partial sums of a share are written and read once more.
// Backward us of 1, 2, 4, 8 shares: 64 blocks (heads of 64, 32 over 8) 48.8 35.3
// 27.4 28.0; 128 (the same) 240 152 124 123; 256 (128, 16 over 8) 445 341 365 429;
// 1536 (64, 12) 137 223 310 483.
int attention_splits(int64_t num_tiles, int kv_heads) {
    const int64_t blocks = num_tiles * kv_heads;
    return blocks >= 512 ? 1 : blocks >= 256 ? 2 : 4;
}

int64_t attention_workspace(const AttnArgs& a) {
    const int64_t rows = 2 * (int64_t)a.heads * a.tokens, pitch = a.dim <= 64 ? 64 : 128;
    return (rows + 3) / 4 * 4 + (a.splits > 1 ? 2 * a.splits * (int64_t)a.kv_heads * a.tokens * pitch
                                              : (int64_t)kAttnRows / 32 * a.num_tiles * a.kv_heads);
}

hipError_t launch_attention_forward(DType t, const AttnArgs& a, hipStream_t s) {
    return t == DType::BF16 ? dispatch<bf16_t>(a, false, s) : dispatch<float>(a, false, s);
}

hipError_t launch_attention_backward(DType t, const AttnArgs& a, hipStream_t s) {
    return t == DType::BF16 ? dispatch<bf16_t>(a, true, s) : dispatch<float>(a, true, s);
}

}  // namespace np
