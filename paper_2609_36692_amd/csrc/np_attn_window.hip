// Packed attention with a sliding window and first tokens that stay visible (sinks):
// which form of the passes (np_attn_passes.h) a call takes.
#include "np_attn_passes.h"

namespace np {
namespace {

template <class T, int DP, bool VEC>
hipError_t run(const AttnArgs& a, bool backward, hipStream_t s) {
    // As without a window.
    const int64_t blocks = (int64_t)a.num_tiles * a.heads;
    constexpr bool small = sizeof(T) == 2;
    if (!VEC || blocks > (small ? 512 : 448)) query_pass<T, DP, VEC, 4, 1, true>(a, backward, s);
    else if (small && blocks > 192) {
        if constexpr (small) query_pass<T, DP, true, 4, 2, true>(a, backward, s);
    } else query_pass<T, DP, true, 2, 2, true>(a, backward, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !backward) return e;
    const dim3 keys((unsigned)(a.num_tiles + a.sink_pieces) * a.kv_heads, a.splits);
    constexpr bool can_hold = VEC && sizeof(T) == 2 && DP == 128;
    if (can_hold && (int64_t)a.num_tiles * a.kv_heads >= 1024)
        attn_dkv_kernel<T, DP, VEC, can_hold, true><<<keys, kThreads, 0, s>>>(a);
    else attn_dkv_kernel<T, DP, VEC, false, true><<<keys, kThreads, 0, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const unsigned tiles = (unsigned)a.num_tiles * a.kv_heads, sinks = (unsigned)a.sink_tiles * a.kv_heads;
    if (a.splits == 1) {
        attn_odd_keys_kernel<T, DP, VEC, true><<<tiles, kThreads, 0, s>>>(a);
        if (sinks) attn_join_kernel<T, DP, true><<<dim3(sinks, DP / 8), kThreads, 0, s>>>(a);
    } else attn_join_kernel<T, DP, true><<<dim3(tiles, DP / 8), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t dispatch(const AttnArgs& a, bool backward, hipStream_t s) {
    const bool vec = whole_rows<T>(a, backward);
    if (a.dim <= 64) return vec ? run<T, 64, true>(a, backward, s) : run<T, 64, false>(a, backward, s);
    return vec ? run<T, 128, true>(a, backward, s) : run<T, 128, false>(a, backward, s);
}

}  // namespace

int window_splits(const AttnArgs& a) { return attention_splits(a.num_tiles, a.kv_heads); }

hipError_t launch_window_forward(DType t, const AttnArgs& a, hipStream_t s) {
    return t == DType::BF16 ? dispatch<bf16_t>(a, false, s) : dispatch<float>(a, false, s);
}

hipError_t launch_window_backward(DType t, const AttnArgs& a, hipStream_t s) {
    return t == DType::BF16 ? dispatch<bf16_t>(a, true, s) : dispatch<float>(a, true, s);
}

}  // namespace np
