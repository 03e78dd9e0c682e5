// Packed attention with a sliding window and first tokens that stay visible (sinks):
// query i sees the keys j <= i of its sequence with j > i - window or j < sinks.  The
// passes are those without a window (np_attn_passes.h, WIN): blocks of 128 queries go
// through the tiles of the first keys and then those from their first query's window on,
// blocks of 128 keys through the queries whose windows reach them, so that work grows with
// tokens x (window + sinks).  A block meets up to 127 rows more than each of its rows sees,
// and masks them on both sides.
//
// Measured (bf16, 16/8 heads of 128, window 1024, 4 first tokens; flops of the visible
// pairs): forward, 16964 tokens, 191-202 us (667-705 TFLOP/s); packed 15932 tokens: forward 165-178 us,
// dq 226-245, dk/dv 356-386, together 727-753 us (540-558).  Matrix instructions take 31 to 38% of the cycles,
// vector ones 41 to 56%.  What is lost against long causal rows (940-1000): the masked 11% of the pairs,
// each block's start and end over 19 tiles instead of a hundred, the last round of
// blocks (2160 on 512 places; dk/dv: 1112, 2.2 rounds that take three), and the masks' registers: forward 256
// at heads of 128 and 179 at heads of 64, where it has 208 and 124 without a window (of 64: two waves per SIMD
// instead of four), and dk/dv with v in LDS spills 8.
// 16 x 1024 tokens, bf16, 12 heads of 64, window 256: forward 38-41 us (300 TFLOP/s), dq 46, dk/dv 60; with 4 first
// tokens 40-44, 47, 74.
// 4 x 1024 tokens, fp32, 12 heads of 64, window 256: forward 40 us, dq 56, dk/dv 91: 384 blocks, so that half of
// the CUs have two and the others one, each a chain of up to 12 tiles that pass through registers and are split there;
// the pipes are 18 to 30% busy.  Forward and dq have two waves per SIMD (224 and 256 registers), dk/dv (337) one.
#include "np_attn_passes.h"

namespace np {
namespace {

template <class T, int DP, bool VEC>
hipError_t run(const AttnArgs& a, bool backward, hipStream_t s) {
    // Few blocks: their waves share the keys, and a block of 128 rows is cut in two.  Windows
    // make a block's chain of tiles short, so that this pays for fewer blocks than
    // without one.  Forward us of (4, 1), (4, 2), (2, 2):
    //   bf16, heads of 64, window 500, blocks of 128 rows 128: 22.3 18.1 13.4, 256: 22.7 18.7
    //     16.8, 320: 23.8 28.1 24.9, 512: 29.4 34.2 30.7; window 100, 256: 17.1 13.1 11.0, 320:
    //     18.7 22.9 17.9; window 1500, 320: 39.1 29.7 28.7, 448: 43.2 49.7 46.9
    //   bf16, 128, 500: 128: 27.1 23.2 18.9, 192: 28.0 23.7 35.0, 256: 28.5 24.5 35.2, 320: 32.4
    //     39.9 49.2
    //   fp32, (4, 1) and (2, 2), 64, 500: 256: 47.6 40.1, 320: 52.5 61.1; 128, 500: 128: 86.6
    //     52.6, 192: 92.7 100, 256: 96.8 103
    // The rule goes by blocks and head size alone; with a window of 1500 it takes (4, 1) at 320 blocks, a third
    // slower than (2, 2).  Rows that do not start on 16 bytes take (4, 1), as without a window.
    const int64_t blocks = (int64_t)a.num_tiles * a.heads;
    if constexpr (!VEC) query_pass<T, DP, VEC, 4, 1, true>(a, backward, s);
    else if (blocks <= (DP == 64 ? 256 : 128)) query_pass<T, DP, VEC, 2, 2, true>(a, backward, s);
    else if (DP == 128 && sizeof(T) == 2 && blocks <= 256) {
        if constexpr (DP == 128 && sizeof(T) == 2) query_pass<T, DP, VEC, 4, 2, true>(a, backward, s);
    } else query_pass<T, DP, VEC, 4, 1, true>(a, backward, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !backward) return e;
    const dim3 keys((unsigned)(a.num_tiles + a.sink_pieces) * a.kv_heads, a.splits);
    // bf16 heads of 128: with v's rows in LDS two blocks fit a CU instead of one, which pays
    // once there are more of them than CUs.  Backward us with them there / in registers
    // (16/8 heads; blocks x shares): window 300: 64 x 1 111 / 103, 128 x 2 92 / 112, 256 x 1 155 / 180,
    // 512 x 1 256 / 283, 1024 x 1 442 / 567; window 1000: 128 x 2 180 / 164, 512 x 1 393 / 421, 1024 x 1
    // 718 / 834.  By blocks x shares alone: at 128 x 2 and a window of 1000 it takes the slower one.
    constexpr bool can_hold = VEC && sizeof(T) == 2 && DP == 128;
    if (can_hold && (int64_t)a.num_tiles * a.kv_heads * a.splits >= 256)
        attn_dkv_kernel<T, DP, VEC, can_hold, true><<<keys, kThreads, 0, s>>>(a);
    else attn_dkv_kernel<T, DP, VEC, false, true><<<keys, kThreads, 0, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const unsigned tiles = (unsigned)a.num_tiles * a.kv_heads, sinks = (unsigned)a.sink_tiles * a.kv_heads;
    if (a.splits == 1) {
        attn_odd_keys_kernel<T, DP, VEC, true><<<tiles, kThreads * kOddWaves<true>, 0, s>>>(a);
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

// Shares of the queries in the dk/dv pass.  Windows bound a block's steps (of 64 queries, us
// each), so that more shares soon cost more, in partial sums written and read (`sums` us
// for a block's share), than the shorter chain gives; `at_once` blocks run side by side.  Backward us of
// 1, 2, 4 shares, blocks of 128 keys and window:
//   bf16, heads of 64, one query head a key head: 64, 300: 54.9 38.7 35.3; 128, 60: 45.3 38.4 46.5;
//     192, 60: 48.5 51.8 55.9; 256, 300: 66.0 64.1 71.0; 384, 300: 76.0 83.8 97.7; 384, 1000: 141 112 124;
//     1024, 1000: 236 255 317; four: 128, 300: 159 105 96; 256, 1000: 431 284 249
//   bf16, 128, two: 64, 300: 103 71 64; 192, 300: 133 110 126; 256, 60: 113 121 135; 384, 1000: 350 310 324;
//     1024, 300: 442 551 679
//   fp32, 64, one: 64, 1000: 165 116 95; 256, 60: 113 121 143; 128, two: 64, 300: 281 184 179; 512, 60: 694 781 886
int window_splits(DType t, const AttnArgs& a) {
    const bool small = a.dim <= 64, bf16 = t == DType::BF16;
    const double step = bf16 ? (small ? 4.3 : 4.9) : small ? 8.0 : 14.0;
    const double sums = bf16 ? (small ? 0.025 : 0.04) : small ? 0.035 : 0.08;
    const double blocks = (double)a.num_tiles * a.kv_heads, at_once = bf16 ? 512 : 256;
    const int64_t rows = (a.window < a.tokens ? a.window : a.tokens) + kAttnRows - 1;
    const double steps = (double)((rows + 63) / 64) * (a.heads / a.kv_heads);
    int best = 1;
    double least = 0;
    for (int s = 1; s <= 4; s *= 2) {
        const double rounds = blocks * s > at_once ? blocks * s / at_once : 1.0;
        const double us = rounds * steps / s * step + (s > 1 ? sums * blocks * s : 0.0);
        if (s == 1 || us < least) {
            best = s;
            least = us;
        }
    }
    return best;
}

hipError_t launch_window_forward(DType t, const AttnArgs& a, hipStream_t s) {
    return t == DType::BF16 ? dispatch<bf16_t>(a, false, s) : dispatch<float>(a, false, s);
}

hipError_t launch_window_backward(DType t, const AttnArgs& a, hipStream_t s) {
    return t == DType::BF16 ? dispatch<bf16_t>(a, true, s) : dispatch<float>(a, true, s);
}

}  // namespace np
