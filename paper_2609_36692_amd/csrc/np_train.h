// Internal declarations of the training-step operators (packed attention,
// 8-bit activation checkpoints): launchers shared by their host side
// (np_train_api.cpp) and their kernels.  Not part of the public ABI.
#pragma once

#include "np_attn_tile.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace np {

enum class DType { F32 = 0, BF16 = 1 };

// ----------------------------------------------------------- attention ---
constexpr int kAttnMaxDim = 128;

// One [tokens, heads, dim] operand; strides in elements, dim contiguous.
struct AttnOperand {
    void* p;
    int64_t tok, head;
};

struct AttnArgs {
    AttnOperand q, k, v, out, dout, dq, dk, dv;
    float* lse;                 // [heads][tokens], natural logarithms
    float* lse2;                // backward workspace, [heads][tokens] each: lse in
    float* delta;               // base 2, and delta
    float* partial;             // [splits][2][kv_heads][tokens][64 or 128], splits > 1
    uint32_t* odd;              // splits = 1: rows of dk and dv that are not finite, a
                                // bit each, [num_tiles][kv_heads][4], in its place
    int splits;                 // shares of a key's queries (dk/dv pass)
    const AttnTile* tiles;      // query tiles, then as many key tiles
    int num_tiles;
    int64_t tokens;
    int heads, kv_heads, dim, causal;
    float scale;
    // Sliding window (launch_window_*): query i sees keys j <= i with j > i - window or
    // j < sinks.
    int window, sinks;
    int sink_tiles, sink_pieces;    // entries of the plan behind its tiles (AttnSink, AttnPiece)
    int sink_rows;              // rows of a key tile that may be sinks, whole waves: 32 .. 128
    float* first_keys;          // [sink_pieces + sink_tiles][splits][2][kv_heads][sink_rows][64 or 128]
};

// Shares into which the dk/dv pass cuts the queries of a key, and the floats of
// workspace that a backward call needs (lse2 and delta, then the partial sums or odd).
int attention_splits(int64_t num_tiles, int kv_heads);
int64_t attention_workspace(const AttnArgs& a);
hipError_t launch_attention_forward(DType t, const AttnArgs& a, hipStream_t s);
hipError_t launch_attention_backward(DType t, const AttnArgs& a, hipStream_t s);

// The same with a sliding window; the workspace is that of a call without one, then
// first_keys.
int window_splits(DType t, const AttnArgs& a);
hipError_t launch_window_forward(DType t, const AttnArgs& a, hipStream_t s);
hipError_t launch_window_backward(DType t, const AttnArgs& a, hipStream_t s);

// --------------------------------------------------------- checkpoints ---
constexpr int kCkptGroup = 64;          // features that share an exponent
inline int64_t ckpt_pitch(int64_t cols) { return (cols + kCkptGroup - 1) / kCkptGroup * kCkptGroup; }

struct CkptOut { int8_t* codes; int8_t* exps; };
struct CkptIn { const int8_t* codes; const int8_t* exps; };

enum class Act { None = 0, Gelu = 1, Swiglu = 2 };

struct CkptPackArgs {
    int64_t rows, cols;
    const void* u; int64_t ld_u;
    const void* up; int64_t ld_up;
    void* h; int64_t ld_h;
    CkptOut cu, cup, ch;
};
hipError_t launch_ckpt_pack(DType t, Act act, const CkptPackArgs& a, hipStream_t s);

struct CkptUnpackArgs {
    int64_t rows, cols;
    CkptIn c;
    void* out; int64_t ld;
};
hipError_t launch_ckpt_unpack(DType t, const CkptUnpackArgs& a, hipStream_t s);

struct CkptGradArgs {
    int64_t rows, cols;
    const void* dh; int64_t ld_dh;
    CkptIn cu, cup;
    void* du; int64_t ld_du;
    void* dup; int64_t ld_dup;
};
hipError_t launch_ckpt_act_grad(DType t, Act act, const CkptGradArgs& a, hipStream_t s);

// dw[i, o] (+)= sum_t value(t, i) dy[t, o], stored as inner x outer or
// outer x inner; `splits` shares of the tokens, joined from `partial`
// ([splits][rows][cols] of the stored matrix) where there are several.
struct WgradArgs {
    int64_t tokens, inner, outer;
    CkptIn x;
    const void* dy; int64_t ld_dy;
    float* dw; int64_t ld_dw;
    int oi, accumulate;
    int splits;
    float* partial;
};
int wgrad_splits(DType t, int64_t tokens, int64_t inner, int64_t outer);
hipError_t launch_wgrad(DType t, const WgradArgs& a, hipStream_t s);

}  // namespace np
