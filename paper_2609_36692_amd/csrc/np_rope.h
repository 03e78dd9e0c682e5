// Internal declarations of the norm and rotation of query and key heads.  Not part of
// the public ABI.
#pragma once

#include "np_train.h"

namespace np {

constexpr int kRopeMaxDim = 256;
constexpr int kRopeMaxHeads = 1 << 16;
constexpr int kRopeMaxAxes = 256;

struct RopeArgs {                  // [2]: queries, keys
    AttnOperand x[2];              // forward, and backward with norm: read
    AttnOperand y[2];              // written: the turned heads, or the gradient of x
    AttnOperand g[2];              // backward: the gradient of the turned heads
    const void* w[2];              // norm weights, or null
    float* dw[2];                  // backward: their gradients, or null
    int heads[2];
    int dim, pairs, axes;
    int adjacent, norm, weight_bf16, positions_64;
    double eps, inv_dim;
    int64_t tokens;
    const double* freqs;           // [pairs], radians a step
    const int32_t* axis;           // [pairs], or null: 0
    const void* positions;         // [axes][tokens]
    int64_t position_stride;
    float* partial;                // [blocks][2][dim], where dw is wanted
};

// Floats of workspace that a backward call needs: where weight gradients are wanted, 2 dim
// for each of up to kRopeMostSums blocks.
constexpr int kRopeMostSums = 512;
int64_t rope_workspace(DType t, const RopeArgs& a);
inline bool rope_sums(const RopeArgs& a) { return a.norm && (a.dw[0] || a.dw[1]); }
hipError_t launch_rope(DType t, const RopeArgs& a, bool backward, hipStream_t s);

}  // namespace np
