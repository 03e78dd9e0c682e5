// Internal declarations of the gradient norm and clipping: what one launch works on
// and its launchers.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace np {

// Tensors of one launch, cut into chunks; the list travels as the kernel's argument (4 KB
// with what the compiler adds), so no table is copied to the device and a captured launch
// keeps its own.  Chunks first[i] .. first[i + 1] - 1 are those
// of tensor i; size: elements, at most kGradMost, and the two flags below.
constexpr int kGradList = 152;
// us with chunks of 8192 / 4096 / 2048 for the sum (scaling: 8192): 124 M fp32 elements 285 / 269 / 275, 1.41 G
// bf16 2134 / 2060 / 2267; scaling in chunks of 16384: 265, 2197.
constexpr uint32_t kGradChunk = 4096, kGradScaleChunk = 8192, kGradSmallChunk = 2048;
constexpr uint32_t kGradMost = 1u << 29;            // a multiple of the chunk
constexpr uint32_t kGradInBf16 = 1u << 30, kGradOutBf16 = 1u << 31;

struct GradList {
    int count;
    uint32_t first[kGradList + 1];
    uint32_t size[kGradList];
    const void* in[kGradList];
    void* out[kGradList];
};

// Workspace: the factor, then a partial sum of each block.
constexpr int kGradPartials = 8192, kGradHead = 8, kGradBlocks = 2048;
constexpr int64_t kGradWorkspace = 8 * (kGradHead + kGradPartials);

// A call of up to kGradSmallChunks chunks of kGradSmallChunk elements is one block's work.  us a
// call of the front end so / by three launches: 100 elements 11.7 / 16.6, 80000 (40 chunks)
// 15.4 / 21.1, 130000 (64) 25.5 / 21.0.
constexpr uint32_t kGradSmallChunks = 48;

hipError_t launch_grad_small(const GradList& l, double max_norm, float* norm, bool scale, hipStream_t s);
hipError_t launch_grad_squares(const GradList& l, int blocks, double* partial, hipStream_t s);
hipError_t launch_grad_total(double* work, int partials, double max_norm, float* norm, hipStream_t s);
hipError_t launch_grad_scale(const GradList& l, int blocks, const double* work, hipStream_t s);

}  // namespace np
