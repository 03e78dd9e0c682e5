// Norm of many gradients together, and their scaling to a limit:
//   norm = sqrt(sum g^2),  out = c g,  c = 1 where norm <= limit, else limit / norm.
//
// Bound by memory: every gradient is read for the norm, and read and written again
// for the scaling, which needs the norm of all.  148 fp32 tensors of 124 M elements: sum 80 us (6.2
// TB/s, a part from the last-level cache), scaling 175 (5.7), both 265 (the copy's rate of 4.76 TB/s
// would take 314); 196 bf16 ones of 1.41 G to fp32: 495 us (5.7) and 1540 (5.5).  The list of
// tensors is the launch's argument, so nothing is uploaded.  Squares are summed in 64 bits: the sum
// neither leaves the range nor rounds (fp32 squares overflow from 2e19 on), and two
// fp64 instructions for an element are hidden behind its load.  The product with c is
// rounded once from 64 bits to fp32 (for bf16 results once more; off by at most
// 2^-8 + 2^-24 of the value).
// Chunks go to blocks in a fixed order and partial sums are joined in theirs: the same
// bits every time, no atomics.
#include "np_grads.h"

#include <cmath>

namespace np {
namespace {

typedef __bf16 bf16_t;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));   // global memory takes 16 bytes on any byte
typedef u32x2 u32x2_any __attribute__((aligned(2)));

constexpr int kThreads = 256;

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// Sum over the block, to thread 0.
template <int NT>
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[NT / 64];
    v = wave_sum(v);
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int i = 1; i < NT / 64; ++i) v += part[i];
    }
    return v;
}

// The tensor that chunk c belongs to: the last one that begins at c or before.
__device__ __forceinline__ int tensor_of(const GradList& l, uint32_t c) {
    const int lane = threadIdx.x & 63;
    int n = 0;
#pragma unroll
    for (int i = 0; i < kGradList; i += 64)
        n += __popcll(__ballot(i + lane < l.count && l.first[min(i + lane, kGradList)] <= c));
    return __builtin_amdgcn_readfirstlane(n - 1);
}

// A piece of 8 or 16 bytes, at any byte.
template <int BYTES> struct Piece { typedef u32x4 type; typedef u32x4_any any; };
template <> struct Piece<8> { typedef u32x2 type; typedef u32x2_any any; };

// f(i, x) for the elements x of [p, p + n) that are this thread's of NT, E or one of
// them from element i on; n <= CHUNK.
template <int NT, uint32_t CHUNK, int E, class T, class F>
__device__ __forceinline__ void each(const T* p, uint32_t n, F f) {
    constexpr int N = CHUNK / (NT * E);
    using P = Piece<E * sizeof(T)>;
    const uint32_t me = threadIdx.x % NT;
    if (n == CHUNK) {
        typename P::type r[N];
#pragma unroll
        for (int k = 0; k < N; ++k) r[k] = *reinterpret_cast<const typename P::any*>(p + (k * NT + me) * E);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            T x[E];
            __builtin_memcpy(x, &r[k], sizeof x);
            f((k * NT + me) * E, x);
        }
    } else {
        for (uint32_t i = me * E; i < n; i += NT * E) {
            if (i + E <= n) {
                const typename P::type r = *reinterpret_cast<const typename P::any*>(p + i);
                T x[E];
                __builtin_memcpy(x, &r, sizeof x);
                f(i, x);
            } else
                for (uint32_t j = i; j < n; ++j) {
                    const T x[1] = {p[j]};
                    f(j, x);
                }
        }
    }
}

template <int NT, uint32_t CHUNK, class T>
__device__ __forceinline__ double squares(const T* p, uint32_t n) {
    double sum = 0.0;
    each<NT, CHUNK, 16 / (int)sizeof(T)>(p, n, [&](uint32_t, const auto& x) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof x / sizeof(T)); ++i) {
            const double v = (double)(float)x[i];
            sum = __builtin_fma(v, v, sum);
        }
    });
    return sum;
}

template <int NT, uint32_t CHUNK, class T, class U>
__device__ __forceinline__ void scale(const T* p, U* out, uint32_t n, double c) {
    // As many elements as fill 16 bytes of the wider type: a wave's store is one piece of memory.
    constexpr int E = 16 / (int)(sizeof(T) > sizeof(U) ? sizeof(T) : sizeof(U));
    each<NT, CHUNK, E>(p, n, [&](uint32_t i, const auto& x) {
        constexpr int M = sizeof x / sizeof(T);
        U y[M];
#pragma unroll
        for (int k = 0; k < M; ++k) y[k] = (U)(float)((double)(float)x[k] * c);
        if constexpr (M == 1) out[i] = y[0];
        else {
            using P = Piece<sizeof y>;
            typename P::type r;
            __builtin_memcpy(&r, y, sizeof y);
            // Past the caches, which may still hold gradients that are read next.  ms with plain stores: 148
            // fp32 tensors of 124 M elements 0.31, so 0.28.
            __builtin_nontemporal_store(r, reinterpret_cast<typename P::any*>(out + i));
        }
    });
}

// Chunk c of the list, by NT threads: its sum of squares, or its scaled elements.
struct Chunk {
    int tensor;
    uint32_t at, n;
    bool in16, out16;
};
template <uint32_t CHUNK>
__device__ __forceinline__ Chunk chunk_of(const GradList& l, uint32_t c) {
    const int t = tensor_of(l, c);
    const uint32_t size = l.size[t], at = (c - l.first[t]) * CHUNK;
    return {t, at, min((size & (kGradInBf16 - 1)) - at, CHUNK), (size & kGradInBf16) != 0, (size & kGradOutBf16) != 0};
}
template <int NT, uint32_t CHUNK>
__device__ __forceinline__ double squares_of(const GradList& l, uint32_t c) {
    const Chunk k = chunk_of<CHUNK>(l, c);
    return k.in16 ? squares<NT, CHUNK>(static_cast<const bf16_t*>(l.in[k.tensor]) + k.at, k.n)
                  : squares<NT, CHUNK>(static_cast<const float*>(l.in[k.tensor]) + k.at, k.n);
}
template <int NT, uint32_t CHUNK>
__device__ __forceinline__ void scale_of(const GradList& l, uint32_t c, double f) {
    const Chunk k = chunk_of<CHUNK>(l, c);
    const void* in = l.in[k.tensor];
    void* out = l.out[k.tensor];
    if (in == out && f == 1.0) return;               // as it is
    auto from = [&](auto* p) {
        if (k.out16) scale<NT, CHUNK>(p + k.at, static_cast<bf16_t*>(out) + k.at, k.n, f);
        else scale<NT, CHUNK>(p + k.at, static_cast<float*>(out) + k.at, k.n, f);
    };
    if (k.in16) from(static_cast<const bf16_t*>(in));
    else from(static_cast<const float*>(in));
}

// partial[b]: the sum of block b's squares.
__global__ void __launch_bounds__(kThreads) grad_squares_kernel(GradList l, double* partial) {
    const uint32_t all = l.first[l.count];
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < all; c += gridDim.x) sum += squares_of<kThreads, kGradChunk>(l, c);
    sum = block_sum<kThreads>(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

__device__ __forceinline__ double factor(double norm, double max_norm) { return norm <= max_norm ? 1.0 : max_norm / norm; }

// The sum of the partial sums, in the same order in every block of as many threads.
template <int NT>
__device__ __forceinline__ double total(const double* partial, int partials) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < partials; i += NT) sum += partial[i];
    return block_sum<NT>(sum);
}

constexpr int kTotalThreads = 1024;

// The norm and the factor.
__global__ void __launch_bounds__(kTotalThreads) grad_total_kernel(double* work, int partials, double max_norm, float* norm) {
    const double sum = total<kTotalThreads>(work + kGradHead, partials);
    if (threadIdx.x == 0) {
        const double n = sqrt(sum);
        work[0] = factor(n, max_norm);
        *norm = (float)n;
    }
}

// Chunks in falling order: the last ones that were read for the norm are the ones
// that a cache may still hold.
__global__ void __launch_bounds__(kThreads) grad_scale_kernel(GradList l, const double* work) {
    const uint32_t all = l.first[l.count];
    const double f = work[0];
    for (uint32_t c = blockIdx.x; c < all; c += gridDim.x) scale_of<kThreads, kGradScaleChunk>(l, all - 1 - c, f);
}

// Norm and scaling of few elements in one block: chunks go to its waves in turn.
__global__ void __launch_bounds__(kTotalThreads) grad_small_kernel(GradList l, double max_norm, float* norm, int scaled) {
    const uint32_t all = l.first[l.count], wave = threadIdx.x / 64;
    double sum = 0.0;
    for (uint32_t c = wave; c < all; c += kTotalThreads / 64) sum += squares_of<64, kGradSmallChunk>(l, c);
    __shared__ double shared;
    sum = block_sum<kTotalThreads>(sum);
    if (threadIdx.x == 0) {
        const double n = sqrt(sum);
        *norm = (float)n;
        shared = factor(n, max_norm);
    }
    __syncthreads();
    if (!scaled) return;
    for (uint32_t c = wave; c < all; c += kTotalThreads / 64) scale_of<64, kGradSmallChunk>(l, c, shared);
}

}  // namespace

hipError_t launch_grad_squares(const GradList& l, int blocks, double* partial, hipStream_t s) {
    grad_squares_kernel<<<blocks, kThreads, 0, s>>>(l, partial);
    return hipGetLastError();
}
hipError_t launch_grad_total(double* work, int partials, double max_norm, float* norm, hipStream_t s) {
    grad_total_kernel<<<1, kTotalThreads, 0, s>>>(work, partials, max_norm, norm);
    return hipGetLastError();
}
hipError_t launch_grad_scale(const GradList& l, int blocks, const double* work, hipStream_t s) {
    grad_scale_kernel<<<blocks, kThreads, 0, s>>>(l, work);
    return hipGetLastError();
}

hipError_t launch_grad_small(const GradList& l, double max_norm, float* norm, bool scale, hipStream_t s) {
    grad_small_kernel<<<1, kTotalThreads, 0, s>>>(l, max_norm, norm, scale);
    return hipGetLastError();
}

}  // namespace np
