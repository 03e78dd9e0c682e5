// Norm of many gradients together, and their scaling to a limit:
//   norm = sqrt(sum g^2),  out = c g,  c = 1 where norm <= limit, else limit / norm.
//
// Bound by memory: every gradient is read for the norm, and read and written again
// for the scaling, which needs the norm of all.  Squares are summed in 64 bits: the sum
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
typedef u32x4 u32x4_any __attribute__((aligned(2)));   // global memory takes 16 bytes on any byte

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

template <class T> constexpr int kE = 16 / sizeof(T);

// f(i, x) for the elements x of [p, p + n) that are this thread's, kE<T> or one of
// them from element i on; n <= kGradChunk.
template <class T, class F>
__device__ __forceinline__ void each(const T* p, uint32_t n, F f) {
    constexpr int E = kE<T>, N = kGradChunk / (kThreads * E);
    if (n == kGradChunk) {
        u32x4 r[N];
#pragma unroll
        for (int k = 0; k < N; ++k) r[k] = *reinterpret_cast<const u32x4_any*>(p + (k * kThreads + threadIdx.x) * E);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            T x[E];
            __builtin_memcpy(x, &r[k], 16);
            f((k * kThreads + threadIdx.x) * E, x);
        }
    } else {
        for (uint32_t i = threadIdx.x * E; i < n; i += kThreads * E) {
            if (i + E <= n) {
                const u32x4 r = *reinterpret_cast<const u32x4_any*>(p + i);
                T x[E];
                __builtin_memcpy(x, &r, 16);
                f(i, x);
            } else
                for (uint32_t j = i; j < n; ++j) {
                    const T x[1] = {p[j]};
                    f(j, x);
                }
        }
    }
}

template <class T>
__device__ __forceinline__ double squares(const T* p, uint32_t n) {
    double sum = 0.0;
    each(p, n, [&](uint32_t, const auto& x) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof x / sizeof(T)); ++i) {
            const double v = (double)(float)x[i];
            sum = __builtin_fma(v, v, sum);
        }
    });
    return sum;
}

template <class T, class U>
__device__ __forceinline__ void scale(const T* p, U* out, uint32_t n, double c) {
    each(p, n, [&](uint32_t i, const auto& x) {
        constexpr int M = sizeof x / sizeof(T);
        U y[M];
#pragma unroll
        for (int k = 0; k < M; ++k) y[k] = (U)(float)((double)(float)x[k] * c);
        if constexpr (M == 1) out[i] = y[0];
        else if constexpr (sizeof y == 8) {
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));
            u32x2 r;
            __builtin_memcpy(&r, y, 8);
            *reinterpret_cast<u32x2*>(out + i) = r;
        } else {
            u32x4 r[sizeof y / 16];
            __builtin_memcpy(r, y, sizeof y);
#pragma unroll
            for (int k = 0; k < (int)(sizeof y / 16); ++k) reinterpret_cast<u32x4_any*>(out + i)[k] = r[k];
        }
    });
}

// partial[b]: the sum of block b's squares.
__global__ void __launch_bounds__(kThreads) grad_squares_kernel(GradList l, double* partial) {
    const uint32_t all = l.first[l.count];
    double sum = 0.0;
    for (uint32_t c = blockIdx.x; c < all; c += gridDim.x) {
        const int t = tensor_of(l, c);
        const uint32_t size = l.size[t], at = (c - l.first[t]) * kGradChunk;
        const uint32_t n = min((size & (kGradInBf16 - 1)) - at, kGradChunk);
        if (size & kGradInBf16) sum += squares(static_cast<const bf16_t*>(l.in[t]) + at, n);
        else sum += squares(static_cast<const float*>(l.in[t]) + at, n);
    }
    sum = block_sum<kThreads>(sum);
    if (threadIdx.x == 0) partial[blockIdx.x] = sum;
}

constexpr int kTotalThreads = 1024;

// The norm and the factor, from the partial sums.
__global__ void __launch_bounds__(kTotalThreads) grad_total_kernel(double* work, int partials, double max_norm, float* norm) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < partials; i += kTotalThreads) sum += work[kGradHead + i];
    sum = block_sum<kTotalThreads>(sum);
    if (threadIdx.x == 0) {
        const double n = sqrt(sum);
        work[0] = n <= max_norm ? 1.0 : max_norm / n;
        *norm = (float)n;
    }
}

__global__ void __launch_bounds__(kThreads) grad_scale_kernel(GradList l, const double* work) {
    const uint32_t all = l.first[l.count];
    const double f = work[0];
    for (uint32_t c = blockIdx.x; c < all; c += gridDim.x) {
        const int t = tensor_of(l, c);
        const uint32_t size = l.size[t], at = (c - l.first[t]) * kGradChunk;
        const uint32_t n = min((size & (kGradInBf16 - 1)) - at, kGradChunk);
        if (l.in[t] == l.out[t] && f == 1.0) continue;      // as it is
        if (size & kGradInBf16) {
            const bf16_t* in = static_cast<const bf16_t*>(l.in[t]) + at;
            if (size & kGradOutBf16) scale(in, static_cast<bf16_t*>(l.out[t]) + at, n, f);
            else scale(in, static_cast<float*>(l.out[t]) + at, n, f);
        } else {
            const float* in = static_cast<const float*>(l.in[t]) + at;
            if (size & kGradOutBf16) scale(in, static_cast<bf16_t*>(l.out[t]) + at, n, f);
            else scale(in, static_cast<float*>(l.out[t]) + at, n, f);
        }
    }
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

}  // namespace np
