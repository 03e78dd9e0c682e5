// Activation checkpoints in 8 bits and their use in the backward pass.
//
// A checkpoint holds groups of 64 consecutive features of a token as int8
// codes with one power-of-two step 2^e: with amax the group's largest
// magnitude, e is the smallest integer in [-126, 121] with
// rint(amax 2^-e) <= 127, and a code is rint(x 2^-e) within +-127.  The step
// is a power of two so that code 2^e is exact in bf16 (7 bits and a sign):
// matrix products of checkpoints on the bf16 matrix instructions then add no
// rounding to that of the codes.  It costs up to one bit against a free
// step; an 8-bit floating type (3 bits of mantissa) keeps 4% of a value
// near the top where these codes keep 0.8% of it at worst.
// A group with a NaN or an infinity has codes 0, e = -128, and stands for NaN.
#include "np_train.h"

#include <type_traits>

namespace np {
namespace {

typedef __bf16 bf16_t;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kThreads = 256;
constexpr int kV = 8;                            // consecutive features of a thread
constexpr int kNonFinite = -128;

__device__ __forceinline__ float pow2(int e) {   // e in [-126, 127]
    return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
}
__device__ __forceinline__ float step_of(int e) { return e == kNonFinite ? NAN : pow2(e); }

__device__ __forceinline__ float logistic(float x) { return 1.f / (1.f + expf(-x)); }
constexpr float kGeluA = 1.5957691216057308f;    // 2 sqrt(2 / pi)
constexpr float kGeluB = 0.044715f;

// Eight features of one row; past the row's end zero.  vec: rows are 16-byte
// aligned.
template <class T>
__device__ __forceinline__ void load8(float (&x)[kV], const T* row, int64_t c, int64_t cols, bool vec) {
    if (vec && c + kV <= cols) {
        T e[kV];
        if constexpr (sizeof(T) == 2) {
            const u32x4 r = *reinterpret_cast<const u32x4*>(row + c);
            __builtin_memcpy(e, &r, sizeof e);
        } else {
            const u32x4 r[2] = {reinterpret_cast<const u32x4*>(row + c)[0],
                                reinterpret_cast<const u32x4*>(row + c)[1]};
            __builtin_memcpy(e, r, sizeof e);
        }
#pragma unroll
        for (int i = 0; i < kV; ++i) x[i] = (float)e[i];
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) x[i] = c + i < cols ? (float)row[c + i] : 0.f;
    }
}

template <class T>
__device__ __forceinline__ void store8(T* row, const float (&x)[kV], int64_t c, int64_t cols, bool vec) {
    T e[kV];
#pragma unroll
    for (int i = 0; i < kV; ++i) e[i] = (T)x[i];
    if (vec && c + kV <= cols) {
        u32x4 r[sizeof(T) * kV / 16];
        __builtin_memcpy(r, e, sizeof e);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) * kV / 16); ++i) reinterpret_cast<u32x4*>(row + c)[i] = r[i];
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i)
            if (c + i < cols) row[c + i] = e[i];
    }
}

// Codes and exponent of a group held by 8 consecutive lanes, 8 features each.
__device__ __forceinline__ void encode(const CkptOut& o, const float (&x)[kV], int64_t row, int64_t c,
                                       int64_t pitch) {
    uint32_t top = 0;                            // largest magnitude, as bits: NaN above infinity
#pragma unroll
    for (int i = 0; i < kV; ++i) top = max(top, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
#pragma unroll
    for (int s = 1; s < 8; s <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, s, 64));
    const bool bad = top >= 0x7f800000u;
    // amax = 1.m 2^(E - 127): 127.5 2^e > amax first for e = E - 133, one more
    // where 1.m reaches 127.5 / 64.
    int e = (int)(top >> 23) - 133 + ((top & 0x7fffffu) >= 0x7f0000u);
    e = min(max(e, -126), 121);
    const float inv = pow2(-e);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        const float v = fminf(fmaxf(rintf(x[i] * inv), -127.f), 127.f);
        w[i / 4] |= ((uint32_t)(bad ? 0 : (int)v) & 0xffu) << (8 * (i % 4));
    }
    *reinterpret_cast<u32x2*>(o.codes + row * pitch + c) = u32x2{w[0], w[1]};
    if ((c & (kCkptGroup - 1)) == 0) o.exps[(row * pitch + c) / kCkptGroup] = (int8_t)(bad ? kNonFinite : e);
}

// The values of eight features.
__device__ __forceinline__ void decode(float (&x)[kV], const CkptIn& in, int64_t row, int64_t c, int64_t pitch) {
    const u32x2 w = *reinterpret_cast<const u32x2*>(in.codes + row * pitch + c);
    const float step = step_of(in.exps[(row * pitch + c) / kCkptGroup]);
#pragma unroll
    for (int i = 0; i < kV; ++i) x[i] = (float)(int8_t)(w[i / 4] >> (8 * (i % 4))) * step;
}

// One thread per eight features of the padded row; a group's eight threads
// are consecutive lanes (the padded row is a multiple of 64 features).
template <class T, Act ACT>
__global__ void __launch_bounds__(kThreads) pack_kernel(CkptPackArgs a, int64_t pitch, bool vec) {
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kV;
    if (i >= a.rows * pitch) return;             // whole groups: rows * pitch is a multiple of 64
    const int64_t row = i / pitch, c = i - row * pitch;
    float u[kV];
    load8(u, static_cast<const T*>(a.u) + row * a.ld_u, c, a.cols, vec);
    encode(a.cu, u, row, c, pitch);
    if constexpr (ACT != Act::None) {
        float h[kV];
        if constexpr (ACT == Act::Gelu) {
#pragma unroll
            for (int j = 0; j < kV; ++j) h[j] = u[j] * logistic(kGeluA * (u[j] + kGeluB * u[j] * u[j] * u[j]));
        } else {
            float g[kV];
            load8(g, static_cast<const T*>(a.up) + row * a.ld_up, c, a.cols, vec);
            encode(a.cup, g, row, c, pitch);
#pragma unroll
            for (int j = 0; j < kV; ++j) h[j] = u[j] * logistic(u[j]) * g[j];
        }
        // The checkpoint of h is that of the value the next layer reads.
#pragma unroll
        for (int j = 0; j < kV; ++j) h[j] = (float)(T)h[j];
        store8(static_cast<T*>(a.h) + row * a.ld_h, h, c, a.cols, vec);
        encode(a.ch, h, row, c, pitch);
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads) unpack_kernel(CkptUnpackArgs a, int64_t pitch, bool vec) {
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kV;
    if (i >= a.rows * pitch) return;
    const int64_t row = i / pitch, c = i - row * pitch;
    float x[kV];
    decode(x, a.c, row, c, pitch);
    store8(static_cast<T*>(a.out) + row * a.ld, x, c, a.cols, vec);
}

template <class T, Act ACT>
__global__ void __launch_bounds__(kThreads) act_grad_kernel(CkptGradArgs a, int64_t pitch, bool vec) {
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kV;
    if (i >= a.rows * pitch) return;
    const int64_t row = i / pitch, c = i - row * pitch;
    float dh[kV], u[kV];
    load8(dh, static_cast<const T*>(a.dh) + row * a.ld_dh, c, a.cols, vec);
    decode(u, a.cu, row, c, pitch);
    if constexpr (ACT == Act::Gelu) {
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            const float x = u[j], s = logistic(kGeluA * (x + kGeluB * x * x * x));
            u[j] = dh[j] * (s + x * s * (1.f - s) * kGeluA * (1.f + 3.f * kGeluB * x * x));
        }
    } else {
        float g[kV];
        decode(g, a.cup, row, c, pitch);
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            const float x = u[j], s = logistic(x);
            u[j] = dh[j] * g[j] * (s * (1.f + x * (1.f - s)));
            g[j] = dh[j] * x * s;
        }
        store8(static_cast<T*>(a.dup) + row * a.ld_dup, g, c, a.cols, vec);
    }
    store8(static_cast<T*>(a.du) + row * a.ld_du, u, c, a.cols, vec);
}

// -------------------------------------------------------- weight gradient ---
// dw[i, o] = sum_t x(t, i) dy(t, o): a matrix product over the tokens whose
// operands both have the summed index as their slow one.  Tiles of BK tokens
// go to LDS as they lie in memory (checkpoints expanded to bf16 on the way,
// exactly), and the transposing LDS reads hand the matrix instructions their
// operands.  fp32 dy is split into three bf16 terms (8 mantissa bits each,
// by truncation, so the split is exact) and takes three products.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// BK x R elements, 16-byte chunk c of row k at c ^ wswz(k): the four rows one
// transposing read takes lie in disjoint banks.
template <int R>
__device__ __forceinline__ int widx(int k, int c) { return k * R + ((c ^ (4 * (k & 3))) << 3); }

// Fragment of the 32x32x16 product: lane l gets column mb + l % 32, rows
// 16 s + 8 (l / 32) .. + 7.
template <int R>
__device__ __forceinline__ bf16x8 wfrag(const bf16_t* lds, int mb, int s, int lane) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int g = lane >> 4, p = lane & 15;
    const int c = (mb >> 3) + 2 * (g & 1) + ((p & 3) >> 1), k = 16 * s + 8 * (g >> 1) + (p >> 2), in = 4 * (p & 1);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + widx<R>(k, c) + in));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + widx<R>(k + 4, c) + in));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

template <class T, bool OI>
__global__ void __launch_bounds__(kThreads, 2) wgrad_kernel(WgradArgs a, int64_t pitch, int64_t chunk, bool vec) {
    constexpr int R = 128, NT = std::is_same_v<T, bf16_t> ? 1 : 3, BK = 32;
    constexpr int NX = BK * R / 16 / kThreads;           // 16 codes each
    constexpr int E = 16 / sizeof(T), NY = BK * R / E / kThreads;
    __shared__ __attribute__((aligned(16))) bf16_t xs[2][BK * R];
    __shared__ __attribute__((aligned(16))) bf16_t ys[2][NT][BK * R];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int tiles_i = (int)((a.inner + R - 1) / R);
    const int64_t i0 = (int64_t)(blockIdx.x % tiles_i) * R, o0 = (int64_t)(blockIdx.x / tiles_i) * R;
    const int64_t t0 = blockIdx.y * chunk, t1 = min(a.tokens, t0 + chunk);
    const T* dy = static_cast<const T*>(a.dy);

    u32x4 rx[NX], ry[NY];
    int8_t re[NX];
    auto load = [&](int64_t t) {
#pragma unroll
        for (int n = 0; n < NX; ++n) {
            const int e = tid + n * kThreads, c = e % (R / 16);
            const int64_t row = t + e / (R / 16), at = row * pitch + i0 + 16 * c;
            rx[n] = u32x4{0, 0, 0, 0};
            re[n] = 0;
            if (row < t1 && i0 + 16 * c < pitch) {
                rx[n] = *reinterpret_cast<const u32x4*>(a.x.codes + at);
                re[n] = a.x.exps[at / kCkptGroup];
            }
        }
#pragma unroll
        for (int n = 0; n < NY; ++n) {
            const int e = tid + n * kThreads, c = e % (R / E);
            const int64_t row = t + e / (R / E), o = o0 + E * c;
            const T* p = dy + row * a.ld_dy + o;
            ry[n] = u32x4{0, 0, 0, 0};
            if (row < t1) {
                if (vec && o + E <= a.outer) {
                    ry[n] = *reinterpret_cast<const u32x4*>(p);
                } else {
                    T v[E];
#pragma unroll
                    for (int i = 0; i < E; ++i) v[i] = o + i < a.outer ? p[i] : T(0.f);
                    __builtin_memcpy(&ry[n], v, 16);
                }
            }
        }
    };
    auto store = [&](int buf) {
#pragma unroll
        for (int n = 0; n < NX; ++n) {
            const int e = tid + n * kThreads, c = e % (R / 16), k = e / (R / 16);
            const float step = step_of(re[n]);
            bf16x8 v[2];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                v[i / 8][i % 8] = (bf16_t)((float)(int8_t)(rx[n][i / 4] >> (8 * (i % 4))) * step);
            *reinterpret_cast<bf16x8*>(xs[buf] + widx<R>(k, 2 * c)) = v[0];
            *reinterpret_cast<bf16x8*>(xs[buf] + widx<R>(k, 2 * c + 1)) = v[1];
        }
#pragma unroll
        for (int n = 0; n < NY; ++n) {
            const int e = tid + n * kThreads, c = e % (R / E), k = e / (R / E);
            if constexpr (NT == 1) {
                *reinterpret_cast<u32x4*>(ys[buf][0] + widx<R>(k, c)) = ry[n];
            } else {
                uint32_t w[3][2];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float x = __builtin_bit_cast(float, (uint32_t)ry[n][i]);
#pragma unroll
                    for (int p = 0; p < 3; ++p) {
                        const uint32_t top = __builtin_bit_cast(uint32_t, x) & 0xffff0000u;
                        const float f = __builtin_bit_cast(float, top);
                        x = x == f ? 0.f : x - f;        // an infinity is its own first term
                        if (i & 1) w[p][i / 2] |= top;
                        else w[p][i / 2] = top >> 16;
                    }
                }
#pragma unroll
                for (int p = 0; p < 3; ++p)
                    *reinterpret_cast<u32x2*>(ys[buf][p] + widx<R>(k, c / 2) + 4 * (c & 1)) = u32x2{w[p][0], w[p][1]};
            }
        }
    };

    // Four waves, 64 x 64 each.
    const int wi = (wave & 1) * 64, wo = (wave >> 1) * 64;
    f32x16 acc[2][2] = {};
    const int steps = (int)((t1 - t0 + BK - 1) / BK);
    if (steps > 0) {
        load(t0);
        store(0);
    }
    for (int it = 0; it < steps; ++it) {
        const bool more = it + 1 < steps;
        if (more) load(t0 + (int64_t)(it + 1) * BK);
        lds_barrier();
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
            bf16x8 fx[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) fx[i] = wfrag<R>(xs[it & 1], wi + 32 * i, s, lane);
#pragma unroll
            for (int p = NT - 1; p >= 0; --p) {
                bf16x8 fy[2];
#pragma unroll
                for (int j = 0; j < 2; ++j) fy[j] = wfrag<R>(ys[it & 1][p], wo + 32 * j, s, lane);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[i][j] = OI ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[j], fx[i], acc[i][j], 0, 0, 0)
                                       : __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[i], fy[j], acc[i][j], 0, 0, 0);
            }
        }
        if (more) store((it + 1) & 1);
    }
    // Lane l: column l % 32 (the contiguous side of the stored matrix), rows
    // 8 (r / 4) + 4 (l / 32) + r % 4.
    const int64_t nr = OI ? a.outer : a.inner, nc = OI ? a.inner : a.outer;
    const bool whole = a.splits == 1;
    float* out = whole ? a.dw : a.partial + blockIdx.y * nr * nc;
    const int64_t ld = whole ? a.ld_dw : nc;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int rr = 8 * (r / 4) + 4 * half + r % 4, cc = lane & 31;
                const int64_t row = OI ? o0 + wo + 32 * j + rr : i0 + wi + 32 * i + rr;
                const int64_t col = OI ? i0 + wi + 32 * i + cc : o0 + wo + 32 * j + cc;
                if (row < nr && col < nc) {
                    float* p = out + row * ld + col;
                    *p = acc[i][j][r] + (whole && a.accumulate ? *p : 0.f);
                }
            }
}

// Adds the shares of the tokens in their order.
__global__ void __launch_bounds__(kThreads) wgrad_join_kernel(WgradArgs a) {
    const int64_t nr = a.oi ? a.outer : a.inner, nc = a.oi ? a.inner : a.outer;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= nr * nc) return;
    float s = 0.f;
    for (int k = 0; k < a.splits; ++k) s += a.partial[k * nr * nc + i];
    float* p = a.dw + i / nc * a.ld_dw + i % nc;
    *p = s + (a.accumulate ? *p : 0.f);
}

template <class T>
bool aligned(const void* p, int64_t ld) {
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % (16 / (int64_t)sizeof(T)) == 0;
}

unsigned blocks_of(int64_t rows, int64_t pitch) {
    return (unsigned)((rows * pitch / kV + kThreads - 1) / kThreads);
}

template <class T>
hipError_t pack(Act act, const CkptPackArgs& a, hipStream_t s) {
    const int64_t pitch = ckpt_pitch(a.cols);
    bool vec = aligned<T>(a.u, a.ld_u);
    if (act != Act::None) vec = vec && aligned<T>(a.h, a.ld_h);
    if (act == Act::Swiglu) vec = vec && aligned<T>(a.up, a.ld_up);
    const unsigned n = blocks_of(a.rows, pitch);
    if (act == Act::None) pack_kernel<T, Act::None><<<n, kThreads, 0, s>>>(a, pitch, vec);
    else if (act == Act::Gelu) pack_kernel<T, Act::Gelu><<<n, kThreads, 0, s>>>(a, pitch, vec);
    else pack_kernel<T, Act::Swiglu><<<n, kThreads, 0, s>>>(a, pitch, vec);
    return hipGetLastError();
}

template <class T>
hipError_t act_grad(Act act, const CkptGradArgs& a, hipStream_t s) {
    const int64_t pitch = ckpt_pitch(a.cols);
    bool vec = aligned<T>(a.dh, a.ld_dh) && aligned<T>(a.du, a.ld_du);
    if (act == Act::Swiglu) vec = vec && aligned<T>(a.dup, a.ld_dup);
    const unsigned n = blocks_of(a.rows, pitch);
    if (act == Act::Gelu) act_grad_kernel<T, Act::Gelu><<<n, kThreads, 0, s>>>(a, pitch, vec);
    else act_grad_kernel<T, Act::Swiglu><<<n, kThreads, 0, s>>>(a, pitch, vec);
    return hipGetLastError();
}

template <class T>
hipError_t wgrad(const WgradArgs& a, hipStream_t s) {
    const int64_t pitch = ckpt_pitch(a.inner);
    const int64_t tiles = ((a.inner + 127) / 128) * ((a.outer + 127) / 128);
    const int64_t chunk = ((a.tokens + a.splits - 1) / a.splits + 31) / 32 * 32;
    const bool vec = aligned<T>(a.dy, a.ld_dy);
    const dim3 grid((unsigned)tiles, (unsigned)a.splits);
    if (a.oi) wgrad_kernel<T, true><<<grid, kThreads, 0, s>>>(a, pitch, chunk, vec);
    else wgrad_kernel<T, false><<<grid, kThreads, 0, s>>>(a, pitch, chunk, vec);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    wgrad_join_kernel<<<(unsigned)((a.inner * a.outer + kThreads - 1) / kThreads), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_ckpt_pack(DType t, Act act, const CkptPackArgs& a, hipStream_t s) {
    return t == DType::BF16 ? pack<bf16_t>(act, a, s) : pack<float>(act, a, s);
}

hipError_t launch_ckpt_unpack(DType t, const CkptUnpackArgs& a, hipStream_t s) {
    const int64_t pitch = ckpt_pitch(a.cols);
    const unsigned n = blocks_of(a.rows, pitch);
    if (t == DType::BF16) unpack_kernel<bf16_t><<<n, kThreads, 0, s>>>(a, pitch, aligned<bf16_t>(a.out, a.ld));
    else unpack_kernel<float><<<n, kThreads, 0, s>>>(a, pitch, aligned<float>(a.out, a.ld));
    return hipGetLastError();
}

hipError_t launch_ckpt_act_grad(DType t, Act act, const CkptGradArgs& a, hipStream_t s) {
    return t == DType::BF16 ? act_grad<bf16_t>(act, a, s) : act_grad<float>(act, a, s);
}

// Shares of the tokens: enough blocks for every CU where the matrix alone has
// too few tiles, at least 256 tokens each.
int wgrad_splits(DType, int64_t tokens, int64_t inner, int64_t outer) {
    const int64_t tiles = ((inner + 127) / 128) * ((outer + 127) / 128);
    const int64_t want = (512 + tiles - 1) / tiles, most = tokens / 256;
    const int64_t n = want < most ? want : most;
    return (int)(n < 1 ? 1 : n > 64 ? 64 : n);
}

hipError_t launch_wgrad(DType t, const WgradArgs& a, hipStream_t s) {
    return t == DType::BF16 ? wgrad<bf16_t>(a, s) : wgrad<float>(a, s);
}

}  // namespace np
