// Activation checkpoints in 8 bits and their use in the backward pass.
//
// A checkpoint holds groups of 64 consecutive features of a token as int8
// codes with one power-of-two step 2^e: with amax the group's largest
// magnitude, e is the smallest integer in [-126, 121] with
// rint(amax 2^-e) <= 127, and a code is rint(x 2^-e) within +-127.  The step
// is a power of two so that code 2^e is exact in bf16 (7 bits and a sign):
// matrix products of checkpoints on the bf16 matrix instructions then add no
// rounding to that of the codes.  It costs up to one bit against a free step.
// An 8-bit floating type with 3 bits of mantissa is off by up to 6% of every
// value, these codes by up to 0.8% of the group's largest.
// A group with a NaN or an infinity has codes 0, e = -128, and stands for NaN.
#include "np_dy_rows.h"
#include "np_train.h"

#include <cmath>
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

// 16 bytes of elements of T, at any element (global memory takes 16-byte
// accesses on any byte).
template <class T> struct Sixteen;
template <> struct Sixteen<bf16_t> { typedef u32x4 type __attribute__((aligned(2))); };
template <> struct Sixteen<float> { typedef u32x4 type __attribute__((aligned(4))); };

// Eight features of one row; past the row's end zero.
template <class T>
__device__ __forceinline__ void load8(float (&x)[kV], const T* row, int64_t c, int64_t cols) {
    if (c + kV <= cols) {
        u32x4 r[sizeof(T) * kV / 16];
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) * kV / 16); ++i)
            r[i] = reinterpret_cast<const typename Sixteen<T>::type*>(row + c)[i];
        T e[kV];
        __builtin_memcpy(e, r, sizeof e);
#pragma unroll
        for (int i = 0; i < kV; ++i) x[i] = (float)e[i];
    } else {
#pragma unroll
        for (int i = 0; i < kV; ++i) x[i] = c + i < cols ? (float)row[c + i] : 0.f;
    }
}

template <class T>
__device__ __forceinline__ void store8(T* row, const float (&x)[kV], int64_t c, int64_t cols) {
    T e[kV];
#pragma unroll
    for (int i = 0; i < kV; ++i) e[i] = (T)x[i];
    if (c + kV <= cols) {
        u32x4 r[sizeof(T) * kV / 16];
        __builtin_memcpy(r, e, sizeof e);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) * kV / 16); ++i)
            reinterpret_cast<typename Sixteen<T>::type*>(row + c)[i] = r[i];
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
// are consecutive lanes (the padded row is a multiple of 64 features).  All
// checkpoints of an activation leave in the pass that computes it: each input is
// read once, 16 bytes a lane.  Bound by memory: SwiGLU with its three checkpoints,
// 8192 x 6144 bf16, 456 MB in 91 us, 5.0 TB/s where a large copy reaches 4.8; the
// checkpoints read back (unpack_kernel) 152 MB in 25 us each.
template <class T, Act ACT>
__global__ void __launch_bounds__(kThreads) pack_kernel(CkptPackArgs a, int64_t pitch) {
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kV;
    if (i >= a.rows * pitch) return;             // whole groups: rows * pitch is a multiple of 64
    const int64_t row = i / pitch, c = i - row * pitch;
    float u[kV];
    load8(u, static_cast<const T*>(a.u) + row * a.ld_u, c, a.cols);
    encode(a.cu, u, row, c, pitch);
    if constexpr (ACT != Act::None) {
        float h[kV];
        if constexpr (ACT == Act::Gelu) {
#pragma unroll
            for (int j = 0; j < kV; ++j) h[j] = u[j] * logistic(kGeluA * (u[j] + kGeluB * u[j] * u[j] * u[j]));
        } else {
            float g[kV];
            load8(g, static_cast<const T*>(a.up) + row * a.ld_up, c, a.cols);
            encode(a.cup, g, row, c, pitch);
#pragma unroll
            for (int j = 0; j < kV; ++j) h[j] = u[j] * logistic(u[j]) * g[j];
        }
        // The checkpoint of h is that of the value the next layer reads.
#pragma unroll
        for (int j = 0; j < kV; ++j) h[j] = (float)(T)h[j];
        store8(static_cast<T*>(a.h) + row * a.ld_h, h, c, a.cols);
        encode(a.ch, h, row, c, pitch);
    }
}

template <class T>
__global__ void __launch_bounds__(kThreads) unpack_kernel(CkptUnpackArgs a, int64_t pitch) {
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kV;
    if (i >= a.rows * pitch) return;
    const int64_t row = i / pitch, c = i - row * pitch;
    float x[kV];
    decode(x, a.c, row, c, pitch);
    store8(static_cast<T*>(a.out) + row * a.ld, x, c, a.cols);
}

// The activation's gradient: dh and the codes in, the gradients out.  Bound by
// memory: SwiGLU, 8192 x 5632 bf16, 370 MB in 75 us (4.9 TB/s); GELU, 4096 x 3072
// fp32, 113 MB in 22 us.
template <class T, Act ACT>
__global__ void __launch_bounds__(kThreads) act_grad_kernel(CkptGradArgs a, int64_t pitch) {
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kV;
    if (i >= a.rows * pitch) return;
    const int64_t row = i / pitch, c = i - row * pitch;
    float dh[kV], u[kV];
    load8(dh, static_cast<const T*>(a.dh) + row * a.ld_dh, c, a.cols);
    decode(u, a.cu, row, c, pitch);
    if constexpr (ACT == Act::Gelu) {
#pragma unroll
        for (int j = 0; j < kV; ++j) {
            const float x = u[j], s = logistic(kGeluA * (x + kGeluB * x * x * x));
            // Far out s (1 - s) is 0: x^2 must not overflow beside it.
            u[j] = dh[j] * (s + x * s * (1.f - s) * kGeluA * (1.f + 3.f * kGeluB * fminf(x * x, 1e30f)));
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
        store8(static_cast<T*>(a.dup) + row * a.ld_dup, g, c, a.cols);
    }
    store8(static_cast<T*>(a.du) + row * a.ld_du, u, c, a.cols);
}

// -------------------------------------------------------- weight gradient ---
// dw[i, o] = sum_t x(t, i) dy(t, o): a matrix product over the tokens whose
// operands both have the summed index as their slow one.  Tiles of BK tokens
// go to LDS as they lie in memory (checkpoints expanded to bf16 on the way,
// exactly), and the transposing LDS reads hand the matrix instructions their
// operands.  fp32 dy is split into three bf16 terms (8 mantissa bits each,
// by truncation, so the split is exact for magnitudes from 2^-100 up) and takes
// three products, which is still 2.4 times the rate of the fp32 instructions.
// Measured: 16384 x 2048 x 6144 bf16 410-430 us from card to card (960-1005 TFLOP/s;
// a library product of bf16 operands reaches 1263 at 8192^3), 4001 x 768 x 2304 fp32
// 58-64 us (220-245; 154 for a library's fp32 product), 53 of them in the products:
// 216 blocks of 32 steps, whose conversions and LDS traffic the one block of a CU
// hides in part (matrix instructions 36% of the cycles).
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

// Tile of BI inner by BO outer features, WI x WO waves, each with the accumulators
// of BI / WI by BO / WO of them.
template <class T, bool OI, DyRows ROWS, int BI, int BO, int WI, int WO>
__global__ void __launch_bounds__(64 * WI * WO, 2) wgrad_kernel(WgradArgs a, int64_t pitch, int64_t chunk) {
    constexpr int NTH = 64 * WI * WO, NT = std::is_same_v<T, bf16_t> ? 1 : 3, BK = (int)kDyTile;
    constexpr int NX = BK * BI / 16 / NTH;               // 16 codes each
    constexpr int E = 16 / sizeof(T), NY = BK * BO / E / NTH;
    constexpr int FI = BI / WI / 32, FO = BO / WO / 32;
    static_assert(NX >= 1 && NY >= 1 && NX * NTH * 16 == BK * BI && NY * NTH * E == BK * BO, "tile does not fill the block");
    __shared__ __attribute__((aligned(16))) bf16_t xs[2][BK * BI];
    __shared__ __attribute__((aligned(16))) bf16_t ys[2][NT][BK * BO];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int tiles_i = (int)((a.inner + BI - 1) / BI);
    // Workgroups go to the 8 XCDs in turn: each takes one run of tiles, so that the
    // columns of dy, the larger operand, are read by one XCD's L2 only.
    int tile = blockIdx.x;
    const int per = gridDim.x / 8;
    if (tile < 8 * per) tile = tile % 8 * per + tile / 8;
    const int64_t i0 = (int64_t)(tile % tiles_i) * BI, o0 = (int64_t)(tile / tiles_i) * BO;
    const int64_t t0 = blockIdx.y * chunk, t1 = min(a.tokens, t0 + chunk);
    const T* dy = static_cast<const T*>(a.dy);

    // BK tokens on their way into registers.  Past the last token and past the
    // last column they are copies of the last ones there are: columns past the end
    // are never stored, rows are cleared by store().
    u32x4 rx[NX], ry[NY];
    int re[NX];
    const int8_t* px[NX];
    const int8_t* pe[NX];
    const T* py[NY];
    const int64_t pitch_e = pitch / kCkptGroup;
#pragma unroll
    for (int n = 0; n < NX; ++n) {
        const int64_t c = min(i0 + 16 * ((tid + n * NTH) % (BI / 16)), pitch - 16), row = t0 + (tid + n * NTH) / (BI / 16);
        px[n] = a.x.codes + row * pitch + c;
        pe[n] = a.x.exps + row * pitch_e + c / kCkptGroup;
    }
#pragma unroll
    for (int n = 0; n < NY; ++n) {
        const int64_t c = o0 + E * ((tid + n * NTH) % (BO / E)), row = t0 + (tid + n * NTH) / (BO / E);
        py[n] = dy + row * a.ld_dy + min(c, ROWS == DyRows::Whole ? a.outer - E : a.outer - 1);
    }
    // Item n of the tile of tokens t .., `last` if that is the last one; moves on.
    auto load_x = [&](int n, int64_t t, auto last) {
        const int64_t over = decltype(last)::value ? max(t + (tid + n * NTH) / (BI / 16) - (t1 - 1), (int64_t)0) : 0;
        rx[n] = *reinterpret_cast<const u32x4*>(px[n] - over * pitch);
        re[n] = pe[n][-over * pitch_e];
        px[n] += BK * pitch;
        pe[n] += BK * pitch_e;
    };
    auto load_y = [&](int n, int64_t t, auto last) {
        const int64_t over = decltype(last)::value ? max(t + (tid + n * NTH) / (BO / E) - (t1 - 1), (int64_t)0) : 0;
        const T* p = py[n] - over * a.ld_dy;
        if constexpr (ROWS == DyRows::Whole || (ROWS == DyRows::Ragged && !decltype(last)::value)) {
            ry[n] = *reinterpret_cast<const typename Sixteen<T>::type*>(p);
        } else {
            const int64_t left = a.outer - (o0 + E * ((tid + n * NTH) % (BO / E)));
            T v[E];
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = i < left ? p[i] : T(0.f);
            __builtin_memcpy(&ry[n], v, 16);
        }
        py[n] += BK * a.ld_dy;
    };
    // value = code * step, exactly for every step from 2^-126 to 2^121; the builtin
    // makes the byte's sign a part of its conversion (one instruction).
    auto store_x = [&](int n, int buf, int64_t t, auto last) {
        const int e = tid + n * NTH, c = e % (BI / 16), k = e / (BI / 16);
        float step = step_of(re[n]);
        if (decltype(last)::value && t + k >= t1) step = 0.f;
        bf16x8 v[2];
#pragma unroll
        for (int i = 0; i < 16; ++i)
            v[i / 8][i % 8] = (bf16_t)((float)(int)__builtin_amdgcn_sbfe(rx[n][i / 4], 8 * (i % 4), 8) * step);
        *reinterpret_cast<bf16x8*>(xs[buf] + widx<BI>(k, 2 * c)) = v[0];
        *reinterpret_cast<bf16x8*>(xs[buf] + widx<BI>(k, 2 * c + 1)) = v[1];
    };
    auto store_y = [&](int n, int buf, int64_t t, auto last) {
        const int e = tid + n * NTH, c = e % (BO / E), k = e / (BO / E);
        u32x4 r = ry[n];
        if (decltype(last)::value && t + k >= t1) r = u32x4{0, 0, 0, 0};
        if constexpr (NT == 1) {
            *reinterpret_cast<u32x4*>(ys[buf][0] + widx<BO>(k, c)) = r;
        } else {
            // Top halves of the four values, then of what is left, twice.
            uint32_t w[3][2], top = 0;
            float x[4];
            __builtin_memcpy(x, &r, 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) top = max(top, r[i] & 0x7fffffffu);
            const bool odd = top >= 0x7f800000u;     // an infinity is its own first term
#pragma unroll
            for (int p = 0; p < 3; ++p)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const uint32_t u0 = __builtin_bit_cast(uint32_t, x[i]), u1 = __builtin_bit_cast(uint32_t, x[i + 1]);
                    w[p][i / 2] = __builtin_amdgcn_perm(u1, u0, 0x07060302u);
                    const float f0 = __builtin_bit_cast(float, u0 & 0xffff0000u);
                    const float f1 = __builtin_bit_cast(float, u1 & 0xffff0000u);
                    x[i] = odd && x[i] == f0 ? 0.f : x[i] - f0;
                    x[i + 1] = odd && x[i + 1] == f1 ? 0.f : x[i + 1] - f1;
                }
#pragma unroll
            for (int p = 0; p < 3; ++p)
                *reinterpret_cast<u32x2*>(ys[buf][p] + widx<BO>(k, c / 2) + 4 * (c & 1)) = u32x2{w[p][0], w[p][1]};
        }
    };

    const int wi = (wave % WI) * (BI / WI), wo = (wave / WI) * (BO / WO);
    f32x16 acc[FI][FO] = {};
    const std::true_type yes;
    const std::false_type no;
    // One step: the products of the tile in buffer `buf`, between them the next
    // tile (tokens t + BK ..) from registers to LDS and the loads of the one after
    // it, item by item.  All three are in one block without branches, so that the
    // matrix instructions of a wave cover its own conversions and LDS traffic.
    constexpr int S = BK / 16, SUB = S * NT;
    auto step = [&](int buf, int64_t t, auto do_store, auto store_last, auto do_load, auto load_last) {
        bf16x8 fx[S][FI], fy[2][FO];
        auto read_y = [&](int q) {                   // q: sub-step, terms fastest, the smallest first
#pragma unroll
            for (int j = 0; j < FO; ++j) fy[q & 1][j] = wfrag<BO>(ys[buf][NT - 1 - q % NT], wo + 32 * j, q / NT, lane);
        };
        auto read_x = [&](int s) {
#pragma unroll
            for (int i = 0; i < FI; ++i) fx[s][i] = wfrag<BI>(xs[buf], wi + 32 * i, s, lane);
        };
        read_x(0);
        read_y(0);
#pragma unroll
        for (int q = 0; q < SUB; ++q) {
            if (q + 1 < SUB) {
                if ((q + 1) % NT == 0) read_x((q + 1) / NT);
                read_y(q + 1);
            }
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int j = 0; j < FO; ++j)
                    acc[i][j] = OI ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(fy[q & 1][j], fx[q / NT][i], acc[i][j], 0, 0, 0)
                                   : __builtin_amdgcn_mfma_f32_32x32x16_bf16(fx[q / NT][i], fy[q & 1][j], acc[i][j], 0, 0, 0);
            if constexpr (decltype(do_store)::value) {
#pragma unroll
                for (int n = 0; n < NX; ++n)
                    if (n * SUB / NX == q) {
                        store_x(n, buf ^ 1, t + BK, store_last);
                        if constexpr (decltype(do_load)::value) load_x(n, t + 2 * BK, load_last);
                    }
#pragma unroll
                for (int n = 0; n < NY; ++n)
                    if (n * SUB / NY == q) {
                        store_y(n, buf ^ 1, t + BK, store_last);
                        if constexpr (decltype(do_load)::value) load_y(n, t + 2 * BK, load_last);
                    }
            }
        }
    };
    const int steps = (int)((t1 - t0 + BK - 1) / BK);
    auto load = [&](int64_t t) {
#pragma unroll
        for (int n = 0; n < NX; ++n) load_x(n, t, yes);
#pragma unroll
        for (int n = 0; n < NY; ++n) load_y(n, t, yes);
    };
    if (steps > 0) {
        load(t0);
#pragma unroll
        for (int n = 0; n < NX; ++n) store_x(n, 0, t0, yes);
#pragma unroll
        for (int n = 0; n < NY; ++n) store_y(n, 0, t0, yes);
        if (steps > 1) load(t0 + BK);
    }
    int it = 0;
    int64_t t = t0;
    for (; it + 3 < steps; ++it, t += BK) {
        lds_barrier();
        step(it & 1, t, yes, no, yes, no);
    }
    if (it + 2 < steps) {
        lds_barrier();
        step(it++ & 1, t, yes, no, yes, yes);
        t += BK;
    }
    if (it + 1 < steps) {
        lds_barrier();
        step(it++ & 1, t, yes, yes, no, no);
        t += BK;
    }
    if (it < steps) {
        lds_barrier();
        step(it & 1, t, no, no, no, no);
    }
    // Lane l: column l % 32 (the contiguous side of the stored matrix), rows
    // 8 (r / 4) + 4 (l / 32) + r % 4.
    const int64_t nr = OI ? a.outer : a.inner, nc = OI ? a.inner : a.outer;
    const bool whole = a.splits == 1;
    float* out = whole ? a.dw : a.partial + blockIdx.y * nr * nc;
    const int64_t ld = whole ? a.ld_dw : nc;
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FO; ++j)
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

// Adds the shares of the tokens in their order, four columns a thread.
__global__ void __launch_bounds__(kThreads) wgrad_join_kernel(WgradArgs a, bool vec) {
    const int64_t nr = a.oi ? a.outer : a.inner, nc = a.oi ? a.inner : a.outer;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (vec) {
        if (4 * i >= nr * nc) return;
        f32x4 s = {};
#pragma unroll 4
        for (int k = 0; k < a.splits; ++k) s += *reinterpret_cast<const f32x4*>(a.partial + k * nr * nc + 4 * i);
        f32x4* p = reinterpret_cast<f32x4*>(a.dw + 4 * i / nc * a.ld_dw + 4 * i % nc);
        *p = a.accumulate ? *p + s : s;
        return;
    }
    for (int64_t e = 4 * i; e < min(4 * i + 4, nr * nc); ++e) {
        float s = 0.f;
        for (int k = 0; k < a.splits; ++k) s += a.partial[k * nr * nc + e];
        float* p = a.dw + e / nc * a.ld_dw + e % nc;
        *p = a.accumulate ? *p + s : s;
    }
}

unsigned blocks_of(int64_t rows, int64_t pitch) {
    return (unsigned)((rows * pitch / kV + kThreads - 1) / kThreads);
}

template <class T>
hipError_t pack(Act act, const CkptPackArgs& a, hipStream_t s) {
    const int64_t pitch = ckpt_pitch(a.cols);
    const unsigned n = blocks_of(a.rows, pitch);
    if (act == Act::None) pack_kernel<T, Act::None><<<n, kThreads, 0, s>>>(a, pitch);
    else if (act == Act::Gelu) pack_kernel<T, Act::Gelu><<<n, kThreads, 0, s>>>(a, pitch);
    else pack_kernel<T, Act::Swiglu><<<n, kThreads, 0, s>>>(a, pitch);
    return hipGetLastError();
}

template <class T>
hipError_t act_grad(Act act, const CkptGradArgs& a, hipStream_t s) {
    const int64_t pitch = ckpt_pitch(a.cols);
    const unsigned n = blocks_of(a.rows, pitch);
    if (act == Act::Gelu) act_grad_kernel<T, Act::Gelu><<<n, kThreads, 0, s>>>(a, pitch);
    else act_grad_kernel<T, Act::Swiglu><<<n, kThreads, 0, s>>>(a, pitch);
    return hipGetLastError();
}

template <class T, bool OI, int BI, int BO, int WI, int WO>
void wgrad_pass(const WgradArgs& a, DyRows rows, hipStream_t s) {
    const int64_t tiles = ((a.inner + BI - 1) / BI) * ((a.outer + BO - 1) / BO);
    const int64_t chunk = ((a.tokens + a.splits - 1) / a.splits + 31) / 32 * 32;
    const dim3 grid((unsigned)tiles, (unsigned)a.splits);
    const int64_t pitch = ckpt_pitch(a.inner);
    if (rows == DyRows::Whole)
        wgrad_kernel<T, OI, DyRows::Whole, BI, BO, WI, WO><<<grid, 64 * WI * WO, 0, s>>>(a, pitch, chunk);
    else if (rows == DyRows::Ragged)
        wgrad_kernel<T, OI, DyRows::Ragged, BI, BO, WI, WO><<<grid, 64 * WI * WO, 0, s>>>(a, pitch, chunk);
    else if constexpr (BI * BO < 256 * 256)
        wgrad_kernel<T, OI, DyRows::Narrow, BI, BO, WI, WO><<<grid, 64 * WI * WO, 0, s>>>(a, pitch, chunk);
}

// bf16: 256 x 256 tiles (64 KB of LDS, 128 accumulators a lane) where there are
// 128 of them or more, else 128 x 128, as for a few narrow columns of dy; fp32,
// three products a tile: 256 x 128.
bool wgrad_large(int64_t inner, int64_t outer) { return ((inner + 255) / 256) * ((outer + 255) / 256) >= 128; }

template <bool OI>
void wgrad(DType t, const WgradArgs& a, hipStream_t s) {
    const DyRows rows = dy_rows(a.outer, a.ld_dy, t == DType::F32 ? 4 : 8);
    if (t == DType::F32) wgrad_pass<float, OI, 256, 128, 4, 2>(a, rows, s);
    else if (wgrad_large(a.inner, a.outer) && rows != DyRows::Narrow) wgrad_pass<bf16_t, OI, 256, 256, 2, 4>(a, rows, s);
    else wgrad_pass<bf16_t, OI, 128, 128, 2, 2>(a, rows, s);
}

}  // namespace

hipError_t launch_ckpt_pack(DType t, Act act, const CkptPackArgs& a, hipStream_t s) {
    return t == DType::BF16 ? pack<bf16_t>(act, a, s) : pack<float>(act, a, s);
}

hipError_t launch_ckpt_unpack(DType t, const CkptUnpackArgs& a, hipStream_t s) {
    const int64_t pitch = ckpt_pitch(a.cols);
    const unsigned n = blocks_of(a.rows, pitch);
    if (t == DType::BF16) unpack_kernel<bf16_t><<<n, kThreads, 0, s>>>(a, pitch);
    else unpack_kernel<float><<<n, kThreads, 0, s>>>(a, pitch);
    return hipGetLastError();
}

hipError_t launch_ckpt_act_grad(DType t, Act act, const CkptGradArgs& a, hipStream_t s) {
    return t == DType::BF16 ? act_grad<bf16_t>(act, a, s) : act_grad<float>(act, a, s);
}

// Shares of the tokens: the number that this estimate of the time finds best, in
// us: 0.4 (fp32 1.3) for a step of 32 tokens of a CU's block, 3/5 of that for each
// more block of 128 x 128 on a CU, a whole step for each more of fp32; 4 for the
// launch that joins the shares, and their bytes written and read at 3 TB/s.
// Estimated and measured with 1, 2, 4, 8 shares: bf16 8192 x 768 x 2304 108 71 55 73
// and 118 73 64 74, 2048^3 32 47 - - and 41 43 55 76, 600 x 2048 x 1024 14 25 - - and
// 19 27 27 38; fp32 4001 x 768 x 2304 164 95 65 83 and 164 93 64 75, 2048^3 83 68 91 -
// and 94 70 83 110.
int wgrad_splits(DType t, int64_t tokens, int64_t inner, int64_t outer) {
    if (t == DType::BF16 && wgrad_large(inner, outer)) return 1;
    const bool f32 = t == DType::F32;
    const int64_t bi = f32 ? 256 : 128, tiles = ((inner + bi - 1) / bi) * ((outer + 127) / 128);
    const int64_t steps = (tokens + 31) / 32;
    int best = 1;
    double least = 0.;
    for (int n = 1; n <= 32 && n <= (steps > 1 ? steps : 1); ++n) {
        const double blocks = (double)tiles * n / 256.;
        const double load = f32 ? std::ceil(blocks) : blocks > 1. / 0.6 ? 0.6 * blocks : 1.;
        const double us = (double)((steps + n - 1) / n) * (f32 ? 1.3 : 0.4) * load +
                          (n > 1 ? 4. + 8. * n * (double)inner * (double)outer / 3e6 : 0.);
        if (n == 1 || us < least) {
            best = n;
            least = us;
        }
    }
    return best;
}

hipError_t launch_wgrad(DType t, const WgradArgs& a, hipStream_t s) {
    if (a.oi) wgrad<true>(t, a, s);
    else wgrad<false>(t, a, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t n = a.inner * a.outer, nc = a.oi ? a.inner : a.outer;
    wgrad_join_kernel<<<(unsigned)((n + 4 * kThreads - 1) / (4 * kThreads)), kThreads, 0, s>>>(a, nc % 4 == 0 && a.ld_dw % 4 == 0 && reinterpret_cast<uintptr_t>(a.dw) % 16 == 0);
    return hipGetLastError();
}

}  // namespace np
