// Norm of every query and key head and the rotation of their positions, in one pass,
// and its backward pass.  For a head x of D features and pair i of its turning features,
//   n_d = x_d r w_d,  r = 1 / sqrt(mean_d x_d^2 + eps)          (norm; else n = x)
//   (y_a, y_b) = (n_a cos t - n_b sin t, n_a sin t + n_b cos t),  t = position * f_i
// and the other features are n itself.  Backward, with g the gradient of y turned back by t:
//   dw_d = sum over rows g_d x_d r,  h_d = g_d w_d,  dx_d = r (h_d - x_d r mean_d(h_d x_d r)).
//
// Bound by memory (forward: each head read and written once; backward: x and dy read, dx
// written): 16384 tokens, 16/8 heads of 128, bf16 38-45 us forward (201 MB; less where the last-level
// cache holds a part), 64 backward and 5 for the weights' sums (302 MB), where a copy's rate of
// 4.76 TB/s would take 42 and 63; fp32 85 forward (403 MB), 207 with the backward pass (1007 MB), a copy 85 and 211.
//
// A group of L lanes has one token and takes heads of it in turn, each lane E pairs, so that
// an angle serves several heads and is not read from a table: position * f in 64 bits (in 32 the
// angle of position 10^6 is off by 0.06), reduced to a quarter turn, then polynomials.
// Queries and keys go to blocks of their own: with weights and their gradients of one operand
// registers do for four waves a SIMD, but for 14 to 16 that the backward pass of bf16
// spills (both operands in one block: 75 us backward).  A lane's pairs are whole 16-byte
// chunks of the two halves of a row (or of its adjacent pairs), so a rotation needs no other
// lane, and the mean of squares log2 L exchanges.  Where they are not, lanes go feature by feature,
// at up to four times a copy's time: us forward and both passes of 16384 tokens, bf16, (a copy's): 41 pairs
// of 16/8 heads of 128 98 288 (42 106), 36 of 16/16 of 72 110 266 (32 79), 10 of 80 119 264 (35
// 88), 25 of 51 81 200 (22 56), and in whole chunks 40 of 80 42 106 (35 88); fp32, 41 of 16/8 of
// 128 97 227 (85 211).
//
// Squares are summed in 64 bits and a row is brought near 1 by a power of two, so rows at
// either end of fp32's range keep their norm; the rest is fp32 and rounded once.
// Weight gradients are summed per lane over its rows, then over the block, then over blocks
// in their order (in 64 bits): the same bits every time, no atomics.
#include "np_rope.h"

#include <cmath>
#include <type_traits>

namespace np {
namespace {

typedef __bf16 bf16_t;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));   // global memory takes 16 bytes on any byte

constexpr int kThreads = 256;

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ double dpp(double v) {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    const i32x2 b = __builtin_bit_cast(i32x2, v);
    return __builtin_bit_cast(double, i32x2{__builtin_amdgcn_update_dpp(0, b.x, CTRL, 0xf, 0xf, true),
                                            __builtin_amdgcn_update_dpp(0, b.y, CTRL, 0xf, 0xf, true)});
}

// Sum over groups of L lanes (4 to 32), the same in each: with the lane 1 and 2 away,
// then the mirrored one of 8 and 16 lanes, whose quads hold the missing half.
template <int L, class V>
__device__ __forceinline__ V group_sum(V v) {
    v += dpp<0xb1>(v);
    v += dpp<0x4e>(v);
    if constexpr (L >= 8) v += dpp<0x141>(v);
    if constexpr (L >= 16) v += dpp<0x140>(v);
    if constexpr (L >= 32) v += __shfl_xor(v, 16, 64);
    return v;
}

// cos and sin of p f pi / 2: whole quarter turns are taken off in 64 bits (added to 1.5 2^52 the
// product is rounded to them, with their number in the lowest bits: up to 2^51 of them), then
// Taylor polynomials of angles up to pi / 4 (what they leave out is below 2^-28 of the result).
__device__ __forceinline__ void turn(double p, double f, float& c, float& s) {
    const double q = p * f, up = q + 6755399441055744.0, whole = up - 6755399441055744.0;
    const float x = (float)(q - whole) * 1.57079632679489661923f, x2 = x * x;
    float u = x2 * 2.7557319223985893e-6f - 1.9841269841269841e-4f;    // 1/9!, 1/7!
    u = __builtin_fmaf(u, x2, 8.3333333333333333e-3f);
    u = __builtin_fmaf(u, x2, -1.6666666666666667e-1f);
    const float sn = __builtin_fmaf(u * x2, x, x);
    float v = x2 * -2.7557319223985888e-7f + 2.4801587301587302e-5f;   // 1/10!, 1/8!
    v = __builtin_fmaf(v, x2, -1.3888888888888889e-3f);
    v = __builtin_fmaf(v, x2, 4.1666666666666667e-2f);
    v = __builtin_fmaf(v, x2, -0.5f);
    const float cs = __builtin_fmaf(v, x2, 1.f);
    const uint32_t k = (uint32_t)__builtin_bit_cast(uint64_t, up);       // modulo 4
    const float a = k & 1 ? sn : cs, b = k & 1 ? cs : sn;
    c = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, a) ^ ((k + 1) << 30 & 0x80000000u));
    s = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, b) ^ (k << 30 & 0x80000000u));
}

// Where the pairs of a lane lie in a row.  VEC: two chunks of E features, from0 and
// from1: halves of a turning row's pairs, or (ADJ, and features that do not turn) side by
// side.  Otherwise pair e of the lane is pair l + e L of the row.
template <class T, int L, bool VEC, bool ADJ>
struct Row {
    static constexpr int E = VEC ? 16 / sizeof(T) : 4;
    int l, dim, pairs;
    __device__ __forceinline__ int pair(int e) const { return VEC ? l * E + e : l + e * L; }
    __device__ __forceinline__ bool turns(int e) const { return pair(e) < pairs; }
    __device__ __forceinline__ int from0() const { return !ADJ && l * E < pairs ? l * E : 2 * l * E; }
    __device__ __forceinline__ int from1() const { return !ADJ && l * E < pairs ? l * E + pairs : 2 * l * E + E; }
    // Features of pair e; dim and above: none.
    __device__ __forceinline__ int first(int e) const {
        if constexpr (VEC) return ADJ ? (e < E / 2 ? from0() + 2 * e : from1() + 2 * e - E) : from0() + e;
        const int p = pair(e);
        return ADJ || p >= pairs ? 2 * p : p;
    }
    __device__ __forceinline__ int second(int e) const {
        if constexpr (VEC) return ADJ ? first(e) + 1 : from1() + e;
        const int p = pair(e);
        return ADJ || p >= pairs ? 2 * p + 1 : p + pairs;
    }
    template <class U>
    __device__ __forceinline__ void pick(const U (&x)[E], const U (&y)[E], U (&a)[E], U (&b)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if constexpr (ADJ) {
                a[e] = e < E / 2 ? x[2 * e % E] : y[2 * e % E];
                b[e] = e < E / 2 ? x[2 * e % E + 1] : y[2 * e % E + 1];
            } else {
                a[e] = x[e];
                b[e] = y[e];
            }
        }
    }
    // E numbers from p on.
    template <class U>
    static __device__ __forceinline__ void pieces(const U* p, U (&x)[E]) {
        u32x4 r[E * sizeof(U) / 16];
#pragma unroll
        for (int i = 0; i < (int)(E * sizeof(U) / 16); ++i) r[i] = reinterpret_cast<const u32x4_any*>(p)[i];
        __builtin_memcpy(x, r, sizeof x);
    }
    template <class U>
    __device__ __forceinline__ void weights(const U* row, float (&a)[E], float (&b)[E]) const {
        U p[E] = {}, q[E] = {};
        if constexpr (VEC && E * sizeof(U) % 16 == 0) {
            U x[E] = {}, y[E] = {};
            if (from0() < dim) pieces(row + from0(), x);
            if (from1() < dim) pieces(row + from1(), y);
            pick(x, y, p, q);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (first(e) < dim) p[e] = row[first(e)];
                if (second(e) < dim) q[e] = row[second(e)];
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            a[e] = (float)p[e];
            b[e] = (float)q[e];
        }
    }
    // Of the lane's pairs, in quarter turns a step (0 for those that stay).
    __device__ __forceinline__ void frequencies(const double* freqs, double (&f)[E]) const {
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = 0.0;
        if (VEC && pair(E - 1) < pairs) pieces(freqs + pair(0), f);
        else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (pair(e) < pairs) f[e] = freqs[pair(e)];
        }
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] *= 0.63661977236758134308;
    }
    __device__ __forceinline__ void load(const T* row, bool live, float (&a)[E], float (&b)[E]) const {
        T p[E], q[E];
        if constexpr (VEC) {
            u32x4 x = {}, y = {};
            if (live && from0() < dim) x = *reinterpret_cast<const u32x4_any*>(row + from0());
            if (live && from1() < dim) y = *reinterpret_cast<const u32x4_any*>(row + from1());
            T u[E], v[E];
            __builtin_memcpy(u, &x, 16);
            __builtin_memcpy(v, &y, 16);
            pick(u, v, p, q);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                p[e] = live && first(e) < dim ? row[first(e)] : (T)0.f;
                q[e] = live && second(e) < dim ? row[second(e)] : (T)0.f;
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            a[e] = (float)p[e];
            b[e] = (float)q[e];
        }
    }
    __device__ __forceinline__ void store(T* row, bool live, const float (&a)[E], const float (&b)[E]) const {
        if constexpr (VEC) {
            T u[E], v[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if constexpr (ADJ) {
                    (e < E / 2 ? u : v)[2 * e % E] = (T)a[e];
                    (e < E / 2 ? u : v)[2 * e % E + 1] = (T)b[e];
                } else {
                    u[e] = (T)a[e];
                    v[e] = (T)b[e];
                }
            }
            u32x4 x, y;
            __builtin_memcpy(&x, u, 16);
            __builtin_memcpy(&y, v, 16);
            if (live && from0() < dim) *reinterpret_cast<u32x4_any*>(row + from0()) = x;
            if (live && from1() < dim) *reinterpret_cast<u32x4_any*>(row + from1()) = y;
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                if (live && first(e) < dim) row[first(e)] = (T)a[e];
                if (live && second(e) < dim) row[second(e)] = (T)b[e];
            }
        }
    }
};

template <class T, int L, bool VEC, bool ADJ, bool BACK>
__global__ void __launch_bounds__(kThreads, 4) rope_kernel(RopeArgs a, int shares_log2) {
    using R = Row<T, L, VEC, ADJ>;
    constexpr int E = R::E, G = kThreads / L;        // pairs of a lane, groups of a block
    const R at{(int)threadIdx.x % L, a.dim, a.pairs};
    const int64_t items = a.tokens << shares_log2, step = (int64_t)gridDim.x * G;
    const int shares = 1 << shares_log2;

    const int o = blockIdx.y;                        // queries or keys
    float w[2][E];
    if (!a.w[o]) {
#pragma unroll
        for (int e = 0; e < E; ++e) w[0][e] = w[1][e] = 1.f;
    } else if (a.weight_bf16) at.weights(static_cast<const bf16_t*>(a.w[o]), w[0], w[1]);
    else at.weights(static_cast<const float*>(a.w[o]), w[0], w[1]);
    double freq[E];                                  // quarter turns a step
    at.frequencies(a.freqs, freq);
    uint64_t axes = 0;                               // of the pairs, a byte each
    if (a.axis)
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (at.turns(e)) axes |= (uint64_t)min((uint32_t)a.axis[at.pair(e)], (uint32_t)a.axes - 1) << (8 * e);
    float dw[2][E] = {};

    for (int64_t item = (int64_t)blockIdx.x * G + threadIdx.x / L; item - threadIdx.x / L < items; item += step) {
        const bool live = item < items;              // all lanes of a wave stay for the exchanges
        const int64_t token = live ? item >> shares_log2 : 0;
        const int share = (int)item & (shares - 1);
        float c[E], s[E];
        auto position = [&](int64_t n) {
            return a.positions_64 ? (double)static_cast<const int64_t*>(a.positions)[n]
                                  : (double)static_cast<const int32_t*>(a.positions)[n];
        };
        const double pos = a.pairs > 0 && !a.axis ? position(token) : 0.0;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            double here = pos;
            if (a.axis) here = position((int64_t)(axes >> (8 * e) & 255) * a.position_stride + token);
            turn(here, freq[e], c[e], s[e]);
        }
        for (int h0 = 0; h0 < a.heads[o]; h0 += shares) {
            const int h = h0 + share;
            const bool on = live && h < a.heads[o];
            const int64_t hh = on ? h : 0;
            auto row = [&](const AttnOperand& x) { return static_cast<T*>(x.p) + token * x.tok + hh * x.head; };
            float x[2][E];
            float r = 1.f;
            int size = 0;
            if (!BACK || a.norm) {
                at.load(row(a.x[o]), on, x[0], x[1]);
                if (a.norm) {
                    double sum = 0.0;
#pragma unroll
                    for (int e = 0; e < E; ++e)
#pragma unroll
                        for (int m = 0; m < 2; ++m) sum = __builtin_fma((double)x[m][e], (double)x[m][e], sum);
                    const double mean = group_sum<L>(sum) * a.inv_dim + a.eps;
                    double q = __builtin_amdgcn_rsq(mean);
                    q *= 1.5 - 0.5 * mean * q * q;
                    // Rows are brought near 1 by a power of two, so that 1 / rms is a normal fp32 number also for
                    // subnormal rows with eps 0 and at the range's end: exact but for features that round
                    // to 0 in the result (the same time: 112 us for 16384 tokens, 16/8 heads of 128).
                    size = -(__builtin_amdgcn_frexp_exp(mean) >> 1);
                    q = __builtin_amdgcn_ldexp(q, -size);
                    r = !on || mean == INFINITY ? 0.f : (float)q;    // a row that is not there: 0, also where eps is
#pragma unroll
                    for (int e = 0; e < E; ++e)
#pragma unroll
                        for (int m = 0; m < 2; ++m) x[m][e] = __builtin_amdgcn_ldexpf(x[m][e], size) * r;
                }
            }
            float y[2][E];
            if constexpr (!BACK) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float u = x[0][e] * w[0][e], v = x[1][e] * w[1][e];
                    // Features that do not turn never meet another.
                    y[0][e] = at.turns(e) ? u * c[e] - v * s[e] : u;
                    y[1][e] = at.turns(e) ? u * s[e] + v * c[e] : v;
                }
            } else {
                float g[2][E];
                at.load(row(a.g[o]), on, g[0], g[1]);
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    y[0][e] = at.turns(e) ? g[0][e] * c[e] + g[1][e] * s[e] : g[0][e];
                    y[1][e] = at.turns(e) ? g[1][e] * c[e] - g[0][e] * s[e] : g[1][e];
                    if (a.norm)
#pragma unroll
                        for (int m = 0; m < 2; ++m) {
                            dw[m][e] = __builtin_fmaf(y[m][e], x[m][e], dw[m][e]);
                            y[m][e] *= w[m][e];
                            sum = __builtin_fmaf(y[m][e], x[m][e], sum);
                        }
                }
                if (a.norm) {
                    const float mean = group_sum<L>(sum) * (float)a.inv_dim;
#pragma unroll
                    for (int e = 0; e < E; ++e)
#pragma unroll
                        for (int m = 0; m < 2; ++m) y[m][e] = __builtin_amdgcn_ldexpf(r * (y[m][e] - x[m][e] * mean), size);
                }
            }
            at.store(row(a.y[o]), on, y[0], y[1]);
        }
    }

    if constexpr (BACK) {
        if (!a.partial) return;                      // the same for all
        __shared__ float part[kThreads / 64][2][E][L];
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float v = dw[m][e];
#pragma unroll
                for (int k = L; k < 64; k <<= 1) v += __shfl_xor(v, k, 64);
                if (lane < L) part[wave][m][e][lane] = v;
            }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * E * L; i += kThreads) {
            const int l = i % L, e = i / L % E, m = i / (L * E);
            float v = 0.f;
#pragma unroll
            for (int k = 0; k < kThreads / 64; ++k) v += part[k][m][e][l];
            const R to{l, a.dim, a.pairs};
            const int d = m ? to.second(e) : to.first(e);
            if (d < a.dim) a.partial[((int64_t)blockIdx.x * 2 + o) * a.dim + d] = v;
        }
    }
}

// Weight gradients from the blocks' sums: 16 features a block, 64 threads for each.
constexpr int kJoinColumns = 16, kJoinRows = 64;
__global__ void __launch_bounds__(kJoinColumns * kJoinRows) rope_join_kernel(RopeArgs a, int blocks) {
    __shared__ double part[kJoinRows][kJoinColumns];
    const int c = threadIdx.x % kJoinColumns, r = threadIdx.x / kJoinColumns;
    const int d = blockIdx.x * kJoinColumns + c, all = 2 * a.dim;
    double sum = 0.0;
    if (d < all) {
#pragma unroll 8
        for (int b = r; b < blocks; b += kJoinRows) sum += (double)a.partial[(int64_t)b * all + d];
    }
    part[r][c] = sum;
    __syncthreads();
    if (r == 0 && d < all) {
#pragma unroll 8
        for (int i = 1; i < kJoinRows; ++i) sum += part[i][c];
        float* dw = a.dw[d / a.dim];
        if (dw) dw[d % a.dim] = (float)sum;
    }
}

// Whether a lane's pairs are whole chunks of 16 bytes.
template <class T>
bool whole_chunks(const RopeArgs& a) {
    constexpr int E = 16 / sizeof(T);
    return a.dim % E == 0 && (a.adjacent || a.pairs % E == 0);
}

// Lanes of a group: enough for every pair (and a feature without a partner).
template <class T>
int lanes(const RopeArgs& a) {
    const int e = whole_chunks<T>(a) ? 16 / (int)sizeof(T) : 4, need = ((a.dim + 1) / 2 + e - 1) / e;
    return need <= 4 ? 4 : need <= 8 ? 8 : need <= 16 ? 16 : 32;
}

// Groups of lanes that share a token's heads (log 2): 48 K groups of one operand or 384 K lanes, or
// one head each.  More of them hide more latency, but make every angle as many times; with several
// axes a position is read for every pair, and a third is enough.  us forward, backward
// with 1, 2, 4, 8 groups a token: 16384 tokens, 16/8 heads of 128, bf16 40.4 71.5, 42.5 68.5, 37.6 64.6,
// 38.8 67.0 (three axes, forward: 45.6 48.3 52.1 60.7); 12/12 of 64, bf16 19.3 43.4, 18.8 39.6, 18.9 38.7, 22.2
// 42.7; 6930 tokens, 16/16 of 80, fp32, forward 37.7 30.0 28.5 32.1 (three axes 38.9 31.9 33.1 40.1); 572, 32/8 of 64,
// bf16 22.8 54.4, 13.4 31.1, 13.4 24.1, 13.0 23.9.
template <class T>
int shares_log2(const RopeArgs& a) {
    const int most = a.heads[0] > a.heads[1] ? a.heads[0] : a.heads[1], part = a.axis ? 3 : 1;
    int n = 0;
    while (part * (a.tokens << n) < 3 << 14 && part * (a.tokens * lanes<T>(a) << n) < 3 << 17 && 1 << n < most) ++n;
    return n;
}

// Blocks of each operand.  With weight gradients as many as the chip holds at once: a block
// sums over all that it does and writes one row of them (16384 tokens, 16/8 of 128, bf16: 512 blocks
// 64.6 us, 768 67.3, 1024 67.0).
template <class T>
int blocks(const RopeArgs& a, bool backward) {
    const int64_t groups = a.tokens << shares_log2<T>(a), n = (groups * lanes<T>(a) + kThreads - 1) / kThreads;
    const int64_t most = backward && rope_sums(a) ? kRopeMostSums : 1024;
    return (int)(n < most ? n : most);
}

template <class T, int L, bool VEC, bool ADJ>
void launch(const RopeArgs& a, bool backward, hipStream_t s) {
    const int n = blocks<T>(a, backward), shares = shares_log2<T>(a);
    if (backward) rope_kernel<T, L, VEC, ADJ, true><<<dim3(n, 2), kThreads, 0, s>>>(a, shares);
    else rope_kernel<T, L, VEC, ADJ, false><<<dim3(n, 2), kThreads, 0, s>>>(a, shares);
}

template <class T, int L>
void launch(const RopeArgs& a, bool backward, hipStream_t s) {
    if (whole_chunks<T>(a)) a.adjacent ? launch<T, L, true, true>(a, backward, s) : launch<T, L, true, false>(a, backward, s);
    else a.adjacent ? launch<T, L, false, true>(a, backward, s) : launch<T, L, false, false>(a, backward, s);
}

template <class T>
hipError_t run(const RopeArgs& a, bool backward, hipStream_t s) {
    if (a.tokens > 0) switch (lanes<T>(a)) {
        case 4: launch<T, 4>(a, backward, s); break;
        case 8: launch<T, 8>(a, backward, s); break;
        case 16: launch<T, 16>(a, backward, s); break;
        default: launch<T, 32>(a, backward, s);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !backward || !rope_sums(a)) return e;
    rope_join_kernel<<<(2 * a.dim + kJoinColumns - 1) / kJoinColumns, kJoinColumns * kJoinRows, 0, s>>>(a, blocks<T>(a, true));
    return hipGetLastError();
}

}  // namespace

int64_t rope_workspace(DType t, const RopeArgs& a) {
    if (!rope_sums(a)) return 0;
    return (int64_t)2 * a.dim * (t == DType::BF16 ? blocks<bf16_t>(a, true) : blocks<float>(a, true));
}

hipError_t launch_rope(DType t, const RopeArgs& a, bool backward, hipStream_t s) {
    return t == DType::BF16 ? run<bf16_t>(a, backward, s) : run<float>(a, backward, s);
}

}  // namespace np
