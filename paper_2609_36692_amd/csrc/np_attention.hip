// Attention over packed sequences with grouped heads, forward and backward,
// on the bf16 matrix instructions of gfx950 (32x32x16); fp32 operands are split
// into three bf16 terms.
//
// For query i and the keys j of its sequence that it sees (j <= i if causal),
//   s_ij = c q_i . k_j,  p_ij = exp(s_ij - lse_i),  o_i = sum_j p_ij v_j,
//   lse_i = log sum_j exp(s_ij),
//   delta_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - delta_i),
//   dq_i = c sum_j ds_ij k_j,  dk_j = c sum_i ds_ij q_i,  dv_j = sum_i p_ij do_i,
// the last two also over the query heads that share the key's head.
//
// All three passes have one form.  A wave owns 32 rows (queries, or keys in
// the dk/dv pass) as the columns of its matrix products and keeps their
// operands in registers; the other side streams through LDS in tiles that
// all four waves of the block read.  A 32 x 32 block of scores then comes
// out with one owned row per lane (both halves of the wave share it), so a
// softmax row needs one exchange between the halves, and the block is
// already in the layout of the second product's right operand: the k slots
// of a matrix instruction may hold the streamed rows in any order as long as
// both operands agree, and the transposing LDS reads of the left operand
// fetch exactly the rows a lane's score registers hold.
//
// Nothing of the size of a score matrix reaches memory: each pass reads its
// operands once per block of 128 rows and writes its results once.  The dq and
// the dk/dv pass each make the scores anew (seven products instead of five), so
// that every result is summed by one wave in one order, without atomics and
// without an array of partial dq.
//
// Measured (one MI355X, where a library product of 8192^3 reaches 1263 TFLOP/s in
// bf16, 154 in fp32), causal, flops of the visible pairs:
//   16384 tokens, 16/8 heads of 128, bf16: forward 1095-1165 us from card to card,
//     940-1000 TFLOP/s
//   packed 16418 tokens (lengths 3 to 4096), same heads: forward 245 us (860),
//     dq 343 us, dk/dv 480-500 us
//   16 x 1024 tokens, 12 heads of 64, bf16: forward 45 us (570), dq 58, dk/dv 77
//   4 x 1024 tokens, 12 heads of 64, fp32: forward 52-56 us (122), backward 195
// Of the forward pass's cycles at heads of 128 the matrix instructions take 49%,
// the vector instructions 58%, LDS reads 50%: two waves per SIMD overlap them in
// part.  At heads of 64 the vector instructions (an exponential for every pair) take
// 63%, the matrix instructions 28%, mostly one after the other.  fp32 takes six
// products for one, which is still 1.3 to 1.9 times as fast as the fp32 instructions
// (a sixteenth of the bf16 rate), us with those / with bf16 terms: 4 x 1024 tokens, 12
// heads of 64, forward 76 / 53, backward 255 / 194; 2948 tokens, 16/8 heads of 128,
// forward 258 / 216, backward 937 / 728; of 126, forward 526 / 299 (4 x 1024, forward:
// vector instructions 51% of the cycles, matrix 33%).  Error of dk and dv
// over 6000 rows 1.04e-6 / 0.43e-6 of their norm, of out 0.35e-6 / 0.23e-6.
#include "np_train.h"

#include <cmath>
#include <type_traits>

namespace np {
namespace {

typedef __bf16 bf16_t;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kThreads = 256;

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Block barrier that orders LDS only, so prefetches from global memory stay
// in flight across it.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

// One 16-byte chunk of a row of `dim` elements, zero past the row's end.
// VEC: rows are 16-byte aligned and dim is a whole number of chunks.
template <class T, bool VEC>
__device__ __forceinline__ u32x4 load_chunk(const T* row, int chunk, int dim, bool live) {
    constexpr int E = 16 / sizeof(T);
    u32x4 r = {0, 0, 0, 0};
    const int d = chunk * E;
    if constexpr (VEC) {
        if (live && d < dim) r = *reinterpret_cast<const u32x4*>(row + d);
    } else if (live && d + E <= dim) {               // at any element
        typedef u32x4 u32x4_any __attribute__((aligned(2)));
        r = *reinterpret_cast<const u32x4_any*>(row + d);
    } else {
        T e[E];
#pragma unroll
        for (int i = 0; i < E; ++i) e[i] = live && d + i < dim ? row[d + i] : T(0.f);
        __builtin_memcpy(&r, e, 16);
    }
    return r;
}

// ------------------------------------------------------------ LDS tiles ---
// ROWS x DP elements, rows of CH 16-byte chunks; chunk c of row r is kept at
// c ^ swz(r).  Row reads take one chunk of 32 consecutive rows, transposing
// reads 32 bytes of each of four consecutive rows: swz sends any eight
// consecutive rows to eight different chunks and any four to four different
// pairs of chunks, so neither kind meets itself in a bank.
__device__ __forceinline__ int swz(int r) { return ((r & 3) << 1) | ((r >> 2) & 1); }

template <class T, int DP>
struct Tile {
    static constexpr int E = 16 / sizeof(T);     // elements of a chunk
    static constexpr int CH = DP / E;            // chunks of a row
    static __device__ __forceinline__ int idx(int r, int c) { return (r * CH + (c & ~7) + ((c & 7) ^ swz(r))) * E; }
};

// Staging of ROWS x DP from rows [row0, row0 + ROWS) of one operand, rows at
// `rows` and past it zero.
template <class T, int DP, int ROWS, bool VEC, int NT>
struct Stage {
    using TL = Tile<T, DP>;
    static constexpr int N = ROWS * TL::CH / NT;
    static_assert(N >= 1 && ROWS * TL::CH % NT == 0, "tile does not fill the block");
    static __device__ __forceinline__ void load(u32x4 (&r)[N], const T* base, int64_t tok, int row0, int rows,
                                                int dim, int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = tid + i * NT, row = row0 + e / TL::CH;
            r[i] = load_chunk<T, VEC>(base + (int64_t)row * tok, e % TL::CH, dim, row < rows);
        }
    }
    static __device__ __forceinline__ void store(const u32x4 (&r)[N], T* lds, int tid) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = tid + i * NT;
            *reinterpret_cast<u32x4*>(lds + TL::idx(e / TL::CH, e % TL::CH)) = r[i];
        }
    }
};

// fp32 operands as three bf16 terms of eight digits each: the digits are cut off,
// so the terms add up to the operand exactly (from 2^-100 up: matrix instructions
// take smaller terms for zero).  The second term is below 2^-7 of the operand, the
// third below 2^-15.  A product of two takes the six largest of the nine products of
// terms; the three left out add up to 8 2^-24 of it at most and 0.7 2^-24 on average,
// always of its sign.  Terms rounded to nearest would leave out 0.9 2^-24 at most, of
// either sign, but the sums' own rounding is larger (error of out, dq, dk, dv over
// 2948 tokens with terms cut off / rounded: 0.27 0.44 0.45 0.40e-6 / 0.26 0.47 0.48
// 0.43e-6), and it takes 2 to 3% longer (4 x 1024 tokens, 12 heads of 64, forward 62.6 /
// 64.7 us).  What is not finite comes out as NaN, and its rows are made again one by one.
__device__ __forceinline__ void split_pair(float x, float y, uint32_t& t0, uint32_t& t1, uint32_t& t2) {
    auto upper = [](float a, float b) {              // of both, a's below
        return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
    };
    auto rest = [](float a) { return a - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, a) & 0xffff0000u); };
    t0 = upper(x, y);
    x = rest(x);
    y = rest(y);
    t1 = upper(x, y);
    t2 = upper(rest(x), rest(y));
}
__device__ __forceinline__ void split(const f32x4& a, const f32x4& b, u32x4 (&t)[3]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x4& v = i < 2 ? a : b;
        uint32_t t0, t1, t2;
        split_pair(v[2 * (i & 1)], v[2 * (i & 1) + 1], t0, t1, t2);
        t[0][i] = t0;
        t[1][i] = t1;
        t[2][i] = t2;
    }
}

// bf16 numbers that stand for an operand, and the elements of a tile's part of
// one of them.
template <class T> constexpr int kTerms = std::is_same_v<T, bf16_t> ? 1 : 3;
template <int DP> constexpr int kPlane = 32 * DP;    // fp32: tiles of 32 rows

// Staging of 32 x DP fp32 numbers, rows at `rows` and past it zero, to three tiles
// of bf16 terms: loaded while the tile before is worked on.
template <int DP, bool VEC, int NT>
struct Split {
    using TL = Tile<bf16_t, DP>;
    static constexpr int N = 32 * TL::CH / NT;
    static_assert(N >= 1 && 32 * TL::CH % NT == 0, "tile does not fill the block");
    u32x4 r[2 * N];
    __device__ __forceinline__ void load(const float* base, int64_t tok, int row0, int rows, int dim, int tid) {
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) {
            const int e = tid + i / 2 * NT, row = row0 + e / TL::CH;
            r[i] = load_chunk<float, VEC>(base + (int64_t)row * tok, 2 * (e % TL::CH) + i % 2, dim, row < rows);
        }
    }
    __device__ __forceinline__ void store(bf16_t* lds, int tid) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = tid + i * NT;
            u32x4 t[3];
            split(__builtin_bit_cast(f32x4, r[2 * i]), __builtin_bit_cast(f32x4, r[2 * i + 1]), t);
#pragma unroll
            for (int n = 0; n < 3; ++n)
                *reinterpret_cast<u32x4*>(lds + n * kPlane<DP> + TL::idx(e / TL::CH, e % TL::CH)) = t[n];
        }
    }
};

// The same tile straight from memory to LDS, without passing through
// registers.  Rows past the end and chunks past the feature count are copies of
// the last ones there are: they meet zero weights or zero owned features, and
// what is not finite among them is caught with the other rows that are not
// (any_nonfinite): an infinity in a row's last chunk makes NaN of the row's score.
// Zeros in place of the copied chunks cost 1.3% at full heads.  One instruction fills 1 KB of LDS per wave, so the swizzle
// is in the order of the chunks that the lanes fetch.
template <class T, int DP, int ROWS, int NT>
struct Direct {
    using TL = Tile<T, DP>;
    static constexpr int N = ROWS * TL::CH / NT;
    static __device__ __forceinline__ void load(T* lds, const T* base, int64_t tok, int row0, int rows, int dim,
                                                int tid) {
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = tid + i * NT, r = e / TL::CH;
            const int c = min((e % TL::CH) ^ swz(r), dim / TL::E - 1);
            const T* src = base + (int64_t)min(row0 + r, rows - 1) * tok + c * TL::E;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                             (__attribute__((address_space(3))) void*)(lds + (i * NT + wave * 64) * TL::E),
                                             16, 0, 0);
        }
    }
};
// Waits for this wave's loads to LDS.
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }   // vmcnt(0)

// Two streamed operands (K and V, or Q and dO) in two LDS buffers.  Tile `it`
// of a loop is in buffer it % 2.  VEC: each tile is on its way to LDS while the
// one before it is worked on; a wave waits for its own part of it, the barrier
// for the other waves', and behind the barrier the other buffer is free, since
// every wave is done with the tile before.  Otherwise tiles pass through
// registers with no overlap (rows that do not start on 16 bytes).
template <class T, int DP, int ROWS, bool VEC, int NT>
struct Pair {
    const T* p0;
    int64_t tok0;
    const T* p1;
    int64_t tok1;
    int rows, dim;
    __device__ __forceinline__ void fill(T (&buf)[2][ROWS * DP], int row0, int tid) const {
        if constexpr (VEC) {
            Direct<T, DP, ROWS, NT>::load(buf[0], p0, tok0, row0, rows, dim, tid);
            Direct<T, DP, ROWS, NT>::load(buf[1], p1, tok1, row0, rows, dim, tid);
        } else {
            using ST = Stage<T, DP, ROWS, false, NT>;
            u32x4 r[ST::N];
            ST::load(r, p0, tok0, row0, rows, dim, tid);
            ST::store(r, buf[0], tid);
            ST::load(r, p1, tok1, row0, rows, dim, tid);
            ST::store(r, buf[1], tid);
        }
    }
    __device__ __forceinline__ void first(T (&smem)[2][2][ROWS * DP], int row0, int tid) const {
        if constexpr (VEC) fill(smem[0], row0, tid);
    }
    // Tile `it` is ready behind this call; row0: its first row, then: that of
    // the tile after it, or -1.
    __device__ __forceinline__ void next(T (&smem)[2][2][ROWS * DP], int it, int row0, int then, int tid) const {
        if constexpr (VEC) {
            wait_loads();
            lds_barrier();
            if (then >= 0) fill(smem[(it + 1) & 1], then, tid);
        } else {
            fill(smem[it & 1], row0, tid);
            lds_barrier();
        }
    }
};

// fp32: through registers, in which a tile waits while the one before it is worked
// on; one buffer or two.
template <int DP, bool VEC, int NT, int BUFS>
struct SplitPair {
    const float* p0;
    int64_t tok0;
    const float* p1;
    int64_t tok1;
    int rows, dim;
    Split<DP, VEC, NT> r0, r1;
    __device__ __forceinline__ void fetch(int row0, int tid) {
        r0.load(p0, tok0, row0, rows, dim, tid);
        r1.load(p1, tok1, row0, rows, dim, tid);
    }
    template <class S> __device__ __forceinline__ void first(S&, int row0, int tid) { fetch(row0, tid); }
    template <class S> __device__ __forceinline__ void next(S& smem, int it, int, int then, int tid) {
        if constexpr (BUFS == 1) lds_barrier();
        r0.store(smem[it % BUFS][0], tid);
        r1.store(smem[it % BUFS][1], tid);
        lds_barrier();
        if (then >= 0) fetch(then, tid);
    }
};
template <class T, int DP, int ROWS, bool VEC, int NT, int BUFS>
using Streamed = std::conditional_t<std::is_same_v<T, bf16_t>, Pair<bf16_t, DP, ROWS, VEC, NT>, SplitPair<DP, VEC, NT, BUFS>>;

// Owned operand of one wave: chunk 2 s + half of row lane % 32, for every s.
template <class T, int DP>
struct Owned {
    static constexpr int S = Tile<bf16_t, DP>::CH / 2;
    u32x4 c[S][kTerms<T>];
    template <bool VEC>
    __device__ __forceinline__ void load(const T* row, int dim, bool live, int half) {
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if constexpr (kTerms<T> == 1) c[s][0] = load_chunk<T, VEC>(row, 2 * s + half, dim, live);
            else split(__builtin_bit_cast(f32x4, load_chunk<T, VEC>(row, 4 * s + 2 * half, dim, live)),
                       __builtin_bit_cast(f32x4, load_chunk<T, VEC>(row, 4 * s + 2 * half + 1, dim, live)), c[s]);
        }
    }
    // From a tile in LDS, rows [base, base + 32).
    __device__ __forceinline__ void load(const T* lds, int base, int lane) {
        using TL = Tile<T, DP>;
#pragma unroll
        for (int s = 0; s < S; ++s)
            c[s][0] = *reinterpret_cast<const u32x4*>(lds + TL::idx(base + (lane & 31), 2 * s + (lane >> 5)));
    }
    __device__ __forceinline__ void negate() {
#pragma unroll
        for (int s = 0; s < S; ++s)
#pragma unroll
            for (int t = 0; t < kTerms<T>; ++t) c[s][t] ^= 0x80008000u;
    }
};

// N blocks of 32 x 32 scores: streamed rows [base[n], base[n] + 32) of a tile
// against the wave's owned rows.  Lane l gets owned row l % 32, register r
// streamed row base + 8 (r / 4) + 4 (l / 32) + r % 4.  The blocks take turns, so
// that no product waits for the one before it.
template <class T, int DP, int N>
__device__ __forceinline__ void scores(f32x16 (&acc)[N], const bf16_t* const (&lds)[N], const int (&base)[N],
                                       const Owned<T, DP>* const (&own)[N], int lane) {
    using TL = Tile<bf16_t, DP>;
    const int half = lane >> 5;
#pragma unroll
    for (int n = 0; n < N; ++n) acc[n] = f32x16{};
#pragma unroll
    for (int s = 0; s < Owned<T, DP>::S; ++s) {
        auto read = [&](int n, int t) {
            return *reinterpret_cast<const bf16x8*>(lds[n] + t * kPlane<DP> + TL::idx(base[n] + (lane & 31), 2 * s + half));
        };
        auto owned = [&](int n, int t) { return __builtin_bit_cast(bf16x8, own[n]->c[s][t]); };
        if constexpr (kTerms<T> == 1) {
#pragma unroll
            for (int n = 0; n < N; ++n)
                acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read(n, 0), owned(n, 0), acc[n], 0, 0, 0);
        } else {
            bf16x8 x[N][3];
#pragma unroll
            for (int n = 0; n < N; ++n)
#pragma unroll
                for (int t = 0; t < 3; ++t) x[n][t] = read(n, t);
            // The smallest products first.
#pragma unroll
            for (int t = 2; t >= 0; --t)
#pragma unroll
                for (int i = 0; i <= t; ++i)
#pragma unroll
                    for (int n = 0; n < N; ++n)
                        acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[n][i], owned(n, t - i), acc[n], 0, 0, 0);
        }
    }
}

template <class T, int DP>
__device__ __forceinline__ f32x16 scores(const bf16_t* lds, int base, const Owned<T, DP>& own, int lane) {
    f32x16 acc[1];
    const bf16_t* const l[1] = {lds};
    const int b[1] = {base};
    const Owned<T, DP>* const o[1] = {&own};
    scores<T, DP, 1>(acc, l, b, o, lane);
    return acc[0];
}

// Streamed rows r0 .. r0 + 3 and r0 + 8 .. r0 + 11 of the group's lanes (r0 is
// that of lane p / 4) at the lane's column of features 32 t ..: within each 16-lane
// group the transposing read returns to lane j the j-th column of the 4 x 16
// block the group addresses (lane p supplies row p / 4, elements 4 (p % 4) ..).
template <int DP>
__device__ __forceinline__ bf16x8 columns(const bf16_t* lds, int r0, int t, int g, int p) {
    using TL = Tile<bf16_t, DP>;
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    const int r1 = r0 + 8, c = 4 * t + 2 * (g & 1) + ((p & 3) >> 1), in = 4 * (p & 1);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + TL::idx(r0, c) + in));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lds + TL::idx(r1, c) + in));
    const s16x8 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, a);
}

// acc[t] (features 32 t .. of the result, by owned row) += tile^T weights,
// over streamed rows [base, base + 32); w in the layout of scores().  The
// weights of bf16 operands are rounded to bf16, as matrix instructions take
// them: relative error up to 2^-8 each, as that of the bf16 result, but of random
// sign along a sum.  fp32
// tiles are summed apart and then added, so that a long sum rounds once a tile at
// its full size: half the error of dk and dv over 6000 rows for 1% of the time.
template <class T, int DP>
__device__ __forceinline__ void accumulate(f32x16 (&acc)[DP / 32], const bf16_t* lds, int base, const f32x16& w,
                                           int lane) {
    const int g = lane >> 4, p = lane & 15;          // group of 16 lanes, lane of it
    if constexpr (std::is_same_v<T, bf16_t>) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            bf16x8 b;
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = (bf16_t)w[8 * s + i];
            const int r0 = base + 16 * s + 4 * (g >> 1) + (p >> 2);
#pragma unroll
            for (int t = 0; t < DP / 32; ++t)
                acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(columns<DP>(lds, r0, t, g, p), b, acc[t], 0, 0, 0);
        }
    } else {
        u32x4 b[2][3];
#pragma unroll
        for (int s = 0; s < 2; ++s)
            split(f32x4{w[8 * s], w[8 * s + 1], w[8 * s + 2], w[8 * s + 3]},
                  f32x4{w[8 * s + 4], w[8 * s + 5], w[8 * s + 6], w[8 * s + 7]}, b[s]);
#pragma unroll
        for (int t = 0; t < DP / 32; ++t) {
            f32x16 sum = {};
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int r0 = base + 16 * s + 4 * (g >> 1) + (p >> 2);
                bf16x8 x[3];
#pragma unroll
                for (int i = 0; i < 3; ++i) x[i] = columns<DP>(lds + i * kPlane<DP>, r0, t, g, p);
#pragma unroll
                for (int n = 2; n >= 0; --n)
#pragma unroll
                    for (int i = 0; i <= n; ++i)
                        sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[i], __builtin_bit_cast(bf16x8, b[s][n - i]), sum, 0, 0, 0);
            }
            acc[t] += sum;
        }
    }
}

// Writes f * acc of the wave's owned rows, `keep` (bit r: row r) of them, to
// rows of `stride` elements from `out`.  The rows pass through the wave's share
// of the LDS tiles (32 x DP words, which every wave must be done with), so that
// memory gets whole rows instead of 8 or 16 bytes of 32 rows at a time.
template <class T, int DP, bool VEC>
__device__ __forceinline__ void store_rows(void* lds, T* out, int64_t stride, const f32x16 (&acc)[DP / 32], float f,
                                           int dim, uint32_t keep, int lane) {
    constexpr int E = 16 / sizeof(T), CH = DP / E, M = (CH < 16 ? CH : 16) - 1;
    T* mine = static_cast<T*>(lds);
    const int row = lane & 31, half = lane >> 5;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int d = 32 * t + 8 * j + 4 * half;
            T e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = (T)(f * acc[t][4 * j + i]);
            typedef uint32_t V __attribute__((ext_vector_type(sizeof(T))));
            V v;
            __builtin_memcpy(&v, e, sizeof v);
            *reinterpret_cast<V*>(mine + (row * CH + ((d / E) ^ (row & M))) * E + d % E) = v;
        }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 32 * CH / 64; ++i) {
        const int r = (i * 64 + lane) / CH, c = lane % CH;
        if (!(keep >> r & 1)) continue;
        const u32x4 v = *reinterpret_cast<const u32x4*>(mine + (r * CH + (c ^ (r & M))) * E);
        T* dst = out + r * stride + c * E;
        if constexpr (VEC) {
            if (c * E < dim) *reinterpret_cast<u32x4*>(dst) = v;
        } else {
            T e[E];
            __builtin_memcpy(e, &v, 16);
#pragma unroll
            for (int k = 0; k < E; ++k)
                if (c * E + k < dim) dst[k] = e[k];
        }
    }
    __builtin_amdgcn_wave_barrier();
}

// A wave's accumulators through its share of the LDS tiles to the wave of the
// other team that owns the same rows, which adds them: acc f0 + other f1.
template <int DP>
__device__ __forceinline__ void hand_over(bf16_t* lds, const f32x16 (&acc)[DP / 32], int lane) {
    f32x4* p = reinterpret_cast<f32x4*>(lds) + lane;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            p[(4 * t + j) * 64] = f32x4{acc[t][4 * j], acc[t][4 * j + 1], acc[t][4 * j + 2], acc[t][4 * j + 3]};
}
template <int DP>
__device__ __forceinline__ void take_over(const bf16_t* lds, f32x16 (&acc)[DP / 32], float f0, float f1, int lane) {
    const f32x4* p = reinterpret_cast<const f32x4*>(lds) + lane;
#pragma unroll
    for (int t = 0; t < DP / 32; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x4 v = p[(4 * t + j) * 64];
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][4 * j + i] = acc[t][4 * j + i] * f0 + v[i] * f1;
        }
}

// Bits of the wave's rows [row0, row0 + 32) that lie before `rows`.
__device__ __forceinline__ uint32_t live_rows(int row0, int rows) {
    return row0 >= rows ? 0u : rows - row0 >= 32 ? ~0u : (1u << (rows - row0)) - 1;
}

template <int NT>
__device__ __forceinline__ bool any_nonfinite(const f32x16 (&acc)[NT]) {
    float t = 0.f;                               // x * 0 is NaN for what is not finite
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) t = __builtin_fmaf(acc[i][r], 0.f, t);
    return !(t == 0.f);
}

// ----------------------------------------------------- rows one by one ---
// A matrix product multiplies the zero weight of a masked place with the
// value there, and 0 * inf is NaN: where a tile on the diagonal holds values
// that are not finite, rows that must not see them come out as NaN.  Rows of
// the tiled passes that are not finite, unless that is their answer (odd_rows),
// are therefore done again here, by one wave each, over the places that they see
// and no others: lanes first along the other side (64 scores at a time), then along
// the features, up to the point where every feature is NaN.  The forward pass also
// sums o before it divides by l, with weights of up to 2^8, so values above 2^120 / l
// may pass fp32's range on the way; here o is a mean at every step.
template <class T, int N>
__device__ __forceinline__ void dot_step(float& s, const T* a, const T* b) {      // N pieces of 16 bytes, at any element
    constexpr int E = 16 / sizeof(T);
    typedef u32x4 u32x4_any __attribute__((aligned(2)));
    u32x4 x[N], y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        x[i] = *reinterpret_cast<const u32x4_any*>(a + i * E);
        y[i] = *reinterpret_cast<const u32x4_any*>(b + i * E);
    }
    T u[N * E], v[N * E];
    __builtin_memcpy(u, x, 16 * N);
    __builtin_memcpy(v, y, 16 * N);
#pragma unroll
    for (int i = 0; i < N * E; ++i) s = __builtin_fmaf((float)u[i], (float)v[i], s);
}
template <class T>
__device__ __forceinline__ float dot(const T* a, const T* b, int dim) {
    constexpr int E = 16 / sizeof(T);
    float s = 0.f;
    int d = 0;
    for (; d + 4 * E <= dim; d += 4 * E) dot_step<T, 4>(s, a + d, b + d);
    for (; d + E <= dim; d += E) dot_step<T, 1>(s, a + d, b + d);
    for (; d < dim; ++d) s = __builtin_fmaf((float)a[d], (float)b[d], s);
    return s;
}

struct Where {                                   // one sequence, one head
    int start, len, head, kv;
};

template <class T>
__device__ __forceinline__ T* row_of(const AttnOperand& o, const Where& w, int row, int head) {
    return static_cast<T*>(o.p) + (int64_t)(w.start + row) * o.tok + (int64_t)head * o.head;
}

// acc += sum_j w_j row_j over rows r0 .. r0 + n - 1 of o; w_j: lane j's w; acc[x]: feature
// lane + 64 x (past the last one: not used).  Eight rows are loaded at a time.
template <class T>
__device__ __forceinline__ void add_rows(float (&acc)[2], float w, const AttnOperand& o, const Where& at, int head,
                                         int r0, int n, int dim, int lane) {
    for (int j0 = 0; j0 < n; j0 += 8) {
        float v[8][2];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const T* row = row_of<T>(o, at, r0 + min(j0 + u, n - 1), head);
#pragma unroll
            for (int x = 0; x < 2; ++x) v[u][x] = (float)row[min(lane + 64 * x, dim - 1)];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const float f = __shfl(w, j0 + u, 64);
#pragma unroll
            for (int x = 0; x < 2; ++x) acc[x] = j0 + u < n ? __builtin_fmaf(f, v[u][x], acc[x]) : acc[x];
        }
    }
}

__device__ __forceinline__ bool all_nan(const float (&g)[2], int lane, int dim) {
    return __all((lane >= dim || g[0] != g[0]) && (lane + 64 >= dim || g[1] != g[1]));
}

template <class T>
__device__ void forward_row(const AttnArgs& a, const Where& w, int qi, bool has_lse, int lane) {
    const T* q = row_of<T>(a.q, w, qi, w.head);
    const int end = a.causal ? qi + 1 : w.len;
    const float c2 = a.scale * kLog2e;
    float m = -INFINITY, l = 0.f, o[2] = {0.f, 0.f};
    for (int k0 = 0; k0 < end; k0 += 64) {
        const int n = min(64, end - k0);
        const float t = lane < n ? dot(q, row_of<T>(a.k, w, k0 + lane, w.kv), a.dim) * c2 : -INFINITY;
        const float mn = fmaxf(m, wave_max(t)), mu = mn == -INFINITY ? 0.f : mn;
        const float p = exp2_fast(t - mu), f = exp2_fast(m - mu);
        const float before = l * f;
        l = before + wave_sum(p);
        m = mn;
        if (l != l) break;                           // so is every feature
        const float r = l > 0.f ? 1.f / l : 0.f;
        o[0] *= before * r;
        o[1] *= before * r;
        add_rows<T>(o, p * r, a.v, w, w.kv, k0, n, a.dim, lane);
        if (has_lse && all_nan(o, lane, a.dim)) break;
    }
    T* out = row_of<T>(a.out, w, qi, w.head);
#pragma unroll
    for (int x = 0; x < 2; ++x)
        if (lane + 64 * x < a.dim) out[lane + 64 * x] = (T)(l > 0.f ? o[x] : NAN);
    if (lane == 0 && !has_lse) a.lse[w.head * a.tokens + w.start + qi] = m * kLn2 + logf(l);
}

// sum_j p dp of one row.
template <class T>
__device__ float delta_row(const AttnArgs& a, const Where& w, int qi, int lane) {
    const T *q = row_of<T>(a.q, w, qi, w.head), *dout = row_of<T>(a.dout, w, qi, w.head);
    const int end = a.causal ? qi + 1 : w.len;
    const float c2 = a.scale * kLog2e, lse2 = a.lse[w.head * a.tokens + w.start + qi] * kLog2e;
    float sum = 0.f;
    for (int j = lane; j < end; j += 64)
        sum += exp2_fast(dot(q, row_of<T>(a.k, w, j, w.kv), a.dim) * c2 - lse2) * dot(dout, row_of<T>(a.v, w, j, w.kv), a.dim);
    return wave_sum(sum);
}

template <class T>
__device__ void dq_row(const AttnArgs& a, const Where& w, int qi, float delta, int lane) {
    const T *q = row_of<T>(a.q, w, qi, w.head), *dout = row_of<T>(a.dout, w, qi, w.head);
    const int end = a.causal ? qi + 1 : w.len;
    const float c2 = a.scale * kLog2e, lse2 = a.lse[w.head * a.tokens + w.start + qi] * kLog2e;
    float g[2] = {0.f, 0.f};
    for (int k0 = 0; k0 < end; k0 += 64) {
        const int n = min(64, end - k0);
        float ds = 0.f;
        if (lane < n) {
            const float p = exp2_fast(dot(q, row_of<T>(a.k, w, k0 + lane, w.kv), a.dim) * c2 - lse2);
            ds = p * (dot(dout, row_of<T>(a.v, w, k0 + lane, w.kv), a.dim) - delta);
        }
        add_rows<T>(g, ds, a.k, w, w.kv, k0, n, a.dim, lane);
        if (all_nan(g, lane, a.dim)) break;
    }
    T* dq = row_of<T>(a.dq, w, qi, w.head);
#pragma unroll
    for (int x = 0; x < 2; ++x)
        if (lane + 64 * x < a.dim) dq[lane + 64 * x] = (T)(a.scale * g[x]);
}

template <class T>
__device__ void dkv_row(const AttnArgs& a, const Where& w, int ki, int lane) {
    const T *k = row_of<T>(a.k, w, ki, w.kv), *v = row_of<T>(a.v, w, ki, w.kv);
    const int beg = a.causal ? ki : 0, group = a.heads / a.kv_heads;
    const float c2 = a.scale * kLog2e;
    float gk[2] = {0.f, 0.f}, gv[2] = {0.f, 0.f};
    bool lost = false;
    for (int h = w.kv * group; h < (w.kv + 1) * group && !lost; ++h)
        for (int q0 = beg; q0 < w.len && !lost; q0 += 64) {
            const int n = min(64, w.len - q0);
            float p = 0.f, ds = 0.f;
            if (lane < n) {
                const int64_t at = h * a.tokens + w.start + q0 + lane;
                p = exp2_fast(dot(row_of<T>(a.q, w, q0 + lane, h), k, a.dim) * c2 - a.lse[at] * kLog2e);
                ds = p * (dot(row_of<T>(a.dout, w, q0 + lane, h), v, a.dim) - a.delta[at]);
            }
            add_rows<T>(gk, ds, a.q, w, h, q0, n, a.dim, lane);
            add_rows<T>(gv, p, a.dout, w, h, q0, n, a.dim, lane);
            lost = all_nan(gk, lane, a.dim) && all_nan(gv, lane, a.dim);
        }
    T *dk = row_of<T>(a.dk, w, ki, w.kv), *dv = row_of<T>(a.dv, w, ki, w.kv);
#pragma unroll
    for (int x = 0; x < 2; ++x)
        if (lane + 64 * x < a.dim) {
            dk[lane + 64 * x] = (T)(a.scale * gk[x]);
            dv[lane + 64 * x] = (T)gv[x];
        }
}

// Owned rows (bit r: row r of the wave's 32) that any lane calls bad.  Not to be asked
// with x < INFINITY alone: the compiler's ballot makes x != INFINITY of that, which
// holds for NaN.
__device__ __forceinline__ uint32_t bad_rows(bool bad) {
    const uint64_t b = __ballot(bad);
    return (uint32_t)b | (uint32_t)(b >> 32);
}

// Most rows that are not finite are right as the tiled passes made them: what they
// see is not finite either, and a NaN early in a long sequence would otherwise send
// every later row here (one NaN in k or v, 4096 tokens, 4 heads of 64: forward 32 ms,
// backward 58, where the tiled passes take 0.07 and 0.13).  What a wave made is wrong
// only
//   - where a place that a row does not see held a value that is not finite: those
//     places lie in the 32 to 64 rows of the tile on the diagonal, and behind the
//     sequence's end, where its last row stands again;
//   - where terms and copies made NaN of an infinity: fp32, and heads that leave a
//     part of the tile to copies (Direct), if an operand holds one;
//   - (forward) where finite values passed the range.
// So the operands' rows are searched, by a wave that has such rows: 16 lanes a row.
struct Odd {
    bool inf, any;                               // an infinity, any value not finite
    int first, last;                             // row
};
template <class T>
__device__ Odd odd_rows(const AttnOperand& o, const Where& w, int head, int from, int to, int dim, int lane) {
    bool inf = false, any = false;
    int first = INT32_MAX, last = -1;
    for (int r = from + (lane >> 4); r < to; r += 4) {
        const T* x = row_of<T>(o, w, r, head);
        bool i = false, n = false;
        for (int d = lane & 15; d < dim; d += 16) {
            const float v = (float)x[d];
            i |= __builtin_fabsf(v) == INFINITY;
            n |= !(__builtin_fabsf(v) < INFINITY);
        }
        inf |= i;
        any |= n;
        if (n) {
            first = min(first, r);
            last = r;
        }
    }
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) {
        first = min(first, __shfl_xor(first, s, 64));
        last = max(last, __shfl_xor(last, s, 64));
    }
    return {(bool)__any(inf), (bool)__any(any), first, last};
}
// Whether what the tiled passes make of visible values is the formula's.
template <class T, int DP, bool VEC>
__device__ __forceinline__ bool faithful(const AttnArgs& a) { return kTerms<T> == 1 && (!VEC || a.dim == DP); }

// The query passes: the highest of the wave's rows, from row qw on, that x (v, or
// k) spoils although it does not see the place, or INT_MAX: all of them.  Rows before
// `done` were multiplied.
template <class T>
__device__ int spoiled_queries(const AttnArgs& a, const Where& w, const AttnOperand& x, int qw, int done, int lane) {
    const Odd o = odd_rows<T>(x, w, w.kv, a.causal ? qw : w.len - 1, min(done, w.len), a.dim, lane);
    return a.causal ? o.last : done > w.len && o.inf ? INT32_MAX : -1;
}

// dk and dv: the keys above the one that this returns, of 32 from row kw on, are spoiled
// by queries that do not see them; INT_MAX: none, -1: all.
template <class T>
__device__ int spoiled_keys(const AttnArgs& a, const Where& w, int kw, bool right, int lane) {
    const int group = a.heads / a.kv_heads;
    // A query that every key of the wave sees and that has no log-sum-exp: all NaN.
    const int sure = a.causal ? min(kw + 31, w.len - 1) : 0;
    bool lost = false;
    for (int h = w.kv * group; h < (w.kv + 1) * group; ++h)
        for (int i = sure + lane; i < w.len; i += 64) {
            const float l = a.lse[h * a.tokens + w.start + i];
            lost |= l != l;
        }
    if (__any(lost)) return INT32_MAX;
    if (!right) {
        bool inf = odd_rows<T>(a.k, w, w.kv, kw, min(kw + 32, w.len), a.dim, lane).inf ||
                   odd_rows<T>(a.v, w, w.kv, kw, min(kw + 32, w.len), a.dim, lane).inf;
        for (int h = w.kv * group; h < (w.kv + 1) * group && !inf; ++h)
            inf = odd_rows<T>(a.q, w, h, a.causal ? kw : 0, w.len, a.dim, lane).inf ||
                  odd_rows<T>(a.dout, w, h, a.causal ? kw : 0, w.len, a.dim, lane).inf;
        if (inf) return -1;
    }
    const bool copies = w.len % 32 != 0;
    int low = INT32_MAX;
    for (int h = w.kv * group; h < (w.kv + 1) * group; ++h)
        for (int x = 0; x < 2; ++x) {
            const AttnOperand& o = x ? a.dout : a.q;
            if (a.causal) low = min(low, odd_rows<T>(o, w, h, kw, min(kw + 32, w.len), a.dim, lane).first);
            if (copies && odd_rows<T>(o, w, h, w.len - 1, w.len, a.dim, lane).inf) return -1;
        }
    return low;
}

// ---------------------------------------------------------------- passes ---
// Rows of a streamed tile (fp32: three terms of it).
template <class T> constexpr int kStream = std::is_same_v<T, bf16_t> ? 64 : 32;
// Rows of each team's tiles in the query passes: half where the tiles of all
// teams would not fit in LDS.
template <class T, int DP, int TEAMS>
constexpr int kStreamed = TEAMS * kStream<T> * DP * 4 * 2 <= 140 * 1024 || kTerms<T> == 3 ? kStream<T> : kStream<T> / 2;
// Buffers for tiles (one where two would leave a CU one block), and the bf16 numbers
// of one tile in the query passes' LDS; the rows of the result pass through the same
// LDS in the end.
template <class T, int DP, int TEAMS> constexpr int kBufs = kTerms<T> == 1 || (TEAMS == 1 && DP == 64) ? 2 : 1;
template <class T, int DP, int WR, int TEAMS>
constexpr int tile_elements() {
    const int tile = kStreamed<T, DP, TEAMS> * DP * kTerms<T>, rows = 32 * DP * WR / kBufs<T, DP, TEAMS>;
    return kTerms<T> == 1 || tile > rows ? tile : rows;
}

// Waves per SIMD a kernel is compiled for: two (256 registers), so that one
// wave's matrix instructions run beside the other's exponentials, unless the
// owned operands and accumulators (`ops` and `accs` per owned row and feature)
// leave no room for them.
template <class T, int DP>
constexpr int waves(int ops, int accs) { return DP * (ops * kTerms<T> / 2.f + accs) / 2 <= 160 ? 2 : 1; }
// The same for the query passes, where LDS may hold only one block of four waves.
template <class T, int DP, int WR, int TEAMS>
constexpr int query_waves(int ops) {
    return WR * TEAMS == 4 && TEAMS * kBufs<T, DP, TEAMS> * 4 * tile_elements<T, DP, WR, TEAMS>() > 80 * 1024 ? 1 : waves<T, DP>(ops, 1);
}

// Block order: key heads fastest, so the blocks of one key head (consecutive
// workgroups go to the 8 XCDs in turn) stay with one XCD's L2 where the
// number of key heads is a multiple of 8; the plan's tiles, longest first,
// slowest.
__device__ __forceinline__ bool locate(const AttnArgs& a, const AttnTile& t, int within, int& row0) {
    return tile_row(t, a.tokens, within, row0);
}

// Forward: blocks of 32 WR queries of one head, TEAMS of waves that take the key
// tiles in turn and add up their (o, m, l) at the end.  One pass over the keys
// with the running maximum and sum of the softmax.
template <class T, int DP, bool VEC, int WR, int TEAMS>
__global__ void __launch_bounds__(64 * WR * TEAMS, (query_waves<T, DP, WR, TEAMS>(1))) attn_fwd_kernel(AttnArgs a) {
    constexpr int NT = 64 * WR, BN = kStreamed<T, DP, TEAMS>, NB = BN / 32, DT = DP / 32;
    constexpr int BUFS = kBufs<T, DP, TEAMS>, TE = tile_elements<T, DP, WR, TEAMS>(), SHARE = BUFS * 2 * TE / WR;
    __shared__ __attribute__((aligned(16))) bf16_t tiles[TEAMS][BUFS][2][TE];
    __shared__ float stat[TEAMS][2][32 * WR];
    const int tid = threadIdx.x % NT, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int team = TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
    const int group = a.heads / a.kv_heads;
    const AttnTile tile = a.tiles[blockIdx.x / a.heads];
    const int kv = blockIdx.x % a.kv_heads, head = kv * group + (blockIdx.x / a.kv_heads) % group;
    int q0;
    if (!locate(a, tile, blockIdx.y * 32 * WR, q0)) return;    // the whole block
    const Where w{tile.start, tile.len, head, kv};
    const int qw = q0 + wave * 32, qi = qw + (lane & 31);
    const bool live = qi < w.len;
    auto& smem = tiles[team];

    Owned<T, DP> q;
    q.template load<VEC>(row_of<T>(a.q, w, live ? qi : 0, head), a.dim, live, half);
    if (a.scale < 0.f) q.negate();                   // so that larger products are larger scores
    const T *kb = row_of<T>(a.k, w, 0, kv), *vb = row_of<T>(a.v, w, 0, kv);
    const int end = a.causal ? min(w.len, q0 + 32 * WR) : w.len, steps = (end + BN - 1) / BN;
    const float c2 = fabsf(a.scale) * kLog2e;

    // m: the largest product so far, or one that was when it was last raised; o
    // and l are raised to it only once a score is 2^8 above it, so that most
    // tiles leave o alone (weights then stay below 2^8, which costs no digit).
    f32x16 o[DT] = {};
    float m = -INFINITY, l = 0.f;
    Streamed<T, DP, BN, VEC, NT, BUFS> keys{kb, a.k.tok, vb, a.v.tok, w.len, a.dim};
    keys.first(smem, team * BN, tid);
    for (int it = 0; it < (steps + TEAMS - 1) / TEAMS; ++it) {
        const int k0 = (it * TEAMS + team) * BN;
        keys.next(smem, it, k0, it * TEAMS + team + TEAMS < steps ? k0 + TEAMS * BN : -1, tid);
        const bf16_t *ks = smem[it % BUFS][0], *vs = smem[it % BUFS][1];
        if (k0 < end && (!a.causal || k0 <= qw + 31)) {    // same for the whole wave
            f32x16 s[NB];
            float mx = m;
            const bool edge = k0 + BN > w.len || (a.causal && k0 + BN - 1 > qw);
            const int last = (a.causal ? min(qi, w.len - 1) : w.len - 1) - k0 - 4 * half;
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b] = scores<T, DP>(ks, 32 * b, q, lane);
            if (edge) {
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (32 * b + 8 * (r / 4) + r % 4 > last) s[b][r] = -INFINITY;
            }
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            if (__any((mx - m) * c2 > 8.f || (m == -INFINITY && mx != -INFINITY))) {
                const float f = m == -INFINITY ? 0.f : exp2_fast((m - mx) * c2);
                m = mx;
                l *= f;
#pragma unroll
                for (int t = 0; t < DT; ++t) o[t] *= f;
            }
            const float mu = m == -INFINITY ? 0.f : m * c2;
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[b][r] = exp2_fast(__builtin_fmaf(s[b][r], c2, -mu));
            if (edge) {                              // also where c is 0
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (32 * b + 8 * (r / 4) + r % 4 > last) s[b][r] = 0.f;
            }
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) l += s[b][r];
#pragma unroll
            for (int b = 0; b < NB; ++b) accumulate<T, DP>(o, vs, 32 * b, s[b], lane);
        }
    }
    l += __shfl_xor(l, 32, 64);
    lds_barrier();                                   // the tiles are free
    bf16_t* mine = &smem[0][0][0] + wave * SHARE;
    if constexpr (TEAMS > 1) {
        if (team > 0) hand_over<DP>(mine, o, lane);
        if (half == 0) {
            stat[team][0][wave * 32 + lane] = m;
            stat[team][1][wave * 32 + lane] = l;
        }
        lds_barrier();
        if (team > 0) return;
        const int row = wave * 32 + (lane & 31);
        float mx = m;
#pragma unroll
        for (int t = 1; t < TEAMS; ++t) mx = fmaxf(mx, stat[t][0][row]);
        float f = m == -INFINITY ? 0.f : exp2_fast((m - mx) * c2);
        l *= f;
#pragma unroll
        for (int t = 1; t < TEAMS; ++t) {
            const float mt = stat[t][0][row], ft = mt == -INFINITY ? 0.f : exp2_fast((mt - mx) * c2);
            take_over<DP>(&tiles[t][0][0][0] + wave * SHARE, o, f, ft, lane);
            l += stat[t][1][row] * ft;
            f = 1.f;
        }
        m = mx;
    }
    uint32_t bad = bad_rows(live && (any_nonfinite(o) || !(l < INFINITY)));
    const uint32_t lost = bad_rows(l != l);          // all NaN, of a visible score
    if (bad) {
        const int sees = a.causal ? qw + 1 : w.len;  // keys that every row of the wave sees
        bool right = faithful<T, DP, VEC>(a);
        if (!right)
            right = !odd_rows<T>(a.q, w, head, qw, min(qw + 32, w.len), a.dim, lane).inf &&
                    !odd_rows<T>(a.k, w, kv, 0, end, a.dim, lane).inf && !odd_rows<T>(a.v, w, kv, 0, end, a.dim, lane).inf;
        if (right) {
            bad &= ~lost;
            if (bad) {
                const int top = odd_rows<T>(a.v, w, kv, 0, sees, a.dim, lane).any
                              ? spoiled_queries<T>(a, w, a.v, qw, ((a.causal ? min(end, qw + 32) : end) + BN - 1) / BN * BN, lane) : INT32_MAX;
                bad &= bad_rows(qi <= top);
            }
        }
    }
    store_rows<T, DP, VEC>(mine, row_of<T>(a.out, w, qw, head), a.out.tok, o, 1.f / l,
                           a.dim, live_rows(qw, w.len) & ~bad, lane);
    // A sum that is not NaN stands: every place it takes in is seen.
    if (live && half == 0 && !(bad & lost & 1u << lane))
        a.lse[head * a.tokens + w.start + qi] = m * fabsf(a.scale) + logf(l);
    for (; bad; bad &= bad - 1)
        forward_row<T>(a, w, qw + __builtin_ctz(bad), !(lost >> __builtin_ctz(bad) & 1), lane);
}

// dq, and delta and the base-2 log-sum-exp for the dk/dv pass: the forward pass's
// blocks, with q and dO owned; three products a tile, K read both ways.
template <class T, int DP, bool VEC, int WR, int TEAMS>
__global__ void __launch_bounds__(64 * WR * TEAMS, (query_waves<T, DP, WR, TEAMS>(2))) attn_dq_kernel(AttnArgs a) {
    constexpr int NT = 64 * WR, BN = kStreamed<T, DP, TEAMS>, NB = BN / 32, DT = DP / 32;
    constexpr int BUFS = kBufs<T, DP, TEAMS>, TE = tile_elements<T, DP, WR, TEAMS>(), SHARE = BUFS * 2 * TE / WR;
    __shared__ __attribute__((aligned(16))) bf16_t tiles[TEAMS][BUFS][2][TE];
    __shared__ float stat[TEAMS][32 * WR];
    const int tid = threadIdx.x % NT, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int team = TEAMS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
    const int group = a.heads / a.kv_heads;
    const AttnTile tile = a.tiles[blockIdx.x / a.heads];
    const int kv = blockIdx.x % a.kv_heads, head = kv * group + (blockIdx.x / a.kv_heads) % group;
    int q0;
    if (!locate(a, tile, blockIdx.y * 32 * WR, q0)) return;    // the whole block
    const Where w{tile.start, tile.len, head, kv};
    const int qw = q0 + wave * 32, qi = qw + (lane & 31);
    const bool live = qi < w.len;
    auto& smem = tiles[team];

    Owned<T, DP> q, dout;
    q.template load<VEC>(row_of<T>(a.q, w, live ? qi : 0, head), a.dim, live, half);
    dout.template load<VEC>(row_of<T>(a.dout, w, live ? qi : 0, head), a.dim, live, half);
    // delta of the lane's row: its half of the chunks, then the other half's.
    float delta = 0.f;
    {
        const T *orow = row_of<T>(a.out, w, live ? qi : 0, head), *drow = row_of<T>(a.dout, w, live ? qi : 0, head);
#pragma unroll
        for (int s = 0; s < Tile<T, DP>::CH / 2; ++s) {
            const u32x4 oc = load_chunk<T, VEC>(orow, 2 * s + half, a.dim, live);
            u32x4 dc;
            if constexpr (kTerms<T> == 1) dc = dout.c[s][0];
            else dc = load_chunk<T, VEC>(drow, 2 * s + half, a.dim, live);
            T x[16 / sizeof(T)], y[16 / sizeof(T)];
            __builtin_memcpy(x, &oc, 16);
            __builtin_memcpy(y, &dc, 16);
#pragma unroll
            for (int i = 0; i < (int)(16 / sizeof(T)); ++i) delta = __builtin_fmaf((float)x[i], (float)y[i], delta);
        }
        delta += __shfl_xor(delta, 32, 64);
    }
    const int64_t at = head * a.tokens + w.start + (live ? qi : 0);
    const float lse2 = live ? a.lse[at] * kLog2e : INFINITY;
    const T *kb = row_of<T>(a.k, w, 0, kv), *vb = row_of<T>(a.v, w, 0, kv);
    const int end = a.causal ? min(w.len, q0 + 32 * WR) : w.len, steps = (end + BN - 1) / BN;
    const float c2 = a.scale * kLog2e;

    Streamed<T, DP, BN, VEC, NT, BUFS> keys{kb, a.k.tok, vb, a.v.tok, w.len, a.dim};
    // p (dp - de) of streamed rows k0 + 32 b .., zero where the row does not see them.
    auto weights = [&](const bf16_t* ks, const bf16_t* vs, int k0, int b, float de) {
        f32x16 s[2];
        const bf16_t* const lds[2] = {ks, vs};
        const int base[2] = {32 * b, 32 * b};
        const Owned<T, DP>* const own[2] = {&q, &dout};
        scores<T, DP, 2>(s, lds, base, own, lane);
#pragma unroll
        for (int r = 0; r < 16; ++r) s[0][r] = exp2_fast(__builtin_fmaf(s[0][r], c2, -lse2)) * (s[1][r] - de);
        if (k0 + 32 * b + 32 > w.len || (a.causal && k0 + 32 * b + 31 > qw)) {
            const int last = (a.causal ? min(qi, w.len - 1) : w.len - 1) - k0 - 32 * b - 4 * half;
#pragma unroll
            for (int r = 0; r < 16; ++r) s[0][r] = 8 * (r / 4) + r % 4 > last ? 0.f : s[0][r];
        }
        return s[0];
    };
    // Whether some row of the wave sees block b of the tile from k0 on.
    auto seen = [&](int k0, int b) { return k0 + 32 * b < end && (!a.causal || k0 + 32 * b <= qw + 31); };
    // delta = do . o carries the rounding of o to its type.  Where a row sees few
    // keys, o is as large as a value and that error as large as the other ones, so
    // blocks with up to kAttnRows keys first sum delta = sum_j p dp from the
    // scores.  With more keys and weights spread over them o averages out (error
    // under a fifth of a rounding of ds), and a second pass over them would cost 2/3
    // of the first.  Not so where one weight is near 1: then the row's ds are near 0
    // and carry an error of up to 2^-8 |do . o| in bf16, small beside the gradients of
    // other rows but not beside their own (600 keys, a weight of 0.98 on
    // one key: dq and dk off by 5% of their norm, 0.3% in blocks of up to 128 keys).
    const int rounds = (steps + TEAMS - 1) / TEAMS;
    if (end <= kAttnRows) {
        float sum = 0.f;
        keys.first(smem, team * BN, tid);
        for (int it = 0; it < rounds; ++it) {
            const int k0 = (it * TEAMS + team) * BN;
            keys.next(smem, it, k0, it * TEAMS + team + TEAMS < steps ? k0 + TEAMS * BN : -1, tid);
#pragma unroll
            for (int b = 0; b < NB; ++b)
                if (seen(k0, b)) {
                    const f32x16 s = weights(smem[it % BUFS][0], smem[it % BUFS][1], k0, b, 0.f);
#pragma unroll
                    for (int r = 0; r < 16; ++r) sum += s[r];
                }
        }
        delta = sum + __shfl_xor(sum, 32, 64);
        if (TEAMS > 1 && half == 0) stat[team][wave * 32 + lane] = delta;
        lds_barrier();                               // the tiles have been read
        if constexpr (TEAMS > 1) {
            delta = 0.f;
#pragma unroll
            for (int t = 0; t < TEAMS; ++t) delta += stat[t][wave * 32 + (lane & 31)];
        }
    }
    f32x16 g[DT] = {};
    keys.first(smem, team * BN, tid);
    for (int it = 0; it < rounds; ++it) {
        const int k0 = (it * TEAMS + team) * BN;
        keys.next(smem, it, k0, it * TEAMS + team + TEAMS < steps ? k0 + TEAMS * BN : -1, tid);
        const bf16_t *ks = smem[it % BUFS][0], *vs = smem[it % BUFS][1];
#pragma unroll
        for (int b = 0; b < NB; ++b)
            if (seen(k0, b)) accumulate<T, DP>(g, ks, 32 * b, weights(ks, vs, k0, b, delta), lane);
    }
    lds_barrier();                                   // the tiles are free
    bf16_t* mine = &smem[0][0][0] + wave * SHARE;
    if constexpr (TEAMS > 1) {
        if (team > 0) hand_over<DP>(mine, g, lane);
        lds_barrier();
        if (team > 0) return;
#pragma unroll
        for (int t = 1; t < TEAMS; ++t)
            take_over<DP>(&tiles[t][0][0][0] + wave * SHARE, g, 1.f, 1.f, lane);
    }
    uint32_t bad = bad_rows(live && any_nonfinite(g));
    // Where p may well be 0 the score of a key that is not finite came out as NaN:
    // fp32, and heads that leave a part of the tile to copies (Direct).
    if ((kTerms<T> == 3 || a.dim < DP) && end <= kAttnRows)
        for (uint32_t left = bad; left; left &= left - 1) {
            const int r = __builtin_ctz(left);
            const float d = delta_row<T>(a, w, qw + r, lane);
            if ((lane & 31) == r) delta = d;
        }
    if (live && half == 0) a.lse2[at] = lse2;
    if (live && half == 0) a.delta[at] = delta;
    bad &= ~bad_rows(lse2 != lse2 || delta != delta);          // all NaN
    if (bad) {
        bool right = faithful<T, DP, VEC>(a);
        if (!right)
            right = !odd_rows<T>(a.q, w, head, qw, min(qw + 32, w.len), a.dim, lane).inf &&
                    !odd_rows<T>(a.dout, w, head, qw, min(qw + 32, w.len), a.dim, lane).inf &&
                    !odd_rows<T>(a.k, w, kv, 0, end, a.dim, lane).inf && !odd_rows<T>(a.v, w, kv, 0, end, a.dim, lane).inf;
        if (right) bad &= bad_rows(qi <= spoiled_queries<T>(a, w, a.k, qw, ((a.causal ? min(end, qw + 32) : end) + 31) / 32 * 32, lane));
    }
    store_rows<T, DP, VEC>(mine, row_of<T>(a.dq, w, qw, head), a.dq.tok, g,
                           a.scale, a.dim, live_rows(qw, w.len) & ~bad, lane);
    for (; bad; bad &= bad - 1) {
        const int r = __builtin_ctz(bad);
        dq_row<T>(a, w, qw + r, __shfl(delta, r, 64), lane);
    }
}

// dk and dv: blocks of 128 keys of one key head, over the queries of every head
// that shares it, so the sum over heads stays in registers; four products a tile,
// Q and dO read both ways.  blockIdx.y: share of the queries.  Owned k and v and
// two sets of accumulators take 192 registers at heads of 128 in bf16: one wave
// per SIMD, or, HELD, two with v's rows in LDS instead.  fp32 takes 160 at heads of
// 64, and two waves per SIMD would spill 60 more: backward of 4 x 1024 tokens, 12
// heads, 205 us with two, 193 with one.
template <class T, int DP, bool VEC, bool HELD>
__global__ void __launch_bounds__(kThreads, (HELD ? 2 : kTerms<T> == 3 ? 1 : waves<T, DP>(2, 2))) attn_dkv_kernel(AttnArgs a) {
    constexpr int BM = HELD ? 32 : kStream<T>, NB = BM / 32, DT = DP / 32;
    __shared__ __attribute__((aligned(16))) char shared[8 * kTerms<T> * BM * DP + (HELD ? 2 * kAttnRows * DP : 0)];
    auto& smem = *reinterpret_cast<bf16_t (*)[2][2][kTerms<T> * BM * DP]>(shared);
    bf16_t* vrows = reinterpret_cast<bf16_t*>(shared) + 4 * BM * DP;   // of the block, if held
    __shared__ __attribute__((aligned(16))) float stat[2][2][BM];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int group = a.heads / a.kv_heads;
    const AttnTile tile = a.tiles[a.num_tiles + blockIdx.x / a.kv_heads];
    const int kv = blockIdx.x % a.kv_heads;
    int kt;
    if (!locate(a, tile, 0, kt)) return;    // the whole block
    const Where w{tile.start, tile.len, kv * group, kv};
    const int share = blockIdx.y;
    const int kw = kt + wave * 32, ki = kw + (lane & 31);
    const bool live = ki < w.len;

    Owned<T, DP> k;
    Owned<T, HELD ? 32 : DP> v;                      // not used if held in LDS
    k.template load<VEC>(row_of<T>(a.k, w, live ? ki : 0, kv), a.dim, live, half);
    if constexpr (HELD) {                            // with zeros for what is not there, as in registers
        using ST = Stage<bf16_t, DP, kAttnRows, true, kThreads>;
        u32x4 r[ST::N];
        ST::load(r, row_of<bf16_t>(a.v, w, 0, kv), a.v.tok, kt, w.len, a.dim, tid);
        ST::store(r, vrows, tid);
    } else v.template load<VEC>(row_of<T>(a.v, w, live ? ki : 0, kv), a.dim, live, half);
    const int first = a.causal ? kt / BM : 0, per = (w.len + BM - 1) / BM - first;
    // Steps of this block's share; step i: queries of tile first + i % per, head
    // kv * group + i / per.
    const int all = per * group, beg = (int)((int64_t)all * share / a.splits),
              steps = (int)((int64_t)all * (share + 1) / a.splits);
    const float c2 = a.scale * kLog2e;

    f32x16 gk[DT] = {}, gv[DT] = {};
    // A step's queries, their log-sum-exps and deltas; fp32: the tile on its way.
    std::conditional_t<kTerms<T> == 1, int, Split<DP, VEC, kThreads>> rq, rd;
    auto fetch = [&](int i, int buf) {
        const int h = w.head + i / per, row0 = (first + i % per) * BM;
        int td = tid;
        if constexpr (HELD) asm volatile("" : "+v"(td));     // as below
        if constexpr (kTerms<T> == 1) {
            const Pair<T, DP, BM, VEC, kThreads> rows{row_of<T>(a.q, w, 0, h), a.q.tok, row_of<T>(a.dout, w, 0, h),
                                                      a.dout.tok, w.len, a.dim};
            rows.fill(smem[buf], row0, td);
        } else {
            rq.load(row_of<T>(a.q, w, 0, h), a.q.tok, row0, w.len, a.dim, td);
            rd.load(row_of<T>(a.dout, w, 0, h), a.dout.tok, row0, w.len, a.dim, td);
        }
        if (tid < 2 * BM) {                          // whole waves
            const float* src = (tid < BM ? a.lse2 : a.delta) + h * a.tokens + w.start + min(row0 + tid % BM, w.len - 1);
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void*)src,
                (__attribute__((address_space(3))) void*)(&stat[buf][0][0] + __builtin_amdgcn_readfirstlane(tid >> 6) * 64),
                4, 0, 0);
        }
    };
    if (beg < steps) fetch(beg, beg & 1);
    for (int it = beg; it < steps; ++it) {
        const int q0 = (first + it % per) * BM;
        wait_loads();
        if constexpr (kTerms<T> == 3) {
            rq.store(smem[it & 1][0], tid);
            rd.store(smem[it & 1][1], tid);
        }
        lds_barrier();
        if (it + 1 < steps) fetch(it + 1, (it + 1) & 1);
        const bf16_t *qs = smem[it & 1][0], *ds = smem[it & 1][1];
        // The lane as of this step: addresses in LDS are then made anew in each, and
        // take no registers from one to the next.
        int ln = lane;
        if constexpr (HELD) asm volatile("" : "+v"(ln));
        const float *lse2 = stat[it & 1][0], *delta = stat[it & 1][1];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            const int qb = q0 + 32 * b;
            if (qb >= w.len || (a.causal && qb + 31 < kw)) continue;   // same for the whole wave
            f32x16 pd[2];
            f32x16 &p = pd[0], &dp = pd[1];
            if constexpr (HELD) {
                p = scores<T, DP>(qs, 32 * b, k, ln);
            } else {
                const bf16_t* const lds[2] = {qs, ds};
                const int base[2] = {32 * b, 32 * b};
                const Owned<T, DP>* const own[2] = {&k, &v};
                scores<T, DP, 2>(pd, lds, base, own, ln);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 ls = *reinterpret_cast<const f32x4*>(lse2 + 32 * b + 8 * j + 4 * half);
#pragma unroll
                for (int i = 0; i < 4; ++i) p[4 * j + i] = exp2_fast(__builtin_fmaf(p[4 * j + i], c2, -ls[i]));
            }
            // Queries of the sequence that see the lane's key.
            const bool edge = (a.causal && qb < kw + 31) || qb + 32 > w.len;
            const int from = a.causal ? ki : 0;
            if (edge) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = qb + 8 * (r / 4) + 4 * half + r % 4;
                    if (row < from || row >= w.len) p[r] = 0.f;
                }
            }
            accumulate<T, DP>(gv, ds, 32 * b, p, ln);
            if constexpr (HELD) {
                Owned<T, DP> held;
                held.load(vrows, wave * 32, ln);
                dp = scores<T, DP>(ds, 32 * b, held, ln);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 de = *reinterpret_cast<const f32x4*>(delta + 32 * b + 8 * j + 4 * half);
#pragma unroll
                for (int i = 0; i < 4; ++i) dp[4 * j + i] = p[4 * j + i] * (dp[4 * j + i] - de[i]);
            }
            if (edge) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = qb + 8 * (r / 4) + 4 * half + r % 4;
                    if (row < from || row >= w.len) dp[r] = 0.f;
                }
            }
            accumulate<T, DP>(gk, qs, 32 * b, dp, ln);
        }
    }
    lds_barrier();                                   // the tiles are free
    T* mine = reinterpret_cast<T*>(shared + wave * (sizeof shared / 4));
    const uint32_t keep = live_rows(kw, w.len);
    if (a.splits > 1) {
        const int64_t at = (kv * a.tokens + w.start + kw) * DP, one = (int64_t)a.kv_heads * a.tokens * DP;
        float* part = a.partial + 2 * share * one + at;
        store_rows<float, DP, true>(mine, part, DP, gk, a.scale, a.dim, keep, lane);
        store_rows<float, DP, true>(mine, part + one, DP, gv, 1.f, a.dim, keep, lane);
        return;
    }
    const uint32_t bad = bad_rows(live && (any_nonfinite(gk) || any_nonfinite(gv)));
    if (lane == 0) a.odd[blockIdx.x * 4 + wave] = bad;
    store_rows<T, DP, VEC>(mine, row_of<T>(a.dk, w, kw, kv), a.dk.tok, gk, a.scale, a.dim, keep, lane);
    store_rows<T, DP, VEC>(mine, row_of<T>(a.dv, w, kw, kv), a.dv.tok, gv, 1.f, a.dim, keep, lane);
}

// Rows of dk and dv that attn_dkv_kernel found not finite: a wave for 32 of them.  In a
// launch of its own (2 us), since in the kernel above their addresses would take scalar
// registers that it has not: kept in vector registers, they slow it by a fifth
// (packed 16418 tokens, 16/8 heads of 128, forward and backward 1097 us / 1235).
template <class T, int DP, bool VEC>
__global__ void __launch_bounds__(kThreads) attn_odd_keys_kernel(AttnArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const AttnTile tile = a.tiles[a.num_tiles + blockIdx.x / a.kv_heads];
    const int kv = blockIdx.x % a.kv_heads, group = a.heads / a.kv_heads;
    int kw;
    if (!locate(a, tile, wave * 32, kw)) return;
    uint32_t bad = a.odd[blockIdx.x * 4 + wave];
    if (!bad) return;
    const Where w{tile.start, tile.len, kv * group, kv};
    const int above = spoiled_keys<T>(a, w, kw, faithful<T, DP, VEC>(a), lane);
    for (; bad; bad &= bad - 1) {
        const int ki = kw + __builtin_ctz(bad);
        if (ki > above) dkv_row<T>(a, w, ki, lane);
    }
}

// Adds the shares of dk and dv, in their order: four features a thread, the rows
// of a tile over DP / 8 blocks.
template <class T, int DP>
__global__ void __launch_bounds__(kThreads) attn_join_kernel(AttnArgs a) {
    constexpr int LR = DP / 4, RB = kThreads / LR;   // threads of a row, rows of a block
    const int lane = threadIdx.x & 63, r = threadIdx.x / LR, d = threadIdx.x % LR * 4;
    const AttnTile tile = a.tiles[a.num_tiles + blockIdx.x / a.kv_heads];
    const int kv = blockIdx.x % a.kv_heads, group = a.heads / a.kv_heads;
    int kt;
    if (!locate(a, tile, 0, kt)) return;    // the whole block
    const Where w{tile.start, tile.len, kv * group, kv};
    const int64_t one = (int64_t)a.kv_heads * a.tokens * DP;
    const int ki = kt + blockIdx.y * RB + r;
    const bool live = ki < w.len;
    f32x4 gk = {}, gv = {};
    if (live && d < a.dim) {
        const float* part = a.partial + (kv * a.tokens + w.start + ki) * DP + d;
#pragma unroll 4
        for (int s = 0; s < a.splits; ++s) {
            gk += *reinterpret_cast<const f32x4*>(part + 2 * s * one);
            gv += *reinterpret_cast<const f32x4*>(part + (2 * s + 1) * one);
        }
    }
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (d + i < a.dim) t += gk[i] * 0.f + gv[i] * 0.f;
    // Rows that are not finite, of this wave: one by one.
    const uint64_t bad = __ballot(live && !(t == 0.f));
    constexpr uint64_t row_lanes = LR == 16 ? 0xffffull : 0xffffffffull;
    const int above = bad ? spoiled_keys<T>(a, w, (ki - lane / LR) / 32 * 32, faithful<T, DP, true>(a), lane) : 0;
    const bool redo = (bad >> (lane / LR * LR) & row_lanes) && ki > above;
    if (live && !redo) {
        T *dk = row_of<T>(a.dk, w, ki, kv), *dv = row_of<T>(a.dv, w, ki, kv);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (d + i < a.dim) {
                dk[d + i] = (T)gk[i];
                dv[d + i] = (T)gv[i];
            }
    }
    for (int k = 0; k < 64 / LR; ++k)
        if ((bad >> (k * LR) & row_lanes) && ki - lane / LR + k > above) dkv_row<T>(a, w, ki - lane / LR + k, lane);
}

// -------------------------------------------------------------- launches ---
template <class T>
bool aligned(const AttnOperand& o) {
    constexpr int E = 16 / sizeof(T);
    return reinterpret_cast<uintptr_t>(o.p) % 16 == 0 && o.tok % E == 0 && o.head % E == 0;
}

// Forward and dq pass: blocks of WR waves along the rows, TEAMS of them along
// the keys.
template <class T, int DP, bool VEC, int WR, int TEAMS>
void query_pass(const AttnArgs& a, bool backward, hipStream_t s) {
    const dim3 grid((unsigned)a.num_tiles * a.heads, kAttnRows / (32 * WR));
    if (backward) attn_dq_kernel<T, DP, VEC, WR, TEAMS><<<grid, 64 * WR * TEAMS, 0, s>>>(a);
    else attn_fwd_kernel<T, DP, VEC, WR, TEAMS><<<grid, 64 * WR * TEAMS, 0, s>>>(a);
}

template <class T, int DP, bool VEC>
hipError_t run(const AttnArgs& a, bool backward, hipStream_t s) {
    // Few blocks: their waves share the keys, so that a block's chain of tiles is
    // half as long, and up to 192 (fp32: 448) of 128 rows they are cut in two.
    // Many blocks: one team, whose blocks run out of step, so that one's softmax
    // meets the other's products.  Forward us of (4, 1), (4, 2), (2, 2):
    //   bf16, heads of 64, blocks of 128 rows 96: 19.5 15.6 12.6, 192: 19.9 16.3 15.1,
    //     288: 20.6 16.5 16.9, 384: 20.9 17.7 18.3, 576: 22.6 26.6 26.2, 960: 31.6 40.5 40.2
    //   bf16, 128: 256: 47.0 39.0 42.1, 512: 55.4 49.3 84.5, 768: 68.0 78.8 130
    //   fp32, 64, (4, 1) and (2, 2): 96: 62 44, 384: 66 54, 768: 86 99, 1536: 159 187
    //   fp32, 128: 128: 127 73, 256: 263 158, 512: 275 297, 1024: 402 593
    // Rows that do not start on 16 bytes take (4, 1) whatever the batch, so that two
    // more forms of each pass need not be built.  Forward us of aligned rows, of others
    // and of others by the rule above: bf16 heads of 64, 1024 tokens of 12 heads 13 30
    // 22, 4 x 1024 20 37 31; fp32 42 62 43, 57 67 55; bf16 128, 2 x 1024 of 16/8 24 47 41.
    const int64_t blocks = (int64_t)a.num_tiles * a.heads;
    constexpr bool small = sizeof(T) == 2;
    if (!VEC || blocks > (small ? 512 : 448)) query_pass<T, DP, VEC, 4, 1>(a, backward, s);
    else if (small && blocks > 192) {
        if constexpr (small) query_pass<T, DP, true, 4, 2>(a, backward, s);
    } else query_pass<T, DP, true, 2, 2>(a, backward, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !backward) return e;
    // bf16 heads of 128: with v's rows in LDS two blocks fit a CU instead of one,
    // for more LDS reads and half tiles.  us with them there / in registers: packed
    // 16418 tokens (1032 blocks) 827 / 873, 16 x 2048 (2048) 1146 / 1254, 4 x 8192
    // (2048) 3890 / 4195; 4 x 2048 (512) 338 / 295, 2 x 2048 (256) 222 / 183.
    const dim3 keys((unsigned)a.num_tiles * a.kv_heads, a.splits);
    constexpr bool can_hold = VEC && sizeof(T) == 2 && DP == 128;
    if (can_hold && (int64_t)a.num_tiles * a.kv_heads >= 1024)
        attn_dkv_kernel<T, DP, VEC, can_hold><<<keys, kThreads, 0, s>>>(a);
    else attn_dkv_kernel<T, DP, VEC, false><<<keys, kThreads, 0, s>>>(a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (a.splits == 1) attn_odd_keys_kernel<T, DP, VEC><<<keys, kThreads, 0, s>>>(a);
    else attn_join_kernel<T, DP><<<dim3((unsigned)a.num_tiles * a.kv_heads, DP / 8), kThreads, 0, s>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t dispatch(const AttnArgs& a, bool backward, hipStream_t s) {
    bool vec = a.dim % (16 / (int)sizeof(T)) == 0 && aligned<T>(a.q) && aligned<T>(a.k) && aligned<T>(a.v) &&
               aligned<T>(a.out);
    if (backward) vec = vec && aligned<T>(a.dout) && aligned<T>(a.dq) && aligned<T>(a.dk) && aligned<T>(a.dv);
    if (a.dim <= 64) return vec ? run<T, 64, true>(a, backward, s) : run<T, 64, false>(a, backward, s);
    return vec ? run<T, 128, true>(a, backward, s) : run<T, 128, false>(a, backward, s);
}

}  // namespace

// Shares of the queries in the dk/dv pass: enough blocks for two on every CU, at
// most 4, since the partial sums of a share are written and read once more.
// Backward us of 1, 2, 4, 8 shares: 64 blocks (heads of 64, 32 over 8) 48.8 35.3
// 27.4 28.0; 128 (the same) 240 152 124 123; 256 (128, 16 over 8) 445 341 365 429;
// 1536 (64, 12) 137 223 310 483.
int attention_splits(int64_t num_tiles, int kv_heads) {
    const int64_t blocks = num_tiles * kv_heads;
    return blocks >= 512 ? 1 : blocks >= 256 ? 2 : 4;
}

int64_t attention_workspace(const AttnArgs& a) {
    const int64_t rows = 2 * (int64_t)a.heads * a.tokens, pitch = a.dim <= 64 ? 64 : 128;
    return (rows + 3) / 4 * 4 + (a.splits > 1 ? 2 * a.splits * (int64_t)a.kv_heads * a.tokens * pitch
                                              : (int64_t)kAttnRows / 32 * a.num_tiles * a.kv_heads);
}

hipError_t launch_attention_forward(DType t, const AttnArgs& a, hipStream_t s) {
    return t == DType::BF16 ? dispatch<bf16_t>(a, false, s) : dispatch<float>(a, false, s);
}

hipError_t launch_attention_backward(DType t, const AttnArgs& a, hipStream_t s) {
    return t == DType::BF16 ? dispatch<bf16_t>(a, true, s) : dispatch<float>(a, true, s);
}

}  // namespace np
