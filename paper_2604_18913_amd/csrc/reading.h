// Device helpers of the calls that read a retrieval into a language model (attend*.hip, read.hip, answers.hip).
#pragma once

#include "common.h"

#include <utility>

namespace lkg {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A bias of -infinity, or so low that it can only be meant to hide, stands as kHidden: 2^this is 0, and its square finite, where
// that of an infinity is not.  Low is what is below kLeastBias (float16's lowest value is not, bfloat16's is): 32 bits hold scores to
// 2^-8 beside that, and beside -1e9 not at all, so that p of a row that sees nothing else, made of y - lse, would be anything.  kLowest is the running maximum of a row that has seen nothing,
// below any other score and above the hidden ones: those weigh 0 from the first tile on, and a sum of 0 tells that nothing was seen.
constexpr float kHidden = -1e15f, kLowest = 0.5f * kHidden, kLeastBias = -7e4f * kLog2e;

// The two 16-bit types: eight values as a matrix instruction takes them, and that instruction on 32 x 32 x 16.
// Lane l holds A[l % 32][8 (l / 32) ..] and B[8 (l / 32) ..][l % 32]; C's element r is row 8 (r / 4) + 4 (l / 32) + r % 4
// of column l % 32.  So C = rows x columns puts a column into a lane (and its partner in the other half), which makes
// softmax sums a loop over registers and one exchange, and C's elements 8 s .. 8 s + 7 are the B of the next product's
// step s as they are, if its A takes the 16 places of the step in the same order: 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3
// in half h, which is what two transposing LDS reads give.
template <class E> struct Vec8 { typedef E type __attribute__((ext_vector_type(8))); };
template <class E> struct Vec4 { typedef E type __attribute__((ext_vector_type(4))); };
typedef __bf16 bf16;
typedef _Float16 fp16;

__device__ __forceinline__ f32x16 mfma(Vec8<bf16>::type a, Vec8<bf16>::type b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(Vec8<fp16>::type a, Vec8<fp16>::type b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

template <class E> __device__ __forceinline__ typename Vec8<E>::type as8(u32x4 x) { return __builtin_bit_cast(typename Vec8<E>::type, x); }

__device__ __forceinline__ f32x16 zero16() {
    f32x16 z;
#pragma unroll
    for (int i = 0; i < 16; i++) z[i] = 0.f;
    return z;
}

// eight elements of a C as the B of the next product, each rounded once to E (nearest even): the operands of a matrix
// instruction have 16 bits, and the products are summed in 32
template <class E, int S> __device__ __forceinline__ typename Vec8<E>::type rounded8(const f32x16 &c) {
    typename Vec8<E>::type r;
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = (E)c[8 * S + i];
    return r;
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }  // 1 ulp, 0 below 2^-126
__device__ __forceinline__ float rcp_fast(float x) { return __builtin_amdgcn_rcpf(x); }    // 1 ulp

// x of this lane and of its partner in the other half of the wavefront.  (The exchange gets two registers: of one given
// twice the compiler takes both results to be the same.)
__device__ __forceinline__ void both_halves(float x, float &lo, float &hi) {
    unsigned a = __builtin_bit_cast(unsigned, x), b = a;
    asm("" : "+v"(b));
    auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    lo = __builtin_bit_cast(float, (unsigned)r[0]);
    hi = __builtin_bit_cast(float, (unsigned)r[1]);
}
__device__ __forceinline__ float halves_max(float x) {
    float lo, hi;
    both_halves(x, lo, hi);
    return fmaxf(lo, hi);
}
__device__ __forceinline__ float halves_sum(float x) {
    float lo, hi;
    both_halves(x, lo, hi);
    return lo + hi;
}

// what the wavefront's lanes have written to LDS is there for its other lanes (LDS runs a wavefront's accesses in order)
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// f(0), f(1), .. f(N - 1), each with its number as a constant: loops that must be unrolled whatever their size, since registers
// are picked by it.
template <class F, int... I> __device__ __forceinline__ void in_turn(F &f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F> __device__ __forceinline__ void in_turn(F f) { in_turn(f, std::make_integer_sequence<int, N>{}); }

// A round's 32 elements go through their stages, one a step, while its `all` matrix instructions are issued: element e begins at
// step e all / 32, so that a step holds one stage each of some neighbouring elements.  A vector instruction that
// waits for the one before it takes twice as long as one that does not (8 clocks for 4 to 5): chains of one element alone
// would leave the units idle half of the time.  The elements whose stage `s` falls on step `at`: [first, behind).
template <int ALL> constexpr int first_of(int at) { return at < 0 ? 0 : at >= ALL ? 32 : (at * 32 + ALL - 1) / ALL; }

template <class E> struct Pair { typedef E type __attribute__((ext_vector_type(2))); };
template <class E> __device__ __forceinline__ unsigned rounded2(float a, float b) {  // nearest even, as rounded8
    typename Pair<E>::type r = {(E)a, (E)b};
    return __builtin_bit_cast(unsigned, r);
}
__device__ __forceinline__ void here(unsigned &x) { asm volatile("" : "+v"(x)); }

// Keeps what makes x in its place among the matrix instructions: the compiler would gather it behind them.
__device__ __forceinline__ void here(float &x) { asm volatile("" : "+v"(x)); }

// A tile in LDS: rows of DP 16-bit values in 16-byte chunks, chunk c of row r at place c ^ spread(r), so that neither the
// 16 rows x one chunk that a row-wise read asks for at a time nor the 4 rows x 64 bytes of a transposing read share banks.
template <int DP> __device__ __forceinline__ int spread(int r) {
    if (DP == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
    return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}

// Places in LDS are 32-bit offsets: a lane's place in a tile is made once, the chunk's part of it is flipped into it (the
// tiles begin at multiples of 8 KiB, so that no flipped bit meets another).
typedef __attribute__((address_space(3))) char lds_char;
__device__ __forceinline__ unsigned lds_place(const void *p) { return (unsigned)(uintptr_t)(lds_char *)p; }

// A[row][16 kk + 8 (l / 32) ..] of the 32 rows at a tile's begin: rows_place of the lane, then a chunk per kk
template <int DP> __device__ __forceinline__ unsigned rows_place(int lane) {
    int r = lane & 31;
    return r * (DP * 2) + (((lane >> 5) ^ spread<DP>(r)) << 4);
}
template <class E> __device__ __forceinline__ typename Vec8<E>::type rows_chunk(unsigned place, int kk) {
    typedef __attribute__((address_space(3))) const u32x4 chunk;
    return as8<E>(*(chunk *)(uintptr_t)(place ^ (kk << 5)));
}

// A = the tile's transpose: lane l gets column 32 dt + l % 32 of the rows r0 + 4 (l / 32) .. + 3 and r0 + 8 + 4 (l / 32) .. + 3,
// r0 = 0 or 16: columns_place of the lane, then a chunk per (r0, dt)
template <int DP> __device__ __forceinline__ unsigned columns_place(int lane) {
    int r = ((lane & 15) >> 2) + 4 * (lane >> 5), c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    return r * (DP * 2) + ((c ^ spread<DP>(r)) << 4) + (lane & 1) * 8;
}
template <class E, int DP> __device__ __forceinline__ typename Vec8<E>::type columns_chunk(unsigned place, int r0, int dt) {
    typedef __attribute__((address_space(3))) s16x4 lds4;
    struct { s16x4 a, b; } both;
    both.a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)((place ^ (dt << 6)) + r0 * (DP * 2)));
    both.b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(uintptr_t)((place ^ (dt << 6) ^ 32) + (r0 + 8) * (DP * 2)));
    return __builtin_bit_cast(typename Vec8<E>::type, both);
}

// ---------------------------------------------------------------- ragged batches
__device__ __forceinline__ long long taken_into(long long x, long long hi) { return x < 0 ? 0 : x > hi ? hi : x; }

// Blocks of 2^shift rows over the documents of a ragged array, without a pass over their lengths: document d has the
// blocks (off[d] mult >> shift) + d up to those of d + 1, at least as many as it needs.  The document of a block by a
// search of the whole wavefront, two rounds for 4,096 documents.
__device__ __forceinline__ long long first_block(const int64_t *off, int d, long long total, int mult, int shift) {
    return (taken_into(off[d], total) * mult >> shift) + d;
}
__device__ __forceinline__ int document_of(const int64_t *off, int n, long long total, int mult, int shift, long long block, int lane) {
    int lo = 0, span = n;
    while (span > 1) {
        int step = (span + 63) >> 6, at = lane * step;
        bool below = at < span && first_block(off, lo + at, total, mult, shift) <= block;
        int count = __popcll(__ballot(below));
        int skip = (count > 0 ? count - 1 : 0) * step;
        lo += skip;
        span = span - skip < step ? span - skip : step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// ---------------------------------------------------------------- scores
// What the kernels make of logoskg_score, in units of log 2.  Without a cap y = z k, k = scale log2 e.  With one
// y = c - 2 c / (2^(z k) + 1), c = cap log2 e, which is c tanh(z scale / cap) for k = 2 log2 e scale / cap (with the sign of z k taken
// off first and put back: 2^.. may be infinite, and is y = c then).  That form's error is c 2^-23 whatever y is, so it is for products above `most` alone, where tanh's
// argument is 1/2 or more; up to there y = z times a polynomial in z^2 (near), exact to 5.5e-7 of y under any cap, which also
// costs five instructions instead of an exponential, a reciprocal and three.
struct ScoreArgs {
    float k, c;
    float slope;    // |y| <= |z| slope
    float most;     // largest |z| that the near form holds for (no cap: any; below 0: none)
    float near[4];
    const void *bias;
    const int32_t *buckets;
    int num_buckets, max_distance;
};

inline ScoreArgs score_args(const logoskg_score &s) {
    ScoreArgs a;
    const float lin = s.scale * kLog2e;
    const double w = s.cap > 0 ? (double)s.scale / s.cap : 0.0, steep = 2.0 * kLog2e * w;
    a.k = s.cap > 0 ? (float)(steep > 3e38 ? 3e38 : steep < -3e38 ? -3e38 : steep) : lin;
    a.c = s.cap > 0 ? (s.cap > 1e37f ? 1e37f : s.cap) * kLog2e : 0.f;  // (twice it is finite; products under such caps are near)
    a.slope = lin < 0 ? -lin : lin;
    a.most = INFINITY;
    // tanh(x) / x on |x| <= 1/2 as a polynomial in x^2: smallest largest relative error, 5.5e-7 (Remez exchange on [0, 1/4])
    const double fit[4] = {0.999999463558197, -0.33326318860054016, 0.13190296292304993, -0.04440222680568695};
    double f = lin;
    for (int i = 0; i < 4; i++, f *= w * w) a.near[i] = (float)(fit[i] * f);
    if (s.cap > 0 && w != 0.0) {
        const double most = 0.5 / (w < 0 ? -w : w);
        a.most = most < 1e18 ? (float)most : 1e18f;  // (z^2 is finite)
        if (!(f > -1e30 && f < 1e30)) {  // a cap so small that the coefficients leave 32 bits: products that are near are 0
            a.most = -1.f;
            for (float &x : a.near) x = 0.f;
        }
    }
    a.bias = s.bias;
    a.buckets = s.buckets;
    a.num_buckets = s.num_buckets;
    a.max_distance = s.max_distance;
    return a;
}

// A score under a cap, of a product that is near
__device__ __forceinline__ float near_capped(const ScoreArgs &s, float z) {
    const float zz = z * z;
    float w = __builtin_fmaf(zz, s.near[3], s.near[2]);
    w = __builtin_fmaf(zz, w, s.near[1]);
    w = __builtin_fmaf(zz, w, s.near[0]);
    return z * w;
}
// .. of any; `share`: 1 / (2^|z k| + 1), of which the backward makes the slope (of -z k it would be near 1, and 1 - share, which the
// slope has as a factor, the rounding error of that)
__device__ __forceinline__ float any_capped(const ScoreArgs &s, float z, float &share) {
    const float zk = z * s.k;
    share = rcp_fast(exp2_fast(__builtin_fabsf(zk)) + 1.f);
    const float far = __builtin_copysignf(__builtin_fmaf(-2.f * s.c, share, s.c), zk), near = near_capped(s, z);
    return __builtin_fabsf(z) <= s.most ? near : far;
}
__device__ __forceinline__ float any_capped(const ScoreArgs &s, float z) {
    float share;
    return any_capped(s, z, share);
}
// Sixteen products of a wavefront's lanes to scores, in place: by the near form, which is cheaper, where all of them are near.  PARTS
// of them at a time: both forms of all sixteen take more registers than the kernels for few rows have; with four at a time 33 rows
// before 5,000 keys (32 / 8 heads of 128) take 77 us, with both forms of each 85.
template <int PARTS> __device__ __forceinline__ void cap_scores(const ScoreArgs &s, f32x16 &z) {
    constexpr int N = 16 / PARTS;
    float size = 0.f;
#pragma unroll
    for (int r = 0; r < 16; r++) size = fmaxf(size, __builtin_fabsf(z[r]));
    const bool far = wave_any(size > s.most);
#pragma unroll
    for (int j = 0; j < PARTS; j++) {
        float y[N];
        if (PARTS == 1 && far) {
#pragma unroll
            for (int e = 0; e < N; e++) y[e] = any_capped(s, z[N * j + e]);
        } else {
#pragma unroll
            for (int e = 0; e < N; e++) y[e] = near_capped(s, z[N * j + e]);
        }
        if (PARTS > 1 && far) {
#pragma unroll
            for (int e = 0; e < N; e++) y[e] = any_capped(s, z[N * j + e]);
        }
#pragma unroll
        for (int e = 0; e < N; e++) z[N * j + e] = y[e];
    }
}

__device__ __forceinline__ int wave_min(int x) {
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
        int y = __shfl_xor(x, s);
        x = y < x ? y : x;
    }
    return x;
}
__device__ __forceinline__ int wave_max(int x) {
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) {
        int y = __shfl_xor(x, s);
        x = y > x ? y : x;
    }
    return x;
}

// Biases of the heads h0 .. h0 + group - 1 by distance, times log2 e, in LDS: [group][2 M + 1]
template <class E> __device__ __forceinline__ void bias_to_lds(float *table, const ScoreArgs &s, int h0, int group, int tid, int threads) {
    const E *bias = (const E *)s.bias;
    int places = 2 * s.max_distance + 1;
    auto lowest = [](float x) { return x < kLeastBias ? kHidden : x; };
    for (int i = tid; i < places; i += threads) {
        int b = s.buckets[i];
        b = b < 0 ? 0 : b >= s.num_buckets ? s.num_buckets - 1 : b;
        for (int g = 0; g < group; g++) table[g * places + i] = lowest((float)bias[(long long)(h0 + g) * s.num_buckets + b] * kLog2e);
    }
}

// Where a distance's entry stands in a table of 2 M + 1 words: one end of the distance is fixed (pos), the other, x, counts
// with `sign`; clamped first, so that no difference leaves 32 bits.
struct Places {
    int lo, hi;     // x is taken into these
    unsigned base;  // of a table of words in LDS: the entry of x is at base + 4 x (wrapping)
};
__device__ __forceinline__ int added(int a, int b) { return __builtin_elementwise_add_sat(a, b); }
// of keys, for a row at q_pos: distance x - q_pos
__device__ __forceinline__ Places places_of_keys(int q_pos, int M, unsigned table) {
    return Places{added(q_pos, -M), added(q_pos, M), table + 4u * ((unsigned)M - (unsigned)q_pos)};
}
__device__ __forceinline__ int clamped(int x, int lo, int hi) { return __builtin_elementwise_min(__builtin_elementwise_max(x, lo), hi); }
__device__ __forceinline__ unsigned place_of_key(const Places &p, int x) { return p.base + 4u * (unsigned)clamped(x, p.lo, p.hi); }
// of rows, for a key at k_pos: distance k_pos - x
__device__ __forceinline__ Places places_of_rows(int k_pos, int M, unsigned table) {
    return Places{added(k_pos, -M), added(k_pos, M), table + 4u * ((unsigned)M + (unsigned)k_pos)};
}
__device__ __forceinline__ unsigned place_of_row(const Places &p, int x) { return p.base - 4u * (unsigned)clamped(x, p.lo, p.hi); }
__device__ __forceinline__ float float_at(unsigned place) { return *(__attribute__((address_space(3))) const float *)(uintptr_t)place; }
__device__ __forceinline__ int int_at(unsigned place) { return *(__attribute__((address_space(3))) const int *)(uintptr_t)place; }

__device__ __forceinline__ int distance_place(int k_pos, int q_pos, int M) { return clamped(__builtin_elementwise_sub_sat(k_pos, q_pos), -M, M) + M; }

template <class F> logoskg_status allow_lds(F *kernel, size_t bytes) {
    if (bytes > (64 << 10)) LKG_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    return LOGOSKG_OK;
}

const char *bad_score(const logoskg_score &s, int heads, int kv_heads);  // attend.hip: why a call refuses it, or NULL
const char *bad_heads(int dtype, int heads, int kv_heads, int dim);

}  // namespace lkg
