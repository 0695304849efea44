// Arguments of the calls by which few tokens of every query attend to its entity list (read.hip, packed.hip), and the join of
// lists that several blocks have read.
#pragma once

#include "attend.h"

namespace lkg {

struct ReadArgs {
    int num_queries, tokens, heads, kv_heads, group, dim, rows, shift;  // rows: tokens x group per key head; 2^shift entries per block
    long long num_entries, num_entities, blocks, first;  // first: block (of the join, row) that a launch begins with
    const int64_t *off;
    const int32_t *entity, *q_pos;
    const uint8_t *hop;
    const void *q, *keys, *values;
    long long key_row, key_head, value_row, value_head;
    ScoreArgs score;
    void *out;
    float *lse;
    float *part_o, *part_ml;  // [blocks][heads x tokens][dim], [..][2]: sums so far of lists cut into several blocks
};

// Lists cut into several blocks: LG lanes per (query, token, head) join the parts, four elements each: the even and the odd ones in
// their order, then the two.  With twice the lanes that a row has (SIDES = 2: lists of many parts) those go side by side, with
// as many (1) one behind the other, four parts asked for at a time; the sums are the same.  65,536 rows of some two parts of 64
// elements: 14 us, side by side 28; 32 rows of 15 parts of 128: 5.2, side by side 3.9.
template <class E, int LG, int SIDES> __global__ __launch_bounds__(256) void k_read_join(ReadArgs a) {
    constexpr int kHalf = LG / SIDES, kStep = 4 * SIDES;
    const int lane = threadIdx.x % LG, side = lane / kHalf;
    const long long at = a.first + (long long)blockIdx.x * (256 / LG) + threadIdx.x / LG, per = (long long)a.tokens * a.heads;
    if (at >= a.num_queries * per) return;
    const int d = (int)(at / per), th = (int)(at % per);
    const long long e0 = taken_into(a.off[d], a.num_entries), e1 = taken_into(a.off[d + 1], a.num_entries);
    const long long len = e1 > e0 ? e1 - e0 : 0;
    if (len <= (1ll << a.shift)) return;
    const long long b0 = first_block(a.off, d, a.num_entries, 1, a.shift), parts = (len + (1ll << a.shift) - 1) >> a.shift;
    const float *ml = a.part_ml + 2 * (b0 * per + th), *part = a.part_o + (b0 * per + th) * a.dim;
    float top = kLowest;
    for (long long i = lane; i < parts; i += LG) top = fmaxf(top, ml[2 * i * per]);
#pragma unroll
    for (int s = LG / 2; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
    const int c = lane % kHalf * 4;
    const bool in = c < a.dim;
    float sums[2] = {0.f, 0.f};
    f32x4 os[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    for (long long i = side; i < parts; i += kStep) {
        float m[4], l[4];
        f32x4 x[4];
#pragma unroll
        for (int u = 0; u < 4; u++)
            if (i + u * SIDES < parts) {
                m[u] = ml[2 * (i + u * SIDES) * per], l[u] = ml[2 * (i + u * SIDES) * per + 1];
                if (in) x[u] = *(const f32x4 *)(part + (i + u * SIDES) * per * a.dim + c);
            }
#pragma unroll
        for (int u = 0; u < 4; u++)
            if (i + u * SIDES < parts) {
                constexpr int kOdd = SIDES == 1;
                const float w = exp2_fast(m[u] - top);
                sums[u & kOdd] = __builtin_fmaf(w, l[u], sums[u & kOdd]);
#pragma unroll
                for (int e = 0; e < 4; e++) os[u & kOdd][e] = __builtin_fmaf(w, x[u][e], os[u & kOdd][e]);
            }
    }
    if (SIDES == 2) {
        sums[1] = __shfl_xor(sums[0], kHalf);
#pragma unroll
        for (int e = 0; e < 4; e++) os[1][e] = __shfl_xor(os[0][e], kHalf);
    }
    const float sum = sums[0] + sums[1];
    if (!in || side > 0) return;
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    typename Vec4<E>::type x;
#pragma unroll
    for (int e = 0; e < 4; e++) x[e] = (E)((os[0][e] + os[1][e]) * inv);
    *(typename Vec4<E>::type *)((E *)a.out + at * a.dim + c) = x;
    if (lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * kLn2;
}

inline int64_t part_bytes(const ReadArgs &a) {  // one block per list: nothing to join
    return a.num_entries <= (1ll << a.shift) ? 0 : (int64_t)a.blocks * a.tokens * a.heads * (a.dim + 2) * 4;
}

// The blocks of a call, each for `heads` groups of key heads, in launches of fewer than 2^32 threads: launch(the grid's x) for
// whole eights of them, which the card's dies share.
template <class F> void each_eight_blocks(ReadArgs &a, int heads, int threads, F launch) {
    launch_ranges((a.blocks + 7) / 8, 1, [&](long long first, long long n) {
        a.first = 8 * first;
        launch((unsigned)(8 * n * heads));
    }, (long long)UINT32_MAX / threads / heads / 8);
}

template <class E> logoskg_status launch_join(ReadArgs a, hipStream_t st) {
    if (!part_bytes(a)) return LOGOSKG_OK;
    const long long n = (long long)a.num_queries * a.tokens * a.heads;
    const bool many = a.num_entries >> a.shift > 8ll * a.num_queries;
    const int lanes = (a.dim <= 64 ? 16 : 32) * (many ? 2 : 1);
    launch_ranges(n, 256 / lanes, [&](long long first, long long rows) {
        a.first = first;
        const dim3 grid((unsigned)((rows * lanes + 255) / 256));
        if (a.dim <= 64) many ? k_read_join<E, 32, 2><<<grid, 256, 0, st>>>(a) : k_read_join<E, 16, 1><<<grid, 256, 0, st>>>(a);
        else many ? k_read_join<E, 64, 2><<<grid, 256, 0, st>>>(a) : k_read_join<E, 32, 1><<<grid, 256, 0, st>>>(a);
    });
    LKG_HIP(hipGetLastError());
    return LOGOSKG_OK;
}

}  // namespace lkg
