// Arguments of the calls by which few tokens of every query attend to its entity list (read.hip, packed.hip), and the join of
// lists that several blocks have read.
#pragma once

#include "attend.h"

namespace lkg {

struct ReadArgs {
    int num_queries, tokens, heads, kv_heads, group, dim, rows, shift;  // rows: tokens x group per key head; 2^shift entries per block
    long long num_entries, num_entities, blocks;
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

// Lists cut into several blocks: a wavefront per (query, token, head) joins the parts, in their order.
template <class E> __global__ __launch_bounds__(256) void k_read_join(ReadArgs a) {
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const int lane = threadIdx.x & 63;
    const long long at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6), per = (long long)a.tokens * a.heads;
    if (at >= a.num_queries * per) return;
    const int d = (int)(at / per), th = (int)(at % per);
    const long long e0 = taken_into(a.off[d], a.num_entries), e1 = taken_into(a.off[d + 1], a.num_entries);
    const long long len = e1 > e0 ? e1 - e0 : 0;
    if (len <= (1ll << a.shift)) return;
    const long long b0 = first_block(a.off, d, a.num_entries, 1, a.shift), parts = (len + (1ll << a.shift) - 1) >> a.shift;
    float top = kLowest;
    for (long long i = lane; i < parts; i += 64) top = fmaxf(top, a.part_ml[2 * ((b0 + i) * per + th)]);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
    const int c = (lane & 31) * 4;
    float sum = 0.f;
    f32x4 o = {0, 0, 0, 0};
    if (c < a.dim)
        for (long long i = lane >> 5; i < parts; i += 2) {
            const long long p = (b0 + i) * per + th;
            const float w = exp2_fast(a.part_ml[2 * p] - top);
            sum = __builtin_fmaf(w, a.part_ml[2 * p + 1], sum);
            f32x4 x = *(const f32x4 *)(a.part_o + p * a.dim + c);
#pragma unroll
            for (int e = 0; e < 4; e++) o[e] = __builtin_fmaf(w, x[e], o[e]);
        }
    sum = halves_sum(sum);
#pragma unroll
    for (int e = 0; e < 4; e++) o[e] = halves_sum(o[e]);
    if (lane >= 32 || c >= a.dim) return;
    const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    typename Vec4<E>::type x;
#pragma unroll
    for (int e = 0; e < 4; e++) x[e] = (E)(o[e] * inv);
    *(typename Vec4<E>::type *)((E *)a.out + at * a.dim + c) = x;
    if (lane == 0) a.lse[at] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * kLn2;
}

inline int64_t part_bytes(const ReadArgs &a) {  // one block per list: nothing to join
    return a.num_entries <= (1ll << a.shift) ? 0 : (int64_t)a.blocks * a.tokens * a.heads * (a.dim + 2) * 4;
}

}  // namespace lkg
