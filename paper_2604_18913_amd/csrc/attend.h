// Arguments and tiles that the forward and the backward of the attention share.
#pragma once

#include "reading.h"

namespace lkg {

constexpr int kAttThreads = 256;  // four wavefronts
constexpr int kAttRowsShift = 7;  // a block's rows: 4 x 32
constexpr int kAttRows = 1 << kAttRowsShift;
constexpr int kFewShift = 5;       // rows of a block where there are few: 32
constexpr size_t kLds = 160 << 10;                        // of a compute unit
constexpr long long kMostRows = (1ll << 31) - (1 << 16);  // of a batch: places in a document are 32-bit, with room for a tile
constexpr long long kMostStride = 1 << 23;                // between rows, in elements: a tile's rows within 2^31 bytes
constexpr int kMostGroup = 128;                           // heads that share a key head

struct AttArgs {
    int num_docs, heads, kv_heads, group, dim, causal;
    long long num_rows, num_keys;
    const int64_t *q_off, *k_off;
    const void *q, *k, *v;
    long long q_row, q_head, k_row, k_head, v_row, v_head;
    const int32_t *prefix, *q_pos, *k_pos;
    ScoreArgs score;
    void *out;
    float *lse;
    // backward
    const void *dout;
    void *dq, *dk, *dv, *dbias;
    float *delta;      // [num_rows][heads] sum of p dP, from the first kernel to the second
    float *bias_part;  // [key_blocks][heads][num_buckets]
    float scale;
    float curve;       // .. of scale (1 - tanh^2) = scale + curve y^2, y = c tanh in units of log 2
    float slope;       // with a cap: 4 scale, of scale (1 - tanh^2) = 4 scale r (1 - r), r = 1 / (2^(z k) + 1)
    long long row_blocks, key_blocks;
    long long few_blocks;  // of 32 rows
    int *row_order, *key_order;  // blocks in the order of their work, or NULL
    int bias_columns;  // 64, or 32 where LDS has no room for them
};

struct AttDoc {  // a document: where its rows and keys begin, and how many there are
    long long row0, key0;
    int rows, keys, prefix;
    // keys that row i sees: the first seen(i)
    __device__ __forceinline__ int seen(int i, int causal) const {
        if (!causal) return keys;
        int n = i + (keys - rows) + 1;  // (rows and keys below 2^31: their sum may not be)
        n = n < prefix ? prefix : n;
        return n < 0 ? 0 : n > keys ? keys : n;
    }
};

__device__ __forceinline__ AttDoc att_doc(const AttArgs &a, int d) {
    AttDoc o;
    o.row0 = taken_into(a.q_off[d], a.num_rows);
    o.key0 = taken_into(a.k_off[d], a.num_keys);
    long long r1 = taken_into(a.q_off[d + 1], a.num_rows), k1 = taken_into(a.k_off[d + 1], a.num_keys);
    o.rows = r1 > o.row0 ? (int)(r1 - o.row0) : 0;
    o.keys = k1 > o.key0 ? (int)(k1 - o.key0) : 0;
    o.prefix = a.prefix ? a.prefix[d] : 0;
    return o;
}

// Rows or keys that no document holds lie before the first document and behind the last, and get zeros.  A block has N places (of
// row x head of the group, or of a key), the first of them at `first` from its document's begin; f(place in the array) for those that
// nobody holds.  All of them fall on some block: what begins before the first document's own blocks on the blocks before those,
// but for the places before the first of these, which block 0 takes too; what lies behind the last document on its blocks.
template <int N, class F> __device__ __forceinline__ void each_spare(long long begin, long long held, long long total, int d, int num_docs, long long block, long long first, int tid, F f) {
    const bool front = d == 0 && first < 0, behind = d + 1 == num_docs && first + N > held;
    if (front || behind)
#pragma unroll 1
        for (int i = tid; i < N; i += kAttThreads) {
            const long long x = first + i;
            if (((front && x < 0) || (behind && x >= held)) && begin + x < total) f(begin + x);
        }
    if (block == 0)
#pragma unroll 1
        for (int i = tid; i < (int)(begin & (N - 1)); i += kAttThreads) f(i);
}
template <class E> __device__ __forceinline__ void clear_row(E *row, int dim) {
#pragma unroll 1
    for (int c = 0; c < dim; c += 8) *(u32x4 *)(row + c) = u32x4{0, 0, 0, 0};
}

// A window of memory from `base` on: reads behind `bytes` give zeros (and touch nothing).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t window(const void *base, long long bytes) {
    bytes = bytes < 0 ? 0 : bytes > 0x7ffffff0 ? 0x7ffffff0 : bytes;
    return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, (int)bytes, 0x00027000);  // raw bytes
}
__device__ __forceinline__ u32x4 window_chunk(__amdgpu_buffer_rsrc_t w, unsigned offset) {
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(w, offset, 0, 0));
}
constexpr unsigned kNowhere = 0x80000000u;  // behind every window

// Moves N rows x DP values of a ragged array's head into a tile through registers, spread over the block's threads: tile after
// tile of a matrix of `rows` rows, zeros behind the last row and behind dim.
template <int N, int DP> struct TileLoad {
    static constexpr int kChunks = N * DP / 8 / kAttThreads, kStep = kAttThreads / (DP / 8);  // rows between a thread's chunks
    const char *at;  // the next tile
    long long left;  // bytes from there to the end of the last row
    unsigned row_bytes, from, to;
    __device__ __forceinline__ void begin(const char *base, unsigned bytes, int row, int rows, int dim, int tid) {
        const int r = tid / (DP / 8), c = tid % (DP / 8);
        row_bytes = bytes;
        go_to(base, row, rows, dim);
        from = c * 8 < dim ? r * bytes + c * 16 : kNowhere;
        to = r * (DP * 2) + ((c ^ spread<DP>(r)) << 4);
    }
    __device__ __forceinline__ void go_to(const char *base, int row, int rows, int dim) {
        at = base + (long long)row * row_bytes;
        left = (long long)(rows - row - 1) * row_bytes + dim * 2;
    }
    __device__ __forceinline__ void load(u32x4 (&x)[kChunks]) {
        const __amdgpu_buffer_rsrc_t w = window(at, left);
#pragma unroll
        for (int i = 0; i < kChunks; i++) x[i] = window_chunk(w, from + i * kStep * row_bytes);
        at += (long long)N * row_bytes;
        left -= (long long)N * row_bytes;
    }
    __device__ __forceinline__ void store(unsigned tile, const u32x4 (&x)[kChunks]) const {  // (kStep is a multiple of 16 rows, over which the spread repeats)
        typedef __attribute__((address_space(3))) u32x4 chunk;
#pragma unroll
        for (int i = 0; i < kChunks; i++) *(chunk *)(uintptr_t)(tile + to + i * kStep * DP * 2) = x[i];
    }
    __device__ __forceinline__ void clear(unsigned tile) const {
        u32x4 x[kChunks];
#pragma unroll
        for (int i = 0; i < kChunks; i++) x[i] = u32x4{0, 0, 0, 0};
        store(tile, x);
    }
};

// B = eight values 16 kk + 8 (l / 32) .. of one row, zeros where the row is none or behind dim
template <class E> __device__ __forceinline__ typename Vec8<E>::type row_chunk(const E *row, bool in, int kk, int dim, int lane) {
    int c = 16 * kk + 8 * (lane >> 5);
    u32x4 x = {0, 0, 0, 0};
    if (in && c < dim) x = *(const u32x4 *)(row + c);
    return as8<E>(x);
}

// A row's output, O^T in the layout of the matrix instruction's result, times `by`.
template <class E, int DP> __device__ __forceinline__ void write_row(const f32x16 (&o)[DP / 32], float by, E *out, int dim, int half) {
#pragma unroll
    for (int i = 0; i < DP / 32; i++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
            int c = 32 * i + 8 * r + 4 * half;
            if (c >= dim) continue;
            typename Vec4<E>::type x;
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = (E)(o[i][4 * r + e] * by);
            *(typename Vec4<E>::type *)(out + c) = x;
        }
}

// Four wavefronts' maxima, sums and outputs of the same 32 rows joined at the largest of their maxima: `top` and `sum` in all,
// the output in the first one's o.  The block's LDS from `lds` on (DP 256 bytes) is free for it behind the first barrier.
struct Joined { float top, sum; };
template <int DP> __device__ __forceinline__ Joined join_wavefronts(f32x16 (&o)[DP / 32], float m, float l, char *lds, float (&wave_m)[4][32], float (&wave_l)[4][32], int wave, int lane) {
    constexpr int kOut = DP / 32;
    const int half = lane >> 5, r31 = lane & 31;
    l = halves_sum(l);
    if (half == 0) wave_m[wave][lane] = m, wave_l[wave][lane] = l;
    __syncthreads();
    const float top = fmaxf(fmaxf(wave_m[0][r31], wave_m[1][r31]), fmaxf(wave_m[2][r31], wave_m[3][r31]));
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; w++) sum += wave_l[w][r31] * exp2_fast(wave_m[w][r31] - top);
    const float shrink = exp2_fast(m - top);
#pragma unroll
    for (int i = 0; i < kOut; i++) o[i] *= shrink;
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    f32x4 *box = (f32x4 *)lds;  // [wavefront][DP / 4][32 rows] (the tiles are read)
#pragma unroll
    for (int round = 2; round > 0; round >>= 1) {
        if (wave >= round && wave < 2 * round) {
#pragma unroll
            for (int i = 0; i < kOut; i++)
#pragma unroll
                for (int r = 0; r < 4; r++)
                    box[((wave - round) * (DP / 4) + 8 * i + 2 * r + half) * 32 + r31] = f32x4{o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
        }
        __syncthreads();
        if (wave < round) {
#pragma unroll
            for (int i = 0; i < kOut; i++)
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    f32x4 x = box[(wave * (DP / 4) + 8 * i + 2 * r + half) * 32 + r31];
#pragma unroll
                    for (int e = 0; e < 4; e++) o[i][4 * r + e] += x[e];
                }
        }
        __syncthreads();
    }
    return Joined{top, sum};
}

logoskg_status attend_args(const logoskg_attention *a, AttArgs *o, const char *call);

}  // namespace lkg
