// Arguments and tiles that the forward and the backward of the attention share.
#pragma once

#include "reading.h"

namespace lkg {

constexpr int kAttThreads = 256;  // four wavefronts
constexpr int kAttRowsShift = 7;  // a block's rows: 4 x 32
constexpr int kAttRows = 1 << kAttRowsShift;
constexpr long long kMostRows = (1ll << 31) - (1 << 16);  // of a batch: places in a document are 32-bit, with room for a tile
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
    float *delta;      // [num_rows][heads] sum of dout out
    float *bias_part;  // [blocks of the dq kernel][heads][num_buckets]
    float scale;
    float slope;       // with a cap: 4 scale, of scale (1 - tanh^2) = 4 scale r (1 - r), r = 1 / (2^(z k) + 1)
    long long row_blocks, key_blocks;
};

struct AttDoc {  // a document: where its rows and keys begin, and how many there are
    long long row0, key0;
    int rows, keys, prefix;
    // keys that row i sees: the first seen(i)
    __device__ __forceinline__ int seen(int i, int causal) const {
        if (!causal) return keys;
        int n = i + keys - rows + 1;  // (rows and keys below 2^31)
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

__device__ const u32x4 kZeroChunk = {0, 0, 0, 0};

// Reads rows [r0, r0 + N) of a ragged array's head (row strides in elements) into registers, N x DP values over the block's
// threads, zeros outside [0, rows) and behind dim.
template <int N, int DP> struct TileLoad {
    static constexpr int kChunks = N * DP / 8 / kAttThreads;
    u32x4 x[kChunks];
    __device__ __forceinline__ void load(const void *base, long long row_stride, int r0, int rows, int dim, int tid) {
#pragma unroll
        for (int i = 0; i < kChunks; i++) {
            int at = i * kAttThreads + tid, r = r0 + at / (DP / 8), c = at % (DP / 8);
            bool in = r < rows && c * 8 < dim;
            x[i] = in ? *(const u32x4 *)((const char *)base + (r * row_stride + c * 8) * 2) : u32x4{0, 0, 0, 0};
        }
    }
    __device__ __forceinline__ void store(char *tile, int tid) const {
#pragma unroll
        for (int i = 0; i < kChunks; i++) {
            int at = i * kAttThreads + tid, r = at / (DP / 8), c = at % (DP / 8);
            *(u32x4 *)(tile + r * (DP * 2) + ((c ^ spread<DP>(r)) << 4)) = x[i];
        }
    }
};

// B = eight values 16 kk + 8 (l / 32) .. of one row, zeros where the row is none or behind dim
template <class E> __device__ __forceinline__ typename Vec8<E>::type row_chunk(const E *row, bool in, int kk, int dim, int lane) {
    int c = 16 * kk + 8 * (lane >> 5);
    u32x4 x = {0, 0, 0, 0};
    if (in && c < dim) x = *(const u32x4 *)(row + c);
    return as8<E>(x);
}

logoskg_status attend_args(const logoskg_attention *a, AttArgs *o, const char *call);

template <class F> logoskg_status allow_lds(F *kernel, size_t bytes) {
    if (bytes > (64 << 10)) LKG_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    return LOGOSKG_OK;
}

}  // namespace lkg
