// Gradients of the attention of a ragged batch (logoskg_attend_backward).
//
// With p = 2^(y - lse), dP = dO V^T and delta = sum of dO O of a row (= sum of p dP), the gradient of the score y is
// dy = p (dP - delta), that of the product z: dz = dy scale (1 - tanh^2); dV = p^T dO, dK = dz^T Q, dQ = dz K, and a
// bucket's bias gets the sum of its dy.  Two kernels make p and dP again, one that keeps keys in registers and passes over
// the rows that see them (dK, dV), one that keeps rows and passes over their keys (dQ, biases): seven products for five, and
// in return no sum depends on the order in which blocks arrive, and none is kept in memory in between.
#include "attend.h"

namespace lkg {

// delta[row][head]: 16 lanes per (row, head), 8 values each
template <class E> __global__ __launch_bounds__(256) void k_att_delta(AttArgs a) {
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) >> 4;
    const int c = (threadIdx.x & 15) * 8;
    float sum = 0.f;
    const bool in = at < a.num_rows * a.heads;
    if (in && c < a.dim) {
        typename Vec8<E>::type x = as8<E>(*(const u32x4 *)((const E *)a.out + at * a.dim + c));
        typename Vec8<E>::type y = as8<E>(*(const u32x4 *)((const E *)a.dout + at * a.dim + c));
#pragma unroll
        for (int i = 0; i < 8; i++) sum = __builtin_fmaf((float)x[i], (float)y[i], sum);
    }
#pragma unroll
    for (int s = 8; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
    if (in && c == 0) a.delta[at] = sum;
}

// ---------------------------------------------------------------- dK, dV
// One block: 128 keys of (document, key head), 32 per wavefront, key = lane, K and V in registers as the B of S = Q K^T and
// dP = dO V^T.  Rows (all heads of the group) pass in tiles of 64 through LDS, where they are read by rows for these two
// products and by columns for dV^T += dO^T p and dK^T += Q^T dz.
constexpr int kGradRows = 64;

struct RowInfo {  // of a row in LDS
    float lse, delta;  // lse in units of log 2, +infinite for rows that see nothing: p = 0
    int seen, pos;
};

template <class E, int DP, bool CAP, bool BIAS>
__global__ __launch_bounds__(kAttThreads, 1) void k_att_dkdv(AttArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int kTile = kGradRows * DP * 2, kSteps = DP / 16, kOut = DP / 32, kChunks = kGradRows * DP / 8 / kAttThreads;
    char *tiles = lds;  // [2][Q, dO]
    RowInfo *info = (RowInfo *)(lds + 4 * kTile);          // [2][kGradRows]
    int *row_table = (int *)(info + 2 * kGradRows);        // [2][kGradRows] where the row's head begins in the table
    float *table = (float *)(row_table + 2 * kGradRows);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int head = blockIdx.x % a.kv_heads;
    const long long block = blockIdx.x / a.kv_heads;
    const int d = document_of(a.k_off, a.num_docs, a.num_keys, 1, kAttRowsShift, block, lane);
    const AttDoc doc = att_doc(a, d);
    const long long kb = (block - first_block(a.k_off, d, a.num_keys, 1, kAttRowsShift)) << kAttRowsShift;
    if (kb >= doc.keys || kb < 0) return;

    const int G = a.group, places = 2 * a.score.max_distance + 1, magic = (65536 + G - 1) / G;
    const int key = (int)kb + wave * 32 + (lane & 31);
    const bool mine = key < doc.keys;
    const E *krow = (const E *)a.k + (doc.key0 + key) * a.k_row + (long long)head * a.k_head;
    const E *vrow = (const E *)a.v + (doc.key0 + key) * a.v_row + (long long)head * a.v_head;
    typename Vec8<E>::type k[kSteps], v[kSteps];
#pragma unroll
    for (int kk = 0; kk < kSteps; kk++) {
        k[kk] = row_chunk<E>(krow, mine, kk, a.dim, lane);
        v[kk] = row_chunk<E>(vrow, mine, kk, a.dim, lane);
    }
    const int k_pos = !mine ? 0 : a.k_pos ? a.k_pos[doc.key0 + key] : key;
    if (BIAS) bias_to_lds<E>(table, a.score, head * G, G, tid, kAttThreads);

    f32x16 dk[kOut], dv[kOut];
#pragma unroll
    for (int i = 0; i < kOut; i++) dk[i] = zero16(), dv[i] = zero16();

    const int kend = doc.keys < kb + kAttRows ? doc.keys : (int)kb + kAttRows;
    int from = 0;  // first row that sees one of the keys
    if (a.causal && kb >= doc.prefix) {
        long long i = kb - ((long long)doc.keys - doc.rows);
        from = i < 0 ? 0 : i > doc.rows ? doc.rows : (int)i;
    }
    const long long vrows = (long long)doc.rows * G;
    const long long v0 = (long long)from * G;
    const int tiles_n = (int)((vrows - v0 + kGradRows - 1) / kGradRows);

    u32x4 qx[kChunks], ox[kChunks];
    RowInfo my_info;
    int my_table = 0;
    auto fetch = [&](int t) {
        const long long base = v0 + (long long)t * kGradRows;
        const int i0 = (int)(base / G), g0 = (int)(base - (long long)i0 * G);
#pragma unroll
        for (int i = 0; i < kChunks; i++) {
            int at = i * kAttThreads + tid, r = at / (DP / 8), c = (at % (DP / 8)) * 8;
            int up = ((g0 + r) * magic) >> 16, row = i0 + up, g = g0 + r - up * G;
            bool in = row < doc.rows && c < a.dim;
            const E *qp = (const E *)a.q + (doc.row0 + row) * a.q_row + (long long)(head * G + g) * a.q_head + c;
            const E *op = (const E *)a.dout + ((doc.row0 + row) * a.heads + head * G + g) * a.dim + c;
            qx[i] = in ? *(const u32x4 *)qp : u32x4{0, 0, 0, 0};
            ox[i] = in ? *(const u32x4 *)op : u32x4{0, 0, 0, 0};
        }
        if (tid < kGradRows) {
            int up = ((g0 + tid) * magic) >> 16, row = i0 + up, g = g0 + tid - up * G;
            bool in = row < doc.rows;
            long long at = in ? (doc.row0 + row) * a.heads + head * G + g : 0;
            float lse = in ? a.lse[at] : -INFINITY;
            my_info.lse = lse == -INFINITY ? INFINITY : lse * kLog2e;
            my_info.delta = in ? a.delta[at] : 0.f;
            my_info.seen = in ? doc.seen(row, a.causal) : 0;
            my_info.pos = !in ? 0 : a.q_pos ? a.q_pos[doc.row0 + row] : row + doc.keys - doc.rows;
            my_table = g * places;
        }
    };
    if (tiles_n > 0) fetch(0);
    for (int t = 0; t < tiles_n; t++) {
        char *qt = tiles + (t & 1) * 2 * kTile, *ot = qt + kTile;
        const RowInfo *inf = info + (t & 1) * kGradRows;
        const int *rt = row_table + (t & 1) * kGradRows;
#pragma unroll
        for (int i = 0; i < kChunks; i++) {
            int at = i * kAttThreads + tid, r = at / (DP / 8), c = at % (DP / 8), place = r * (DP * 2) + ((c ^ spread<DP>(r)) << 4);
            *(u32x4 *)(qt + place) = qx[i];
            *(u32x4 *)(ot + place) = ox[i];
        }
        if (tid < kGradRows) {
            info[(t & 1) * kGradRows + tid] = my_info;
            row_table[(t & 1) * kGradRows + tid] = my_table;
        }
        __syncthreads();
        if (t + 1 < tiles_n) fetch(t + 1);
        const bool edge = doc.seen((int)((v0 + (long long)t * kGradRows) / G), a.causal) < kend;

#pragma unroll
        for (int u = 0; u < 2; u++) {
            f32x16 s = zero16(), dp = zero16();
#pragma unroll
            for (int kk = 0; kk < kSteps; kk++) {
                s = mfma(tile_rows<E, DP>(qt, 32 * u, kk, lane), k[kk], s);
                dp = mfma(tile_rows<E, DP>(ot, 32 * u, kk, lane), v[kk], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; r++) {
                const int at = 32 * u + 8 * (r / 4) + 4 * half + r % 4;
                const RowInfo ri = inf[at];
                float y, w = 0.f;
                if (CAP) {
                    w = rcp_fast(exp2_fast(s[r] * a.score.k) + 1.f);
                    y = __builtin_fmaf(-2.f * a.score.c, w, a.score.c);
                } else y = s[r] * a.score.k;
                if (BIAS) y += table[rt[at] + distance_place(k_pos, ri.pos, a.score.max_distance)];
                float p = exp2_fast(y - ri.lse);
                if (edge) p = key < ri.seen ? p : 0.f;
                float dy = p * (dp[r] - ri.delta);
                if (edge) dy = key < ri.seen ? dy : 0.f;
                s[r] = p;
                dp[r] = CAP ? dy * a.slope * (w * (1.f - w)) : dy * a.scale;
            }
            typename Vec8<E>::type p0 = rounded8<E, 0>(s), p1 = rounded8<E, 1>(s), z0 = rounded8<E, 0>(dp), z1 = rounded8<E, 1>(dp);
#pragma unroll
            for (int i = 0; i < kOut; i++) {
                dv[i] = mfma(tile_columns<E, DP>(ot, 32 * u, i, lane), p0, dv[i]);
                dv[i] = mfma(tile_columns<E, DP>(ot, 32 * u + 16, i, lane), p1, dv[i]);
                dk[i] = mfma(tile_columns<E, DP>(qt, 32 * u, i, lane), z0, dk[i]);
                dk[i] = mfma(tile_columns<E, DP>(qt, 32 * u + 16, i, lane), z1, dk[i]);
            }
        }
    }
    if (!mine) return;
    const long long place = ((doc.key0 + key) * a.kv_heads + head) * a.dim;
#pragma unroll
    for (int i = 0; i < kOut; i++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
            int c = 32 * i + 8 * r + 4 * half;
            if (c >= a.dim) continue;
            typename Vec4<E>::type x, y;
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = (E)dk[i][4 * r + e], y[e] = (E)dv[i][4 * r + e];
            *(typename Vec4<E>::type *)((E *)a.dk + place + c) = x;
            *(typename Vec4<E>::type *)((E *)a.dv + place + c) = y;
        }
}

// ---------------------------------------------------------------- dQ, biases
// One block: 128 rows as in the forward, keys in tiles of 32.  A lane adds its dy to its own column of [buckets][64] in LDS:
// no two lanes share an address, so the sums have an order.
constexpr int kGradKeys = 32;

template <class E, int DP, bool CAP, bool BIAS>
__global__ __launch_bounds__(kAttThreads, 2) void k_att_dq(AttArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int kTile = kGradKeys * DP * 2, kSteps = DP / 16, kOut = DP / 32;
    char *tiles = lds;                               // [2][K, V]
    int *kpos = (int *)(lds + 4 * kTile);            // [2][kGradKeys]
    float *sums = (float *)(kpos + 2 * kGradKeys);   // [4 wavefronts][num_buckets][64]
    const int nb = a.score.num_buckets, M = a.score.max_distance, places = 2 * M + 1, G = a.group;
    int *column = (int *)(sums + (BIAS ? 4 * nb * 64 : 0));  // [places] where a distance's bucket begins
    float *table = (float *)(column + (BIAS ? places : 0));
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int head = blockIdx.x % a.kv_heads;
    const long long block = a.row_blocks - 1 - blockIdx.x / a.kv_heads;
    const int d = document_of(a.q_off, a.num_docs, a.num_rows, G, kAttRowsShift, block, lane);
    const AttDoc doc = att_doc(a, d);
    const long long first = (block - first_block(a.q_off, d, a.num_rows, G, kAttRowsShift)) << kAttRowsShift;
    const long long vrows = (long long)doc.rows * G;
    float *part = BIAS ? a.bias_part + (block * a.heads + head * G) * nb : nullptr;
    if (first >= vrows || first < 0) {
        if (BIAS)
            for (int i = tid; i < G * nb; i += kAttThreads) part[i] = 0.f;
        return;
    }

    const long long vr = first + wave * 32 + (lane & 31);
    const bool mine = vr < vrows;
    const int row = mine ? (int)(vr / G) : 0, g = mine ? (int)(vr % G) : 0, h = head * G + g;
    const int seen = mine ? doc.seen(row, a.causal) : 0;
    const int least = doc.seen((int)(first / G), a.causal);
    const long long last_v = first + kAttRows < vrows ? first + kAttRows - 1 : vrows - 1;
    const int most = doc.seen((int)(last_v / G), a.causal);
    const long long place = (doc.row0 + row) * a.heads + h;
    const E *qrow = (const E *)a.q + (doc.row0 + row) * a.q_row + (long long)h * a.q_head;
    const E *orow = (const E *)a.dout + place * a.dim;
    typename Vec8<E>::type q[kSteps], o[kSteps];
#pragma unroll
    for (int kk = 0; kk < kSteps; kk++) {
        q[kk] = row_chunk<E>(qrow, mine, kk, a.dim, lane);
        o[kk] = row_chunk<E>(orow, mine, kk, a.dim, lane);
    }
    float lse = mine ? a.lse[place] : -INFINITY;
    lse = lse == -INFINITY ? INFINITY : lse * kLog2e;
    const float delta = mine ? a.delta[place] : 0.f;
    const int q_pos = !mine ? 0 : a.q_pos ? a.q_pos[doc.row0 + row] : row + doc.keys - doc.rows;
    const float *my_table = table + g * places;
    float *my_sums = sums + wave * nb * 64 + lane;
    if (BIAS) {
        bias_to_lds<E>(table, a.score, head * G, G, tid, kAttThreads);
        for (int i = tid; i < places; i += kAttThreads) {
            int b = a.score.buckets[i];
            column[i] = (b < 0 ? 0 : b >= nb ? nb - 1 : b) * 64;
        }
        for (int i = tid; i < 4 * nb * 64; i += kAttThreads) sums[i] = 0.f;
    }
    const char *kbase = (const char *)a.k + (doc.key0 * a.k_row + (long long)head * a.k_head) * 2;
    const char *vbase = (const char *)a.v + (doc.key0 * a.v_row + (long long)head * a.v_head) * 2;
    f32x16 dq[kOut];
#pragma unroll
    for (int i = 0; i < kOut; i++) dq[i] = zero16();

    TileLoad<kGradKeys, DP> kload, vload;
    int kp = 0;
    auto fetch = [&](int t) {
        kload.load(kbase, a.k_row, t * kGradKeys, doc.keys, a.dim, tid);
        vload.load(vbase, a.v_row, t * kGradKeys, doc.keys, a.dim, tid);
        int j = t * kGradKeys + tid;
        if (BIAS && tid < kGradKeys) kp = a.k_pos && j < doc.keys ? a.k_pos[doc.key0 + j] : j;
    };
    const int tiles_n = (most + kGradKeys - 1) / kGradKeys;
    if (tiles_n > 0) fetch(0);
    for (int t = 0; t < tiles_n; t++) {
        char *kt = tiles + (t & 1) * 2 * kTile, *vt = kt + kTile;
        int *kpt = kpos + (t & 1) * kGradKeys;
        kload.store(kt, tid);
        vload.store(vt, tid);
        if (BIAS && tid < kGradKeys) kpt[tid] = kp;
        __syncthreads();
        if (t + 1 < tiles_n) fetch(t + 1);
        f32x16 s = zero16(), dp = zero16();
#pragma unroll
        for (int kk = 0; kk < kSteps; kk++) {
            s = mfma(tile_rows<E, DP>(kt, 0, kk, lane), q[kk], s);
            dp = mfma(tile_rows<E, DP>(vt, 0, kk, lane), o[kk], dp);
        }
        const bool edge = (t + 1) * kGradKeys > least;
#pragma unroll
        for (int r = 0; r < 16; r++) {
            const int at = 8 * (r / 4) + 4 * half + r % 4;
            float y, w = 0.f;
            if (CAP) {
                w = rcp_fast(exp2_fast(s[r] * a.score.k) + 1.f);
                y = __builtin_fmaf(-2.f * a.score.c, w, a.score.c);
            } else y = s[r] * a.score.k;
            int apart = 0;
            if (BIAS) {
                apart = distance_place(kpt[at], q_pos, M);
                y += my_table[apart];
            }
            float dy = exp2_fast(y - lse) * (dp[r] - delta);
            if (edge) dy = t * kGradKeys + at < seen ? dy : 0.f;
            if (BIAS) __hip_atomic_fetch_add(my_sums + column[apart], dy, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            dp[r] = CAP ? dy * a.slope * (w * (1.f - w)) : dy * a.scale;
        }
        typename Vec8<E>::type z0 = rounded8<E, 0>(dp), z1 = rounded8<E, 1>(dp);
#pragma unroll
        for (int i = 0; i < kOut; i++) {
            dq[i] = mfma(tile_columns<E, DP>(kt, 0, i, lane), z0, dq[i]);
            dq[i] = mfma(tile_columns<E, DP>(kt, 16, i, lane), z1, dq[i]);
        }
    }
    if (mine) {
        E *out = (E *)a.dq + place * a.dim;
#pragma unroll
        for (int i = 0; i < kOut; i++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
                int c = 32 * i + 8 * r + 4 * half;
                if (c >= a.dim) continue;
                typename Vec4<E>::type x;
#pragma unroll
                for (int e = 0; e < 4; e++) x[e] = (E)dq[i][4 * r + e];
                *(typename Vec4<E>::type *)(out + c) = x;
            }
    }
    if (BIAS) {  // the columns of a head's rows, rotated by the bucket so that neighbouring threads read other banks
        __syncthreads();
        for (int i = tid; i < G * nb; i += kAttThreads) {
            const int gg = i / nb, b = i % nb;
            float sum = 0.f;
            for (int w = 0; w < 4; w++)
                for (int e = 0; e < 64; e++) {
                    int l = (e + b) & 63;
                    if ((int)((first + w * 32 + (l & 31)) % G) == gg) sum += sums[(w * nb + b) * 64 + l];
                }
            part[i] = sum;
        }
    }
}

// dbias[head][bucket] = the blocks' parts, one after the other in 1024 / num_buckets strands
template <class E> __global__ __launch_bounds__(1024) void k_att_dbias(AttArgs a) {
    __shared__ float strand[1024];
    const int nb = a.score.num_buckets, h = blockIdx.x, strands = 1024 / nb, b = threadIdx.x % nb, s = threadIdx.x / nb;
    float sum = 0.f;
    if (s < strands)
        for (long long i = s; i < a.row_blocks; i += strands) sum += a.bias_part[(i * a.heads + h) * nb + b];
    strand[threadIdx.x] = sum;
    __syncthreads();
    if (s != 0) return;
    for (int i = 1; i < strands; i++) sum += strand[i * nb + b];
    ((E *)a.dbias)[h * nb + b] = (E)sum;
}

static int64_t delta_bytes(const AttArgs &a) { return (a.num_rows * a.heads * 4 + 15) / 16 * 16; }
static int64_t backward_bytes(const AttArgs &a) {
    return delta_bytes(a) + (a.score.bias ? a.row_blocks * a.heads * (int64_t)a.score.num_buckets * 4 : 0);
}

template <class E, int DP, bool CAP, bool BIAS> static logoskg_status launch_backward(const AttArgs &a, hipStream_t st) {
    const size_t table = BIAS ? (size_t)a.group * (2 * a.score.max_distance + 1) * 4 : 0;
    if (a.num_keys) {
        size_t bytes = 4 * kGradRows * DP * 2 + 2 * kGradRows * (sizeof(RowInfo) + 4) + table;
        LKG_TRY(allow_lds(k_att_dkdv<E, DP, CAP, BIAS>, bytes));
        k_att_dkdv<E, DP, CAP, BIAS><<<dim3((unsigned)(a.key_blocks * a.kv_heads)), kAttThreads, bytes, st>>>(a);
        LKG_HIP(hipGetLastError());
    }
    if (a.num_rows) {
        size_t bytes = 4 * kGradKeys * DP * 2 + 2 * kGradKeys * 4 + table;
        if (BIAS) bytes += (size_t)4 * a.score.num_buckets * 64 * 4 + (size_t)(2 * a.score.max_distance + 1) * 4;
        LKG_TRY(allow_lds(k_att_dq<E, DP, CAP, BIAS>, bytes));
        k_att_dq<E, DP, CAP, BIAS><<<dim3((unsigned)(a.row_blocks * a.kv_heads)), kAttThreads, bytes, st>>>(a);
        LKG_HIP(hipGetLastError());
    }
    return LOGOSKG_OK;
}

template <class E> static logoskg_status backward(const AttArgs &a, hipStream_t st) {
    if (a.num_rows) {
        long long n = a.num_rows * a.heads;
        k_att_delta<E><<<dim3((unsigned)((n + 15) / 16)), 256, 0, st>>>(a);
        LKG_HIP(hipGetLastError());
    }
    const bool cap = a.score.c > 0, bias = a.score.bias != nullptr, wide = a.dim > 64;
    if (wide) LKG_TRY((cap ? bias ? launch_backward<E, 128, true, true>(a, st) : launch_backward<E, 128, true, false>(a, st)
                           : bias ? launch_backward<E, 128, false, true>(a, st) : launch_backward<E, 128, false, false>(a, st)));
    else LKG_TRY((cap ? bias ? launch_backward<E, 64, true, true>(a, st) : launch_backward<E, 64, true, false>(a, st)
                      : bias ? launch_backward<E, 64, false, true>(a, st) : launch_backward<E, 64, false, false>(a, st)));
    if (bias) {
        k_att_dbias<E><<<dim3((unsigned)a.heads), 1024, 0, st>>>(a);  // (no row: no parts, zeros)
        LKG_HIP(hipGetLastError());
    }
    return LOGOSKG_OK;
}

}  // namespace lkg

using namespace lkg;

extern "C" int64_t logoskg_attend_backward_bytes(const logoskg_attention *in) {
    AttArgs a;
    return attend_args(in, &a, "logoskg_attend_backward_bytes") == LOGOSKG_OK ? backward_bytes(a) : -1;
}

extern "C" logoskg_status logoskg_attend_backward(const logoskg_attention *in, const logoskg_attention_grad *g) {
    AttArgs a;
    LKG_TRY(attend_args(in, &a, "logoskg_attend_backward"));
    const char *why = nullptr;
    if (!g || g->struct_size != sizeof(logoskg_attention_grad)) why = "struct_size of the gradients";
    else if (a.num_rows && (!g->dout || !g->dq)) why = "dout or dq is NULL";
    else if (a.num_keys && (!g->dk || !g->dv)) why = "dk or dv is NULL";
    else if (a.score.bias && !g->dbias) why = "dbias is NULL";
    else if (((uintptr_t)g->dout | (uintptr_t)g->dq | (uintptr_t)g->dk | (uintptr_t)g->dv | (uintptr_t)g->workspace) & 15) why = "an array is not 16-byte aligned";
    if (why) { set_error("logoskg_attend_backward: %s", why); return LOGOSKG_EINVAL; }
    if (g->workspace_bytes < backward_bytes(a) || (backward_bytes(a) && !g->workspace)) {
        set_error("logoskg_attend_backward: the workspace has %lld of %lld bytes", (long long)g->workspace_bytes, (long long)backward_bytes(a));
        return LOGOSKG_ERANGE;
    }
    a.dout = g->dout; a.dq = g->dq; a.dk = g->dk; a.dv = g->dv; a.dbias = g->dbias;
    a.delta = (float *)g->workspace;
    a.bias_part = (float *)((char *)g->workspace + delta_bytes(a));
    a.key_blocks = (a.num_keys >> kAttRowsShift) + a.num_docs;
    if (a.key_blocks * a.kv_heads >= (1ll << 31) || (a.num_rows * a.heads + 15) / 16 >= (1ll << 31)) { set_error("logoskg_attend_backward: too many rows"); return LOGOSKG_EINVAL; }
    if (a.num_rows == 0) a.row_blocks = 0;
    LKG_HIP(hipSetDevice(in->device));
    return in->dtype == LOGOSKG_BF16 ? backward<bf16>(a, (hipStream_t)in->stream) : backward<fp16>(a, (hipStream_t)in->stream);
}
