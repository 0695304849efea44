// Attention of a ragged batch with capped scores, a learned distance bias and a prefix + causal mask (logoskg_attend).
#include "attend.h"

namespace lkg {

// One block: 128 rows of (document, key head), where a row is a (row of q, head of the group) pair, so that the heads that
// share a key head share its tiles.  A wavefront holds 32 rows: lane l works for row l % 32 and half of the keys, so a row's
// maximum and sum are its own registers and one exchange with the other half.  Keys pass in tiles of 64 through two
// buffers in LDS; S^T = K Q^T, p = 2^(y - m), O^T += V^T P^T with m the running maximum.
constexpr int kKeys = 64;

template <class E, int DP, bool CAP, bool BIAS>
__global__ __launch_bounds__(kAttThreads, 2) void k_attend(AttArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int kTile = kKeys * DP * 2, kSteps = DP / 16, kOut = DP / 32;
    char *tiles = lds;                                 // [2][K, V]
    int *kpos = (int *)(lds + 4 * kTile);              // [2][kKeys]
    float *table = (float *)(lds + 4 * kTile + 2 * kKeys * 4);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int head = blockIdx.x % a.kv_heads;
    const long long block = a.row_blocks - 1 - blockIdx.x / a.kv_heads;  // the last rows of a document see most: first
    const int d = document_of(a.q_off, a.num_docs, a.num_rows, a.group, kAttRowsShift, block, lane);
    const AttDoc doc = att_doc(a, d);
    const long long first = (block - first_block(a.q_off, d, a.num_rows, a.group, kAttRowsShift)) << kAttRowsShift;
    const long long vrows = (long long)doc.rows * a.group;
    if (first >= vrows || first < 0) return;

    const long long vr = first + wave * 32 + (lane & 31);
    const bool mine = vr < vrows;
    const int row = mine ? (int)(vr / a.group) : 0, g = mine ? (int)(vr % a.group) : 0;
    const int seen = mine ? doc.seen(row, a.causal) : 0;
    // of the block's first and last row
    const int least = doc.seen((int)(first / a.group), a.causal);
    const long long last_v = first + kAttRows < vrows ? first + kAttRows - 1 : vrows - 1;
    const int most = doc.seen((int)(last_v / a.group), a.causal);

    const int h = head * a.group + g;
    const E *qrow = (const E *)a.q + (doc.row0 + row) * a.q_row + (long long)h * a.q_head;
    typename Vec8<E>::type q[kSteps];
#pragma unroll
    for (int kk = 0; kk < kSteps; kk++) q[kk] = row_chunk<E>(qrow, mine, kk, a.dim, lane);
    const int q_pos = !mine ? 0 : a.q_pos ? a.q_pos[doc.row0 + row] : row + doc.keys - doc.rows;
    const int M = a.score.max_distance;
    const float *my_table = table + g * (2 * M + 1);
    if (BIAS) bias_to_lds<E>(table, a.score, head * a.group, a.group, tid, kAttThreads);

    const char *kbase = (const char *)a.k + (doc.key0 * a.k_row + (long long)head * a.k_head) * 2;
    const char *vbase = (const char *)a.v + (doc.key0 * a.v_row + (long long)head * a.v_head) * 2;
    f32x16 o[kOut];
#pragma unroll
    for (int i = 0; i < kOut; i++) o[i] = zero16();
    float m = kLowest, l = 0.f;

    TileLoad<kKeys, DP> kload, vload;
    int kp = 0;
    const int tiles_n = (most + kKeys - 1) / kKeys;
    auto fetch = [&](int t) {
        kload.load(kbase, a.k_row, t * kKeys, doc.keys, a.dim, tid);
        vload.load(vbase, a.v_row, t * kKeys, doc.keys, a.dim, tid);
        int j = t * kKeys + tid;
        if (BIAS && tid < kKeys) kp = a.k_pos && j < doc.keys ? a.k_pos[doc.key0 + j] : j;
    };
    if (tiles_n > 0) fetch(0);
    for (int t = 0; t < tiles_n; t++) {
        char *kt = tiles + (t & 1) * 2 * kTile, *vt = kt + kTile;
        int *kpt = kpos + (t & 1) * kKeys;
        kload.store(kt, tid);
        vload.store(vt, tid);
        if (BIAS && tid < kKeys) kpt[tid] = kp;
        __syncthreads();  // (the buffer's last readers are behind the barrier of the round before)
        if (t + 1 < tiles_n) fetch(t + 1);

        f32x16 s[2];
#pragma unroll
        for (int u = 0; u < 2; u++) {
            s[u] = zero16();
#pragma unroll
            for (int kk = 0; kk < kSteps; kk++) s[u] = mfma(tile_rows<E, DP>(kt, 32 * u, kk, lane), q[kk], s[u]);
        }
        const bool edge = (t + 1) * kKeys > least;  // some row does not see all of the tile
        float top = kLowest;
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int r = 0; r < 16; r++) {
                float y;
                if (CAP) y = __builtin_fmaf(-2.f * a.score.c, rcp_fast(exp2_fast(s[u][r] * a.score.k) + 1.f), a.score.c);
                else y = s[u][r] * a.score.k;
                int at = 32 * u + 8 * (r / 4) + 4 * half + r % 4;
                if (BIAS) y += my_table[distance_place(kpt[at], q_pos, M)];
                if (edge) y = t * kKeys + at < seen ? y : -INFINITY;
                s[u][r] = y;
                top = fmaxf(top, y);
            }
        top = halves_max(top);
        if (wave_any(top > m)) {
            float up = fmaxf(m, top), shrink = exp2_fast(m - up);
            m = up;
            l *= shrink;
#pragma unroll
            for (int i = 0; i < kOut; i++) o[i] *= shrink;
        }
#pragma unroll
        for (int u = 0; u < 2; u++) {
#pragma unroll
            for (int r = 0; r < 16; r++) {
                s[u][r] = exp2_fast(s[u][r] - m);
                l += s[u][r];
            }
            typename Vec8<E>::type p0 = rounded8<E, 0>(s[u]), p1 = rounded8<E, 1>(s[u]);
#pragma unroll
            for (int i = 0; i < kOut; i++) {
                o[i] = mfma(tile_columns<E, DP>(vt, 32 * u, i, lane), p0, o[i]);
                o[i] = mfma(tile_columns<E, DP>(vt, 32 * u + 16, i, lane), p1, o[i]);
            }
        }
    }
    l = halves_sum(l);
    if (!mine) return;
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;  // (a NaN stays one)
    const long long place = (doc.row0 + row) * a.heads + h;
    E *out = (E *)a.out + place * a.dim;
#pragma unroll
    for (int i = 0; i < kOut; i++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
            int c = 32 * i + 8 * r + 4 * half;
            if (c >= a.dim) continue;
            typename Vec4<E>::type x;
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = (E)(o[i][4 * r + e] * inv);
            *(typename Vec4<E>::type *)(out + c) = x;
        }
    if (half == 0) a.lse[place] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

const char *bad_heads(int dtype, int heads, int kv_heads, int dim) {
    if (dtype != LOGOSKG_BF16 && dtype != LOGOSKG_F16) return "the type is neither LOGOSKG_BF16 nor LOGOSKG_F16";
    if (kv_heads < 1 || heads < kv_heads || heads % kv_heads != 0 || heads > 65535) return "heads is no multiple of kv_heads";
    if (heads / kv_heads > kMostGroup) return "more than 128 heads share a key head";
    if (dim < 8 || dim > 128 || dim % 8 != 0) return "dim is no multiple of 8 in [8, 128]";
    return nullptr;
}

const char *bad_score(const logoskg_score &s, int heads, int kv_heads) {
    if (!(s.cap >= 0.f) || s.cap > 3e38f || !(s.scale > -3e38f && s.scale < 3e38f)) return "scale or cap is no usable number";
    if (!s.bias) return nullptr;
    if (!s.buckets) return "a bias without buckets";
    if (s.num_buckets < 1 || s.num_buckets > LOGOSKG_MAX_BUCKETS) return "num_buckets outside [1, LOGOSKG_MAX_BUCKETS]";
    if (s.max_distance < 0 || s.max_distance > LOGOSKG_MAX_DISTANCE) return "max_distance outside [0, LOGOSKG_MAX_DISTANCE]";
    if ((long long)(heads / kv_heads) * (2 * s.max_distance + 1) > LOGOSKG_BIAS_PLACES) return "heads / kv_heads * (2 max_distance + 1) above LOGOSKG_BIAS_PLACES";
    return nullptr;
}

static bool odd_place(const void *p, long long s0, long long s1) { return ((uintptr_t)p & 15) || (s0 & 7) || (s1 & 7); }

logoskg_status attend_args(const logoskg_attention *a, AttArgs *o, const char *call) {
    if (!a || a->struct_size != sizeof(logoskg_attention)) { set_error("%s: struct_size", call); return LOGOSKG_EINVAL; }
    const char *why = bad_heads(a->dtype, a->heads, a->kv_heads, a->dim);
    if (!why) why = bad_score(a->score, a->heads, a->kv_heads);
    if (!why && (a->num_docs < 0 || a->num_rows < 0 || a->num_keys < 0 || a->num_rows >= kMostRows || a->num_keys >= kMostRows))
        why = "a count is negative or too large";
    if (!why && a->num_docs == 0 && (a->num_rows || a->num_keys)) why = "rows or keys without a document";
    if (!why && a->num_docs > 0 && (!a->q_off || !a->k_off)) why = "offsets are NULL";
    if (!why && a->num_rows && (!a->q || !a->out || !a->lse)) why = "q, out or lse is NULL";
    if (!why && a->num_keys && (!a->k || !a->v)) why = "k or v is NULL";
    if (!why && (odd_place(a->q, a->q_row, a->q_head) || odd_place(a->k, a->k_row, a->k_head) || odd_place(a->v, a->v_row, a->v_head) || odd_place(a->out, 0, 0)))
        why = "an array is not 16-byte aligned, or a stride no multiple of 8";
    if (why) { set_error("%s: %s", call, why); return LOGOSKG_EINVAL; }
    memset(o, 0, sizeof *o);
    o->num_docs = a->num_docs; o->heads = a->heads; o->kv_heads = a->kv_heads; o->group = a->heads / a->kv_heads;
    o->dim = a->dim; o->causal = a->causal; o->num_rows = a->num_rows; o->num_keys = a->num_keys;
    o->q_off = a->q_off; o->k_off = a->k_off; o->q = a->q; o->k = a->k; o->v = a->v;
    o->q_row = a->q_row; o->q_head = a->q_head; o->k_row = a->k_row; o->k_head = a->k_head; o->v_row = a->v_row; o->v_head = a->v_head;
    o->prefix = a->prefix; o->q_pos = a->q_pos; o->k_pos = a->k_pos;
    o->score = score_args(a->score);
    o->out = a->out; o->lse = a->lse;
    o->row_blocks = (a->num_rows * o->group >> kAttRowsShift) + a->num_docs;
    o->scale = a->score.scale;
    o->slope = 4.f * a->score.scale;
    if (o->row_blocks * a->kv_heads >= (1ll << 31)) { set_error("%s: too many rows", call); return LOGOSKG_EINVAL; }
    return LOGOSKG_OK;
}

template <class E, int DP, bool CAP, bool BIAS> static logoskg_status launch_attend(const AttArgs &a, hipStream_t st) {
    size_t bytes = 4 * kKeys * DP * 2 + 2 * kKeys * 4 + (BIAS ? (size_t)a.group * (2 * a.score.max_distance + 1) * 4 : 0);
    LKG_TRY(allow_lds(k_attend<E, DP, CAP, BIAS>, bytes));
    k_attend<E, DP, CAP, BIAS><<<dim3((unsigned)(a.row_blocks * a.kv_heads)), kAttThreads, bytes, st>>>(a);
    LKG_HIP(hipGetLastError());
    return LOGOSKG_OK;
}
template <class E, int DP> static logoskg_status launch_attend(const AttArgs &a, hipStream_t st) {
    bool cap = a.score.c > 0, bias = a.score.bias != nullptr;
    return cap ? bias ? launch_attend<E, DP, true, true>(a, st) : launch_attend<E, DP, true, false>(a, st)
               : bias ? launch_attend<E, DP, false, true>(a, st) : launch_attend<E, DP, false, false>(a, st);
}

}  // namespace lkg

using namespace lkg;

extern "C" logoskg_status logoskg_attend(const logoskg_attention *in) {
    AttArgs a;
    LKG_TRY(attend_args(in, &a, "logoskg_attend"));
    if (a.num_rows == 0) return LOGOSKG_OK;
    LKG_HIP(hipSetDevice(in->device));
    hipStream_t st = (hipStream_t)in->stream;
    if (in->dtype == LOGOSKG_BF16) return a.dim > 64 ? launch_attend<bf16, 128>(a, st) : launch_attend<bf16, 64>(a, st);
    return a.dim > 64 ? launch_attend<fp16, 128>(a, st) : launch_attend<fp16, 64>(a, st);
}
