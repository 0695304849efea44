// Few tokens of every query attend to the query's entity list, keys and values in a table by entity
// (logoskg_read_entities).
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

constexpr int kReadTile = 32;       // entries of a wavefront at a time
constexpr int kReadLeastShift = 7;  // four wavefronts, a tile each

// One block: 2^shift entries of a list, one key head, 32 rows (token, head of the group); its wavefronts take every fourth
// tile of 32 entries and join at the end.  The bytes of the entries are all that counts (a row of the matrix instructions
// may well be empty): keys go from memory into the registers that the instruction reads, values through the wavefront's
// own piece of LDS, where they are read by columns; no wavefront waits for another.
//
// Memory bounds it: 64 lists of up to 20,000 entities of a table of 407,000 (8 key heads of 128, float16) 597 us, 4.5 TB/s of the
// rows read, a copy's rate 4.85; 1,024 lists of up to 3,000 of 3 M (8 of 64, four tokens) 820 us, 3.9 TB/s: a key head's piece
// of a row is one line of 128 bytes.  One list of 900: 10 us and 4 for the join, both chains of loads.
template <class E, int DP, bool CAP, bool BIAS>
__global__ __launch_bounds__(256, 2) void k_read(ReadArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int kTile = kReadTile * DP * 2, kSteps = DP / 16, kOut = DP / 32, kRow = DP / 8;  // kRow: chunks of a row
    float *table = (float *)(lds + 4 * kTile);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    char *vt = lds + wave * kTile;
    const unsigned my_columns = columns_place<DP>(lane) + lds_place(vt);
    __shared__ int ids[4][kReadTile], hops[4][kReadTile];
    __shared__ float wave_m[4][32], wave_l[4][32];
    // the key heads of a block's entries one behind the other on one of the card's eight dies, which blocks take turns with:
    // their rows lie side by side
    const unsigned turn = blockIdx.x >> 3;
    const int head = turn % a.kv_heads;
    const long long block = (long long)(turn / a.kv_heads) * 8 + (blockIdx.x & 7);
    if (block >= a.blocks) return;
    const int d = document_of(a.off, a.num_queries, a.num_entries, 1, a.shift, block, lane);
    const long long b0 = first_block(a.off, d, a.num_entries, 1, a.shift);
    const long long e0 = taken_into(a.off[d], a.num_entries), e1 = taken_into(a.off[d + 1], a.num_entries);
    const long long len = e1 > e0 ? e1 - e0 : 0, from = (block - b0) << a.shift;
    if (from < 0 || (from > 0 && from >= len)) return;  // before the first list, or behind one (an empty list's first block writes its zeros)
    const bool alone = len <= (1ll << a.shift);
    const int n = (int)(len - from < (1ll << a.shift) ? len - from : 1ll << a.shift);
    const int32_t *entity = a.entity ? a.entity + e0 + from : nullptr;
    const uint8_t *hop = a.hop ? a.hop + e0 + from : nullptr;

    const int vr = blockIdx.y * 32 + (lane & 31);
    const bool mine = vr < a.rows;
    const int token = mine ? vr / a.group : 0, g = mine ? vr % a.group : 0;
    const long long place = ((long long)d * a.tokens + token) * a.heads + head * a.group + g;
    typename Vec8<E>::type q[kSteps];
#pragma unroll
    for (int kk = 0; kk < kSteps; kk++) q[kk] = row_chunk<E>((const E *)a.q + place * a.dim, mine, kk, a.dim, lane);
    const int q_pos = a.q_pos ? a.q_pos[d] : 0, M = a.score.max_distance;
    const float *my_table = table + g * (2 * M + 1);
    if (BIAS) {
        bias_to_lds<E>(table, a.score, head * a.group, a.group, tid, 256);
        __syncthreads();
    }
    f32x16 o[kOut];
#pragma unroll
    for (int i = 0; i < kOut; i++) o[i] = zero16();
    float m = kLowest, l = 0.f;

    const E *keys = (const E *)a.keys + (long long)head * a.key_head, *values = (const E *)a.values + (long long)head * a.value_head;
    auto id_of = [&](int t) {  // row of the table of this lane's entry of tile t, -1 for none
        int at = t * kReadTile + (lane & 31);
        if (at >= n) return -1;
        long long id = entity ? entity[at] : e0 + from + at;
        return id >= 0 && id < a.num_entities ? (int)id : -1;
    };
    auto hop_of = [&](int t) {
        int at = t * kReadTile + (lane & 31);
        return hop && at < n ? (int)hop[at] : 0;
    };
    u32x4 k[kSteps], v[DP / 16];
    auto fetch = [&](int id) {  // keys and values of a tile, once its rows stand in ids
        const E *krow = keys + (long long)(id < 0 ? 0 : id) * a.key_row;
#pragma unroll
        for (int kk = 0; kk < kSteps; kk++) {
            int c = 16 * kk + 8 * half;
            k[kk] = id >= 0 && c < a.dim ? *(const u32x4 *)(krow + c) : u32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < DP / 16; i++) {
            int at = i * 64 + lane, r = at / kRow, c = (at % kRow) * 8;
            long long vid = ids[wave][r];
            v[i] = vid >= 0 && c < a.dim ? *(const u32x4 *)(values + vid * a.value_row + c) : u32x4{0, 0, 0, 0};
        }
    };
    // A tile's rows of the table are known two rounds, its keys and values asked for one round ahead.
    const int tiles_n = (n + kReadTile - 1) / kReadTile;
    int id = id_of(wave), next_id = id_of(wave + 4), next_hop = 0, now_hop = 0;
    if (BIAS) now_hop = hop_of(wave), next_hop = hop_of(wave + 4);
    if (wave < tiles_n) {
        if (lane < 32) ids[wave][lane] = id;
        wave_sync();
        fetch(id);
    }
    for (int t = wave; t < tiles_n; t += 4) {
        const unsigned seen = (unsigned)__ballot(id >= 0);
        f32x16 s = zero16();
#pragma unroll
        for (int kk = 0; kk < kSteps; kk++) s = mfma(as8<E>(k[kk]), q[kk], s);
#pragma unroll
        for (int i = 0; i < DP / 16; i++) {
            int at = i * 64 + lane, r = at / kRow, c = at % kRow;
            *(u32x4 *)(vt + r * (DP * 2) + ((c ^ spread<DP>(r)) << 4)) = v[i];
        }
        if (lane < 32) {
            ids[wave][lane] = next_id;
            if (BIAS) hops[wave][lane] = now_hop;
        }
        wave_sync();
        id = next_id;
        now_hop = next_hop;
        if (t + 4 < tiles_n) fetch(id);
        next_id = id_of(t + 8);
        if (BIAS) next_hop = hop_of(t + 8);
        if (CAP) cap_scores<4>(a.score, s);
        float top = kLowest;
#pragma unroll
        for (int r = 0; r < 16; r++) {
            float y = CAP ? s[r] : s[r] * a.score.k;
            const int at = 8 * (r / 4) + 4 * half + r % 4;
            if (BIAS) y += my_table[distance_place(hops[wave][at], q_pos, M)];
            if (seen != ~0u) y = seen >> at & 1 ? y : -INFINITY;
            s[r] = y;
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
        for (int r = 0; r < 16; r++) {
            s[r] = exp2_fast(s[r] - m);
            l += s[r];
        }
        typename Vec8<E>::type p0 = rounded8<E, 0>(s), p1 = rounded8<E, 1>(s);
#pragma unroll
        for (int i = 0; i < kOut; i++) {
            o[i] = mfma(columns_chunk<E, DP>(my_columns, 0, i), p0, o[i]);
            o[i] = mfma(columns_chunk<E, DP>(my_columns, 16, i), p1, o[i]);
        }
        wave_sync();
    }
    const Joined all = join_wavefronts<DP>(o, m, l, lds, wave_m, wave_l, wave, lane);
    const float top = all.top;
    if (wave != 0 || !mine) return;
    if (alone) {
        const float sum = all.sum;
        const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
        write_row<E, DP>(o, inv, (E *)a.out + place * a.dim, a.dim, half);
        if (half == 0) a.lse[place] = sum == 0.f ? -INFINITY : (top + __log2f(sum)) * kLn2;
    } else {
        typedef float f32x4 __attribute__((ext_vector_type(4)));
        const long long at = (block * a.tokens + token) * a.heads + head * a.group + g;
#pragma unroll
        for (int i = 0; i < kOut; i++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
                int c = 32 * i + 8 * r + 4 * half;
                if (c < a.dim) *(f32x4 *)(a.part_o + at * a.dim + c) = f32x4{o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
            }
        if (half == 0) a.part_ml[2 * at] = top, a.part_ml[2 * at + 1] = all.sum;
    }
}

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

static logoskg_status read_args(const logoskg_entity_read *r, ReadArgs *a, const char *call) {
    if (!r || r->struct_size != sizeof(logoskg_entity_read)) { set_error("%s: struct_size", call); return LOGOSKG_EINVAL; }
    const char *why = bad_heads(r->dtype, r->heads, r->kv_heads, r->dim);
    if (!why) why = bad_score(r->score, r->heads, r->kv_heads);
    if (!why && (r->num_queries < 0 || r->tokens < 1 || r->tokens > 65535 || r->num_entries < 0 || r->num_entities < 0)) why = "a count is out of range";
    if (!why && r->num_entities >= (1ll << 31) && r->entity) why = "num_entities is 2^31 or more";
    if (!why && !r->entity && r->num_entities < r->num_entries) why = "fewer rows than entries";
    if (!why && r->num_entities >= (1ll << 31)) why = "num_entities is 2^31 or more";
    if (!why && r->num_queries && (!r->off || !r->q || !r->out || !r->lse)) why = "off, q, out or lse is NULL";
    if (!why && r->num_entries && r->num_entities && (!r->keys || !r->values)) why = "keys or values is NULL";
    if (!why && ((((uintptr_t)r->q | (uintptr_t)r->keys | (uintptr_t)r->values | (uintptr_t)r->out | (uintptr_t)r->workspace) & 15) ||
                 ((r->key_row | r->key_head | r->value_row | r->value_head) & 7)))
        why = "an array is not 16-byte aligned, or a stride no multiple of 8";
    if (why) { set_error("%s: %s", call, why); return LOGOSKG_EINVAL; }
    memset(a, 0, sizeof *a);
    a->num_queries = r->num_queries; a->tokens = r->tokens; a->heads = r->heads; a->kv_heads = r->kv_heads;
    a->group = r->heads / r->kv_heads; a->dim = r->dim; a->rows = a->tokens * a->group;
    a->num_entries = r->num_entries; a->num_entities = r->num_entities;
    a->off = r->off; a->entity = r->entity; a->q_pos = r->q_pos; a->hop = r->hop;
    a->q = r->q; a->keys = r->keys; a->values = r->values;
    a->key_row = r->key_row; a->key_head = r->key_head; a->value_row = r->value_row; a->value_head = r->value_head;
    a->score = score_args(r->score);
    a->out = r->out; a->lse = r->lse;
    // blocks of 128 entries, larger ones (up to 4,096) where there are more than 2,048 of them: four rounds of the card's 512
    const long long row_groups = (a->rows + 31) / 32;
    a->shift = kReadLeastShift;
    while (a->shift < 12 && (a->num_entries >> a->shift) * a->kv_heads * row_groups > 2048) a->shift++;
    a->blocks = (a->num_entries >> a->shift) + a->num_queries;
    if ((a->blocks + 8) * a->kv_heads >= (1ll << 31) || row_groups > 65535 || (long long)a->num_queries * a->tokens * a->heads >= (1ll << 32)) { set_error("%s: too many rows", call); return LOGOSKG_EINVAL; }
    return LOGOSKG_OK;
}

static int64_t part_bytes(const ReadArgs &a) {  // one block per list: nothing to join
    return a.num_entries <= (1ll << a.shift) ? 0 : (int64_t)a.blocks * a.tokens * a.heads * (a.dim + 2) * 4;
}

template <class E, int DP, bool CAP, bool BIAS> static logoskg_status launch_read(const ReadArgs &a, hipStream_t st) {
    size_t bytes = 4 * kReadTile * DP * 2 + (BIAS ? (size_t)a.group * (2 * a.score.max_distance + 1) * 4 : 0);
    LKG_TRY(allow_lds(k_read<E, DP, CAP, BIAS>, bytes));
    k_read<E, DP, CAP, BIAS><<<dim3((unsigned)((a.blocks + 7) / 8 * 8 * a.kv_heads), (unsigned)((a.rows + 31) / 32)), 256, bytes, st>>>(a);
    LKG_HIP(hipGetLastError());
    return LOGOSKG_OK;
}
template <class E> static logoskg_status read(const ReadArgs &a, hipStream_t st) {
    const bool cap = a.score.c > 0, bias = a.score.bias != nullptr;
    if (a.dim > 64) LKG_TRY((cap ? bias ? launch_read<E, 128, true, true>(a, st) : launch_read<E, 128, true, false>(a, st)
                                 : bias ? launch_read<E, 128, false, true>(a, st) : launch_read<E, 128, false, false>(a, st)));
    else LKG_TRY((cap ? bias ? launch_read<E, 64, true, true>(a, st) : launch_read<E, 64, true, false>(a, st)
                      : bias ? launch_read<E, 64, false, true>(a, st) : launch_read<E, 64, false, false>(a, st)));
    if (part_bytes(a)) {
        long long n = (long long)a.num_queries * a.tokens * a.heads;
        k_read_join<E><<<dim3((unsigned)((n + 3) / 4)), 256, 0, st>>>(a);
        LKG_HIP(hipGetLastError());
    }
    return LOGOSKG_OK;
}

}  // namespace lkg

using namespace lkg;

extern "C" int64_t logoskg_read_entities_bytes(const logoskg_entity_read *r) {
    ReadArgs a;
    return read_args(r, &a, "logoskg_read_entities_bytes") == LOGOSKG_OK ? part_bytes(a) : -1;
}

extern "C" logoskg_status logoskg_read_entities(const logoskg_entity_read *r) {
    ReadArgs a;
    LKG_TRY(read_args(r, &a, "logoskg_read_entities"));
    if (r->workspace_bytes < part_bytes(a) || (part_bytes(a) && !r->workspace)) {
        set_error("logoskg_read_entities: the workspace has %lld of %lld bytes", (long long)r->workspace_bytes, (long long)part_bytes(a));
        return LOGOSKG_ERANGE;
    }
    if (a.num_queries == 0) return LOGOSKG_OK;
    a.part_o = (float *)r->workspace;
    a.part_ml = a.part_o + (part_bytes(a) ? a.blocks * a.tokens * a.heads * a.dim : 0);
    LKG_HIP(hipSetDevice(r->device));
    return r->dtype == LOGOSKG_BF16 ? read<bf16>(a, (hipStream_t)r->stream) : read<fp16>(a, (hipStream_t)r->stream);
}
