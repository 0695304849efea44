// Entity lists as bit masks, and a step's logits under penalties, biases and masks (logoskg_entity_mask,
// logoskg_constrain_logits).
#include "reading.h"

namespace lkg {

typedef unsigned long long u64;

constexpr int kMostMaskPieces = 96, kMostMaskList = 1 << 16;  // of a query (entries: on average): made in LDS up to these

// f(entry) of the entries [b, e) of a list, by a block's threads: in 16-byte chunks, four of a thread in flight, what lies before and
// behind the whole ones alone.
template <int THREADS, class F> __device__ __forceinline__ void for_entries(const int32_t *list, long long b, long long e, int tid, F f) {
    const long long a0 = b + ((16 - ((uintptr_t)(list + b) & 15)) & 15) / 4, chunks = e > a0 ? (e - a0) / 4 : 0, a1 = a0 + chunks * 4;
    if (chunks == 0) {
        if (b + tid < e) f(list[b + tid]);  // (six at most)
        return;
    }
    if (b + tid < a0) f(list[b + tid]);
    if (a1 + tid < e) f(list[a1 + tid]);
    const int4 *whole = (const int4 *)(list + a0);
    long long i = tid;
    for (; i + 3 * THREADS < chunks; i += 4 * THREADS) {
        const int4 x[4] = {whole[i], whole[i + THREADS], whole[i + 2 * THREADS], whole[i + 3 * THREADS]};
#pragma unroll
        for (int u = 0; u < 4; u++) f(x[u].x), f(x[u].y), f(x[u].z), f(x[u].w);
    }
    for (; i < chunks; i += THREADS) {
        const int4 x = whole[i];
        f(x.x), f(x.y), f(x.z), f(x.w);
    }
}

// Masks come out in one of two ways.  Where a list can be looked through once for every piece of its mask, a block makes a
// piece in LDS and writes it once (k_mask_piece): no cleared memory and no atomics on it.  Else the masks are cleared and
// the ids set by atomics (k_mask_clear, k_mask_set).  1,024 lists of up to 30,000 of 3 M ids: 115 us, 3.9 TB/s, nearly all of it
// the masks' 384 MB (a fill writes 6.9 TB/s, and the blocks are not all at the same phase).
__global__ __launch_bounds__(1024) void k_mask_piece(const int64_t *off, const int32_t *ids, long long n, long long num_ids, long long words, int pieces, int piece_words, u64 *mask) {
    extern __shared__ u64 bits[];
    const int tid = threadIdx.x, q = blockIdx.x / pieces;
    const long long w0 = (long long)(blockIdx.x % pieces) * piece_words;
    const int count = (int)(words - w0 < piece_words ? words - w0 : piece_words);
    for (int i = tid; i < count; i += 1024) bits[i] = 0;
    const long long e0 = taken_into(off[q], n), e1 = taken_into(off[q + 1], n), lo = w0 * 64;
    const unsigned size = (unsigned)(lo + (long long)count * 64 < num_ids ? (long long)count * 64 : num_ids - lo);
    auto set = [&](int id) {
        const unsigned at = (unsigned)id - (unsigned)lo;  // (ids and lo are below 2^31: one compare for both ends)
        if (at < size) atomicOr(&((unsigned *)bits)[at >> 5], 1u << (at & 31));
    };
    __syncthreads();
    for_entries<1024>(ids, e0, e1, tid, set);
    __syncthreads();
    for (int i = tid; i < count; i += 1024) mask[q * words + w0 + i] = bits[i];
}

__global__ __launch_bounds__(256) void k_mask_clear(ulonglong2 *mask, long long pairs, u64 *last) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < pairs; i += (long long)gridDim.x * 256) mask[i] = ulonglong2{0, 0};
    if (last && blockIdx.x == 0 && threadIdx.x == 0) *last = 0;
}

constexpr int kMaskEntries = 1024;  // of a block

// One atomic "or" per run of neighbouring lanes whose ids share a word (lists ascend, so that most runs are whole words):
// the first lane of a run takes the bits of the others.
__global__ __launch_bounds__(256) void k_mask_set(const int64_t *off, const int32_t *ids, long long n, int Q, long long num_ids, long long words, u64 *mask, long long first) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long base = (first + blockIdx.x) * kMaskEntries + wave * 256;
    if (base >= n) return;
    // the list of the wavefront's first entry; later ones move on from it
    int lo = 0, hi = Q;  // off[lo] <= base < off[hi]
    while (hi - lo > 1) {
        int step = (hi - lo + 63) >> 6, at = lo + lane * step;
        int count = __popcll(__ballot(at < hi && off[at] <= base));
        lo += (count > 0 ? count - 1 : 0) * step;
        hi = lo + step < hi ? lo + step : hi;
    }
    int q = lo;
    for (int i = 0; i < 4; i++) {
        const long long at = base + i * 64 + lane;
        while (q + 1 < Q && at < n && off[q + 1] <= at) q++;
        const long long id = at < n ? ids[at] : -1;
        const bool in = id >= 0 && id < num_ids && at >= off[q] && at < off[q + 1];
        const long long word = in ? (long long)q * words + (id >> 6) : -1 - lane;
        u64 bit = in ? 1ull << (id & 63) : 0;
        const long long before = __shfl_up(word, 1);  // (of all lanes)
        const bool head = lane == 0 || before != word;
        const u64 heads = __ballot(head);
        const int end = (heads >> lane >> 1) ? lane + __ffsll((long long)(heads >> lane >> 1)) : 64;  // of my run
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            u64 other = __shfl_down(bit, s);
            if (lane + s < end) bit |= other;
        }
        if (in && head) __hip_atomic_fetch_or(mask + word, bit, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

// ---------------------------------------------------------------- logits
struct LogitArgs {
    int num_rows;
    long long vocab, row, words, num_history, num_bias, pieces, first;  // pieces of a row; row that a launch begins with
    const void *logits;
    void *out;
    const int64_t *history_off, *bias_off;
    const int32_t *history, *bias_id;
    const float *repetition, *presence, *frequency, *bias_value;
    const u64 *mask;
};

constexpr int kBiasHits = 512;  // of a piece: listed in LDS
constexpr int kBiasIds = 1024;  // ids that are looked after at a time in a piece with more of them

// One block: a piece of 16 ids per thread of a row.  The logits pass once through registers under the mask, in 16-byte chunks
// from the first whole one of the row on, where logits and out lie alike; else one by one.  What the lists ask for is few
// ids, and comes behind: the row's history is counted in LDS for the ids of the piece, in 16 bits (32 where the history is so long
// that a count might not fit, for half of the ids at a time); its biases that fall into the piece are marked, and listed with
// their places in the row's list, of which the last counts; then every thread looks through 16 neighbouring ids and writes
// those again that a list holds and the mask allows.  (A chunk that looks after its own ids has some instructions for each of
// its eight as soon as one lane of the wavefront has one.)  Whole numbers only are added up by atomics.
//
// Where more biases fall into a piece than are listed (a bias on every id), the row's list is gone through again for every 1,024 ids of
// it, and the last place of each id is the largest: 16 rows of 150,001 bfloat16 logits, 300 / 30,000 / 150,001 biases each, take
// 13 / 290 / 970 us.
template <class T, int THREADS> __global__ __launch_bounds__(THREADS) void k_logits(LogitArgs a) {
    constexpr int kPiece = 16 * THREADS, kChunk = 16 / sizeof(T), kChunks = 16 / kChunk;  // ids of a chunk; chunks of a thread
    typedef T chunk __attribute__((ext_vector_type(kChunk)));
    __shared__ __attribute__((aligned(16))) unsigned count[kPiece / 2];
    __shared__ unsigned marked[kPiece / 32];
    __shared__ union {
        struct { int id[kBiasHits], at[kBiasHits]; float value[kBiasHits]; } hit;
        int last[kBiasIds];  // place in the row's list
    } few;
    __shared__ int hits;
    const int tid = threadIdx.x;
    const long long b = a.first + blockIdx.x / a.pieces;
    const T *in = (const T *)a.logits + b * a.row;
    T *out = (T *)a.out + b * a.row;
    // ids of the row before its first whole chunk; pieces begin there, the first one with what lies before
    const int lead = (int)((16 - ((uintptr_t)in & 15)) & 15) / (int)sizeof(T);
    const bool alike = (((uintptr_t)in ^ (uintptr_t)out) & 15) == 0;
    const long long piece = blockIdx.x % a.pieces, v0 = piece * kPiece + lead - kChunk;  // a chunk more than the ids that may lie before
    const long long lo = piece == 0 ? 0 : v0, hi = v0 + kPiece < a.vocab ? v0 + kPiece : a.vocab;
    if (lo >= hi) return;
    const u64 *mask = a.mask ? a.mask + b * a.words : nullptr;
    auto allowed = [&](long long v) { return !mask || (mask[v >> 6] >> (v & 63) & 1); };
    chunk x[kChunks];
    u64 word[kChunks], behind[kChunks];  // of the mask: that of a chunk's first id, and the next where the chunk goes on into it
    if (alike) {
#pragma unroll
        for (int i = 0; i < kChunks; i++) {
            const long long v = v0 + (long long)(i * THREADS + tid) * kChunk;
            word[i] = ~0ull, behind[i] = ~0ull;
            if (v >= lo && v + kChunk <= hi) {
                x[i] = *(const chunk *)(in + v);
                if (mask) {
                    word[i] = mask[v >> 6];
                    if ((v & 63) > 64 - kChunk) behind[i] = mask[(v >> 6) + 1];
                }
            }
        }
    }
    long long h0 = 0, h1 = 0, s0 = 0, s1 = 0;
    if (a.history_off) h0 = taken_into(a.history_off[b], a.num_history), h1 = taken_into(a.history_off[b + 1], a.num_history);
    if (a.bias_off) s0 = taken_into(a.bias_off[b], a.num_bias), s1 = taken_into(a.bias_off[b + 1], a.num_bias);
    const bool said = h1 > h0, biased = s1 > s0, wide = h1 - h0 > 65535;
    const float rep = a.repetition ? a.repetition[b] : 1.f, pres = a.presence ? a.presence[b] : 0.f, freq = a.frequency ? a.frequency[b] : 0.f;
    const float inv_rep = 1.f / rep;  // (a product with it is within two units of the last place of 32 bits)
    auto penalised = [&](float y, unsigned c) { return c > 0 ? y * (y > 0.f ? inv_rep : rep) - __builtin_fmaf(freq, (float)c, pres) : y; };
    auto bias_of = [&](long long v) __attribute__((always_inline)) {  // of a marked id
        const int at = (int)(v - v0);
        int last = -1;
        float value = 0.f;
        for (int i = 0; i < hits; i++)
            if (few.hit.id[i] == at && few.hit.at[i] > last) last = few.hit.at[i], value = few.hit.value[i];
        return value;
    };
    auto from_of = [&](int round) { return round == 0 ? lo : lo > v0 + kPiece / 2 ? lo : v0 + kPiece / 2; };  // ids of a round
    auto to_of = [&](int round) { return wide && round == 0 && v0 + kPiece / 2 < hi ? v0 + kPiece / 2 : hi; };
    auto clear = [&] {
        for (int i = tid; i < (int)(sizeof(count) / 16); i += THREADS) ((u32x4 *)count)[i] = u32x4{0, 0, 0, 0};
    };
    auto count_history = [&](int round) {
        const long long w0 = v0 + round * (kPiece / 2), from = from_of(round), to = to_of(round);
        const unsigned base = (unsigned)w0, skip = (unsigned)(from - w0), size = to > from ? (unsigned)(to - from) : 0;
        for_entries<THREADS>(a.history, h0, h1, tid, [&](int id) {
            const unsigned at = (unsigned)id - base;
            if (at - skip >= size) return;
            if (wide) atomicAdd(&count[at], 1u);
            else atomicAdd(&count[at >> 1], at & 1 ? 65536u : 1u);
        });
    };
    const bool listed = said || biased;
    u64 allow[2] = {~0ull, ~0ull};  // of the ids that this thread looks through in a round
    auto look_up = [&](int round) {
        const long long v = v0 + (wide ? 8 * tid + round * (kPiece / 2) : 16 * tid);
        for (int i = 0; i < 2; i++) {
            const long long w = (v >> 6) + i;
            if (mask) allow[i] = w >= 0 && w < a.words ? mask[w] : 0;
        }
    };
    // (the logits themselves are written: in place, an allowed one still stands as it came)
    auto write_again = [&](int round) __attribute__((always_inline)) {
        const int mine = wide ? 8 : 16, at0 = mine * tid, all0 = at0 + round * (kPiece / 2);
        const long long first = v0 + all0;
        const int sh = (int)(first & 63);
        unsigned again = biased ? marked[all0 >> 5] >> (all0 & 31) : 0;
        if (said) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const unsigned c = count[8 * tid + i];
                again |= wide ? (unsigned)(c != 0) << i : (unsigned)((c & 65535u) != 0) << 2 * i | (unsigned)(c >> 16 != 0) << (2 * i + 1);
            }
        }
        again &= (unsigned)(allow[0] >> sh | allow[1] << 1 << (63 - sh)) & ((1u << mine) - 1);
        if (!again) return;
        float next = (float)in[first + __ffs(again) - 1];
        while (again) {
            const int e = __ffs(again) - 1, at = at0 + e;
            float y = next;
            again &= again - 1;
            if (again) next = (float)in[first + __ffs(again) - 1];
            y = penalised(y, !said ? 0u : wide ? count[at] : count[at >> 1] >> (16 * (at & 1)) & 65535u);
            if (biased && (marked[(all0 + e) >> 5] >> ((all0 + e) & 31) & 1)) y += bias_of(first + e);
            out[first + e] = (T)y;
        }
    };
    // .. where more biases fall into the piece than are listed: the places of kBiasIds ids at a time from the row's list again
    auto write_many = [&](int round) __attribute__((always_inline)) {
#pragma unroll 1
        for (int s = 0; s < (wide ? kPiece / 2 : kPiece); s += kBiasIds) {
            const long long w0 = v0 + round * (kPiece / 2) + s;
            __syncthreads();
            for (int i = tid; i < kBiasIds; i += THREADS) few.last[i] = -1;
            __syncthreads();
            for (long long i = s0 + tid; i < s1; i += THREADS) {
                const long long at = a.bias_id[i] - w0;
                if (at >= 0 && at < kBiasIds) atomicMax(&few.last[at], (int)(i - s0));
            }
            __syncthreads();
#pragma unroll 1
            for (int i = tid; i < kBiasIds; i += THREADS) {
                const long long v = w0 + i;
                if (v < lo || v >= hi || !allowed(v)) continue;
                const int at = s + i;
                const unsigned c = !said ? 0u : wide ? count[at] : count[at >> 1] >> (16 * (at & 1)) & 65535u;
                if (c == 0 && few.last[i] < 0) continue;
                float y = penalised((float)in[v], c);
                if (few.last[i] >= 0) y += a.bias_value[s0 + few.last[i]];
                out[v] = (T)y;
            }
        }
    };
    auto write_listed = [&](int round) __attribute__((always_inline)) {
        if (__builtin_expect(hits > kBiasHits, 0)) write_many(round);
        else write_again(round);
    };
    if (listed) {
        for (int i = tid; i < kPiece / 32; i += THREADS) marked[i] = 0;
        if (tid == 0) hits = 0;
        clear();
        __syncthreads();
        for (long long i = s0 + tid; i < s1; i += THREADS) {
            const long long id = a.bias_id[i];
            if (id >= lo && id < hi) {
                atomicOr(&marked[(int)(id - v0) >> 5], 1u << ((id - v0) & 31));
                const int n = atomicAdd(&hits, 1);
                if (n < kBiasHits) few.hit.id[n] = (int)(id - v0), few.hit.at[n] = (int)(i - s0), few.hit.value[n] = a.bias_value[i];
            }
        }
        count_history(0);
        look_up(0);
    }
    if (alike) {
#pragma unroll
        for (int i = 0; i < kChunks; i++) {
            const long long v = v0 + (long long)(i * THREADS + tid) * kChunk;
            if (v >= lo && v + kChunk <= hi) {
                const int sh = (int)(v & 63);
                const unsigned bits = (unsigned)(word[i] >> sh | behind[i] << 1 << (63 - sh));
#pragma unroll
                for (int e = 0; e < kChunk; e++) x[i][e] = bits >> e & 1 ? x[i][e] : (T)-INFINITY;
                *(chunk *)(out + v) = x[i];
            } else {
                for (long long w = v < lo ? lo : v; w < v + kChunk && w < hi; w++) out[w] = allowed(w) ? in[w] : (T)-INFINITY;
            }
        }
    } else {
        for (long long v = lo + tid; v < hi; v += THREADS) out[v] = allowed(v) ? in[v] : (T)-INFINITY;
    }
    if (!listed) return;
    __syncthreads();
    write_listed(0);
    if (!wide) return;
    __syncthreads();
    clear();
    __syncthreads();
    count_history(1);
    look_up(1);
    __syncthreads();
    write_listed(1);
}

template <class T> static logoskg_status launch_logits(LogitArgs a, hipStream_t st) {
    // Pieces of 4,096 ids, 256 threads: 256 rows of 150,001 bfloat16 logits with histories of up to 4,000 ids and 300 biases take 44 us
    // (3.6 TB/s; a copy of the logits and masks 33), with next to no lists 29; pieces of 2,048 take 49 and 29, of 8,192
    // 48 and 29, of 16,384 73 and 45 us.  (256 rows of 32,000 float32 logits with 8,000 ids each: 26, 28, 24, 22 us.)
    a.pieces = (a.vocab + 4096 + 15) / 4096;
    launch_ranges(a.num_rows, 1, [&](long long first, long long n) {
        a.first = first;
        k_logits<T, 256><<<dim3((unsigned)(a.pieces * n)), 256, 0, st>>>(a);
    }, kMaxBlocks / a.pieces);
    LKG_HIP(hipGetLastError());
    return LOGOSKG_OK;
}

}  // namespace lkg

using namespace lkg;

extern "C" logoskg_status logoskg_entity_mask(int32_t device, const int64_t *off, const int32_t *ids, int64_t num_entries,
                                              int32_t num_queries, int64_t num_ids, uint64_t *mask, void *stream) {
    const char *why = nullptr;
    if (num_entries < 0 || num_queries < 0 || num_ids < 0 || num_ids > (1ll << 31) || num_entries >= (1ll << 40)) why = "a count is out of range";
    else if (num_queries && num_ids && !mask) why = "mask is NULL";
    else if (num_queries && num_ids && (!off || (num_entries && !ids))) why = "off or ids is NULL";
    else if ((uintptr_t)mask & 15) why = "mask is not 16-byte aligned";
    if (why) { set_error("logoskg_entity_mask: %s", why); return LOGOSKG_EINVAL; }
    const long long words = (num_ids + 63) / 64, all = words * num_queries;
    if (all == 0) return LOGOSKG_OK;
    LKG_HIP(hipSetDevice(device));
    hipStream_t st = (hipStream_t)stream;
    // Pieces of up to 16,384 words (128 KiB of LDS), smaller ones down to 512 where there are fewer than 512 of them.
    int piece_words = 16384;
    while (piece_words > 512 && (words + piece_words - 1) / piece_words * num_queries < 512) piece_words /= 2;
    const long long pieces = (words + piece_words - 1) / piece_words;
    if (pieces <= kMostMaskPieces && num_entries / num_queries <= kMostMaskList && pieces * num_queries <= kMaxBlocks / 4) {  // (blocks of 1,024: fewer than 2^32 threads)
        LKG_TRY(allow_lds(k_mask_piece, (size_t)piece_words * 8));
        k_mask_piece<<<dim3((unsigned)(pieces * num_queries)), 1024, piece_words * 8, st>>>(off, ids, num_entries, num_ids, words, (int)pieces, piece_words, (u64 *)mask);
        LKG_HIP(hipGetLastError());
        return LOGOSKG_OK;
    }
    const long long blocks = (all / 2 + 255) / 256;
    k_mask_clear<<<dim3((unsigned)(blocks < 1 ? 1 : blocks > 8192 ? 8192 : blocks)), 256, 0, st>>>((ulonglong2 *)mask, all / 2, all & 1 ? (u64 *)mask + all - 1 : nullptr);
    LKG_HIP(hipGetLastError());
    if (num_entries) {
        launch_ranges((num_entries + kMaskEntries - 1) / kMaskEntries, 1, [&](long long first, long long n) {
            k_mask_set<<<dim3((unsigned)n), 256, 0, st>>>(off, ids, num_entries, num_queries, num_ids, words, (u64 *)mask, first);
        });
        LKG_HIP(hipGetLastError());
    }
    return LOGOSKG_OK;
}

extern "C" logoskg_status logoskg_constrain_logits(const logoskg_logits *l) {
    const char *why = nullptr;
    if (!l || l->struct_size != sizeof(logoskg_logits)) why = "struct_size";
    else if (l->dtype < LOGOSKG_F32 || l->dtype > LOGOSKG_F16) why = "unknown type";
    else if (l->num_rows < 0 || l->vocab < 0 || l->vocab >= (1ll << 31) || l->num_history < 0 || l->num_bias < 0 || l->num_history >= (1ll << 31) || l->num_bias >= (1ll << 31)) why = "a count is out of range";
    else if (l->row < l->vocab && l->num_rows > 1) why = "rows overlap";
    else if (l->num_rows && l->vocab && (!l->logits || !l->out)) why = "logits or out is NULL";
    else if (l->history_off && l->num_history && !l->history) why = "history is NULL";
    else if (l->bias_off && l->num_bias && (!l->bias_id || !l->bias_value)) why = "bias_id or bias_value is NULL";
    if (why) { set_error("logoskg_constrain_logits: %s", why); return LOGOSKG_EINVAL; }
    if (l->num_rows == 0 || l->vocab == 0) return LOGOSKG_OK;
    LogitArgs a;
    memset(&a, 0, sizeof a);
    a.num_rows = l->num_rows; a.vocab = l->vocab; a.row = l->row; a.words = (l->vocab + 63) / 64;
    a.num_history = l->num_history; a.num_bias = l->num_bias;
    a.logits = l->logits; a.out = l->out;
    a.history_off = l->history_off; a.history = l->history; a.bias_off = l->bias_off; a.bias_id = l->bias_id;
    a.bias_value = l->bias_value; a.repetition = l->repetition; a.presence = l->presence; a.frequency = l->frequency;
    a.mask = (const u64 *)l->mask;
    LKG_HIP(hipSetDevice(l->device));
    hipStream_t st = (hipStream_t)l->stream;
    if (l->dtype == LOGOSKG_F32) return launch_logits<float>(a, st);
    return l->dtype == LOGOSKG_BF16 ? launch_logits<bf16>(a, st) : launch_logits<fp16>(a, st);
}
