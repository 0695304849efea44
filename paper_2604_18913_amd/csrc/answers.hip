// Entity lists as bit masks, and a step's logits under penalties, biases and masks (logoskg_entity_mask,
// logoskg_constrain_logits).
#include "reading.h"

namespace lkg {

typedef unsigned long long u64;

__global__ __launch_bounds__(256) void k_mask_clear(ulonglong2 *mask, long long pairs, u64 *last) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < pairs; i += (long long)gridDim.x * 256) mask[i] = ulonglong2{0, 0};
    if (last && blockIdx.x == 0 && threadIdx.x == 0) *last = 0;
}

constexpr int kMaskEntries = 1024;  // of a block

// One atomic "or" per run of neighbouring lanes whose ids share a word (lists ascend, so that most runs are whole words):
// the first lane of a run takes the bits of the others.
__global__ __launch_bounds__(256) void k_mask_set(const int64_t *off, const int32_t *ids, long long n, int Q, long long num_ids, long long words, u64 *mask) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long base = (long long)blockIdx.x * kMaskEntries + wave * 256;
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
    long long vocab, row, words, num_history, num_bias;
    const void *logits;
    void *out;
    const int64_t *history_off, *bias_off;
    const int32_t *history, *bias_id;
    const float *repetition, *presence, *frequency, *bias_value;
    const u64 *mask;
};

constexpr int kPiece = 8192;  // ids of a block

// One block: a piece of a row.  The row's history is counted into LDS for the ids of the piece, its biases' last entries are
// found the same way, and the piece passes once through registers.  Whole numbers only are added up by atomics.
template <class T> __global__ __launch_bounds__(512) void k_logits(LogitArgs a) {
    __shared__ int count[kPiece];
    __shared__ int which[kPiece];
    const int tid = threadIdx.x;
    const long long pieces = (a.vocab + kPiece - 1) / kPiece, b = blockIdx.x / pieces, v0 = (blockIdx.x % pieces) * kPiece;
    const int n = (int)(a.vocab - v0 < kPiece ? a.vocab - v0 : kPiece);
    long long h0 = 0, h1 = 0, s0 = 0, s1 = 0;
    if (a.history_off) h0 = taken_into(a.history_off[b], a.num_history), h1 = taken_into(a.history_off[b + 1], a.num_history);
    if (a.bias_off) s0 = taken_into(a.bias_off[b], a.num_bias), s1 = taken_into(a.bias_off[b + 1], a.num_bias);
    const bool said = h1 > h0, biased = s1 > s0;
    if (said)
        for (int i = tid; i < n; i += 512) count[i] = 0;
    if (biased)
        for (int i = tid; i < n; i += 512) which[i] = -1;
    if (said || biased) __syncthreads();
    for (long long i = h0 + tid; i < h1; i += 512) {
        long long id = a.history[i] - v0;
        if (a.history[i] >= 0 && id >= 0 && id < n) atomicAdd(&count[id], 1);
    }
    for (long long i = s0 + tid; i < s1; i += 512) {
        long long id = a.bias_id[i] - v0;
        if (a.bias_id[i] >= 0 && id >= 0 && id < n) atomicMax(&which[id], (int)(i - s0));
    }
    if (said || biased) __syncthreads();
    const float rep = a.repetition ? a.repetition[b] : 1.f, pres = a.presence ? a.presence[b] : 0.f, freq = a.frequency ? a.frequency[b] : 0.f;
    const T *in = (const T *)a.logits + b * a.row + v0;
    T *out = (T *)a.out + b * a.row + v0;
    const u64 *mask = a.mask ? a.mask + b * a.words + (v0 >> 6) : nullptr;
    for (int i = tid; i < n; i += 512) {
        float x = (float)in[i];
        if (said) {
            int c = count[i];
            if (c > 0) x = (x > 0.f ? x / rep : x * rep) - (freq * c + pres);
        }
        if (biased && which[i] >= 0) x += a.bias_value[s0 + which[i]];
        if (mask && !(mask[i >> 6] >> (i & 63) & 1)) x = -INFINITY;
        out[i] = (T)x;
    }
}

}  // namespace lkg

using namespace lkg;

extern "C" logoskg_status logoskg_entity_mask(int32_t device, const int64_t *off, const int32_t *ids, int64_t num_entries,
                                              int32_t num_queries, int64_t num_ids, uint64_t *mask, void *stream) {
    const char *why = nullptr;
    if (num_entries < 0 || num_queries < 0 || num_ids < 0 || num_ids > (1ll << 31) || num_entries >= (1ll << 40)) why = "a count is out of range";
    else if (num_queries && num_ids && !mask) why = "mask is NULL";
    else if (num_entries && num_queries && (!off || !ids)) why = "off or ids is NULL";
    else if ((uintptr_t)mask & 15) why = "mask is not 16-byte aligned";
    if (why) { set_error("logoskg_entity_mask: %s", why); return LOGOSKG_EINVAL; }
    const long long words = (num_ids + 63) / 64, all = words * num_queries;
    if (all == 0) return LOGOSKG_OK;
    LKG_HIP(hipSetDevice(device));
    hipStream_t st = (hipStream_t)stream;
    const long long blocks = (all / 2 + 255) / 256;
    k_mask_clear<<<dim3((unsigned)(blocks < 1 ? 1 : blocks > 8192 ? 8192 : blocks)), 256, 0, st>>>((ulonglong2 *)mask, all / 2, all & 1 ? (u64 *)mask + all - 1 : nullptr);
    LKG_HIP(hipGetLastError());
    if (num_entries) {
        k_mask_set<<<dim3((unsigned)((num_entries + kMaskEntries - 1) / kMaskEntries)), 256, 0, st>>>(off, ids, num_entries, num_queries, num_ids, words, (u64 *)mask);
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
    const long long blocks = (l->vocab + kPiece - 1) / kPiece * l->num_rows;
    if (blocks >= (1ll << 31)) { set_error("logoskg_constrain_logits: too many rows"); return LOGOSKG_EINVAL; }
    LKG_HIP(hipSetDevice(l->device));
    hipStream_t st = (hipStream_t)l->stream;
    if (l->dtype == LOGOSKG_F32) k_logits<float><<<dim3((unsigned)blocks), 512, 0, st>>>(a);
    else if (l->dtype == LOGOSKG_BF16) k_logits<bf16><<<dim3((unsigned)blocks), 512, 0, st>>>(a);
    else k_logits<fp16><<<dim3((unsigned)blocks), 512, 0, st>>>(a);
    LKG_HIP(hipGetLastError());
    return LOGOSKG_OK;
}
