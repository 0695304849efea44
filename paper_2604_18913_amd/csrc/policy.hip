// The loss of sampled answers over their logits, and its gradient (logoskg_token_logp, logoskg_policy_loss,
// logoskg_policy_loss_backward).
#include "training.h"

namespace lkg {

static_assert(sizeof(logoskg_policy) == 184, "the ctypes binding mirrors this layout");

typedef unsigned long long u64;

struct PolicyArgs {
    int num_rows, num_masks;
    long long vocab, row, words;
    const void *logits;
    const int32_t *target, *mask_row;
    const u64 *mask;
    float scale, kl, low, high;
    const float *advantage, *old, *ref, *weight;
    float *logp, *lse, *loss, *row_loss;
    void *dlogits;
    const float *dloss;
};

enum { kLogp, kLoss, kLossAndGradient, kBackward };  // what a launch does

// The largest and the sum of exp2((x - largest) k) so far.  Differences are made before the scaling, so that rows at the
// lowest values of a type have a sum too.
struct Sum {
    float top, sum;
    __device__ __forceinline__ void join(float other_top, float other_sum, float k) {
        const float up = fmaxf(top, other_top), at = up == -INFINITY ? 0.f : up;
        sum = sum * exp2_fast((top - at) * k) + other_sum * exp2_fast((other_top - at) * k);
        top = up;
    }
};

// A row's loss and what its logp's gradient is, weight included; 0 and 0 for rows that do not count.
__device__ __forceinline__ void row_terms(const PolicyArgs &a, int r, float logp, bool counts, float &loss, float &slope) {
    loss = slope = 0.f;
    if (!counts) return;
    const float A = a.advantage[r], w = a.weight ? a.weight[r] : 1.f;
    if (A != 0.f) {  // (an infinite ratio times 0 is nothing, too)
        const float ratio = a.old ? expf(logp - a.old[r]) : 1.f;
        const float near = fminf(fmaxf(ratio, 1.f - a.low), 1.f + a.high), inside = ratio * A, border = near * A;
        if (inside <= border || inside != inside) loss = -inside, slope = -inside;
        else loss = -border;
    }
    if (a.kl > 0.f) {
        const float d = a.ref[r] - logp, e = expm1f(d);
        loss += a.kl * (e - d);
        slope -= a.kl * e;
    }
    loss *= w;
    slope *= w;
    if (w == 0.f) loss = slope = 0.f;
}

// Exponents up to this size, in units of log 2, are made in one step, x k minus a product that is rounded before: 2^-19 of the exponential
// at most.
constexpr float kNear = 64.f;

// x where the bit is set, `other` where it is not: of a bit as a whole word two instructions
__device__ __forceinline__ float by_bit(unsigned bits, int e, float x, float other) {
    const unsigned m = (unsigned)__builtin_amdgcn_sbfe((int)bits, e, 1);
    return __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, x) & m) | (__builtin_bit_cast(unsigned, other) & ~m));
}

// One row by a block of THREADS threads: a sweep over its logits for the largest and the sum, another for the gradient.  The
// first KEEP chunks of a thread, all that there are in rows of up to 16 KEEP THREADS bytes, are asked for at once and stay in registers
// for the second sweep.
template <int THREADS> struct RowShared { float tops[THREADS / 64], sums[THREADS / 64], said[2]; };
template <class T, int THREADS, int MODE, bool MASKED, int KEEP> __device__ __forceinline__ void policy_row(const PolicyArgs &a, int r, int tid, RowShared<THREADS> &shared) {
    constexpr int V = 16 / sizeof(T), kWaves = THREADS / 64;
    const int lane = tid & 63, wave = tid >> 6;
    float *tops = shared.tops, *sums = shared.sums, *said = shared.said;
    auto all_here = [] {  // (rows of a wavefront each need no more than its own order)
        if (THREADS == 64) wave_sync();
        else __syncthreads();
    };
    const T *in = (const T *)a.logits + (long long)r * a.row;
    const long long vocab = a.vocab;
    const int target = a.target[r];
    const long long mask_at = !MASKED ? 0 : a.mask_row ? a.mask_row[r] : r;
    const bool closed = MASKED && (mask_at < 0 || mask_at >= a.num_masks);  // (such a row's mask is not read: nothing is allowed)
    const u64 *mask = MASKED && !closed ? a.mask + mask_at * a.words : nullptr;
    const float k = a.scale * kLog2e;
    const long long lead0 = ((16 - ((uintptr_t)in & 15)) & 15) / sizeof(T), lead = lead0 < vocab ? lead0 : vocab;
    const long long chunks = closed ? 0 : (vocab - lead) / V, tail = lead + (vocab - lead) / V * V;
    auto allowed = [&](long long v) { return !MASKED || (!closed && (mask[v >> 6] >> (v & 63) & 1)); };
    auto bits_of = [&](long long v) -> unsigned {  // of the V ids from v on, and others above: the two bytes that they stand in
        if (!MASKED) return ~0u;
        typedef unsigned short __attribute__((aligned(1))) two_bytes;
        const long long last = a.words * 8 - 2, at = v >> 3 < last ? v >> 3 : last;
        return (unsigned)*(const two_bytes *)((const char *)mask + at) >> (int)(v - 8 * at);
    };
    Some<T> kept[KEEP];
    unsigned kept_bits[MASKED ? KEEP : 1];
    Sum s = {-INFINITY, 0.f};
    float lse, logp, slope;
    if (MODE != kBackward) {
        auto take = [&](float x) { s.join(x, x == -INFINITY ? 0.f : 1.f, k); };
        if (tid < lead && allowed(tid)) take((float)in[tid]);
        if (tail + tid < vocab && allowed(tail + tid)) take((float)in[tail + tid]);
        auto take_chunk = [&](const Some<T> &x, unsigned bits) __attribute__((always_inline)) {
            float y[V], top = s.top;
#pragma unroll
            for (int e = 0; e < V; e++) {
                y[e] = (float)x[e];
                if (MASKED) y[e] = by_bit(bits, e, y[e], -INFINITY);
                top = fmaxf(top, y[e]);
            }
            const float at = top == -INFINITY ? 0.f : top;
            float sum = s.sum * exp2_fast((s.top - at) * k);
            const float from = -at * k;
            if (__builtin_expect(__builtin_fabsf(from) < kNear, 1)) {
#pragma unroll
                for (int e = 0; e < V; e++) sum += exp2_fast(__builtin_fmaf(y[e], k, from));
            } else {
#pragma unroll
                for (int e = 0; e < V; e++) sum += exp2_fast((y[e] - at) * k);
            }
            s.top = top, s.sum = sum;
        };
#pragma unroll
        for (int i = 0; i < KEEP; i++)
            if (tid + i * THREADS < chunks) {
                const long long v = lead + (long long)(tid + i * THREADS) * V;
                kept[i] = *(const Some<T> *)(in + v);
                if (MASKED) kept_bits[i] = bits_of(v);
            }
#pragma unroll
        for (int i = 0; i < KEEP; i++)
            if (tid + i * THREADS < chunks) take_chunk(kept[i], MASKED ? kept_bits[i] : ~0u);
        for (long long c = tid + KEEP * THREADS; c < chunks; c += THREADS) take_chunk(*(const Some<T> *)(in + lead + c * V), bits_of(lead + c * V));
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const float top = __shfl_xor(s.top, d), sum = __shfl_xor(s.sum, d);
            s.join(top, sum, k);
        }
        if (kWaves > 1) {
            if (lane == 0) tops[wave] = s.top, sums[wave] = s.sum;
            all_here();
            s = Sum{tops[0], sums[0]};
            for (int w = 1; w < kWaves; w++) s.join(tops[w], sums[w], k);
        }
        const float total = logf(s.sum);
        lse = s.top * a.scale + total;
        if (s.sum == 0.f) lse = -INFINITY;
        if (tid == 0) {
            logp = 0.f;
            if (target >= 0 && target < vocab) {
                const float x = allowed(target) ? (float)in[target] : -INFINITY;
                logp = x == -INFINITY ? -INFINITY : (x - s.top) * a.scale - total;
            }
            a.logp[r] = logp;
            a.lse[r] = lse;
        }
    } else {
        lse = a.lse[r];
        if (tid == 0) {
            logp = -INFINITY;
            if (target >= 0 && target < vocab && allowed(target)) {
                const float x = (float)in[target];
                logp = x == -INFINITY ? x : __builtin_fmaf(x, a.scale, -lse);
            }
        }
    }
    if (MODE == kLogp) return;
    if (tid == 0) {
        float loss;
        row_terms(a, r, logp, target >= 0 && target < vocab && logp != -INFINITY, loss, slope);
        if (MODE != kBackward) a.row_loss[r] = loss;
        else if (a.dloss) slope *= *a.dloss;
        said[0] = slope * a.scale;
        said[1] = logp;
    }
    if (MODE == kLoss) return;
    all_here();
    slope = said[0];
    logp = said[1];
    T *out = (T *)a.dlogits + (long long)r * vocab;
    if (slope == 0.f || closed) {  // zeros, whatever the logits are
        const long long lead1 = ((16 - ((uintptr_t)out & 15)) & 15) / sizeof(T), before = lead1 < vocab ? lead1 : vocab, whole = (vocab - before) / V, behind = before + whole * V;
        if (tid < before) out[tid] = (T)0.f;
        if (behind + tid < vocab) out[behind + tid] = (T)0.f;
        for (long long c = tid; c < whole; c += THREADS) *(Some<T> *)(out + before + c * V) = Some<T>{};
        return;
    }
    constexpr int kKept = MODE == kBackward ? 0 : KEEP;
    auto write_row = [&](auto far) __attribute__((always_inline)) {  // (where lse is far from 0, its rounding would be that of the shares)
        const float from = far ? -__log2f(s.sum) : -lse * kLog2e;
        auto share = [&](float x) { return exp2_fast(__builtin_fmaf(far ? x - s.top : x, k, from)) * -slope; };
        auto write_chunk = [&](long long v, const Some<T> &x, unsigned bits) __attribute__((always_inline)) {
            Some<T> y;
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float z = share((float)x[e]);
                y[e] = (T)(MASKED ? by_bit(bits, e, z, 0.f) : z);
            }
            store_some<T>(out + v, y, V);
        };
        if (tid < lead) out[tid] = (T)(allowed(tid) ? share((float)in[tid]) : 0.f);
        if (tail + tid < vocab) out[tail + tid] = (T)(allowed(tail + tid) ? share((float)in[tail + tid]) : 0.f);
#pragma unroll
        for (int i = 0; i < kKept; i++)
            if (tid + i * THREADS < chunks) write_chunk(lead + (long long)(tid + i * THREADS) * V, kept[i], MASKED ? kept_bits[i] : ~0u);
        for (long long c = tid + kKept * THREADS; c < chunks; c += THREADS) write_chunk(lead + c * V, *(const Some<T> *)(in + lead + c * V), bits_of(lead + c * V));
    };
    if (MODE == kBackward || __builtin_fabsf(lse * kLog2e) < kNear) write_row(std::false_type{});
    else write_row(std::true_type{});
    if (THREADS == 64) __threadfence_block();  // (a thread's share of the target is written over)
    all_here();
    if (tid == 0) out[target] = (T)(-slope * expm1f(logp));
}

template <class T, int THREADS, int MODE, bool MASKED, int KEEP> __global__ __launch_bounds__(THREADS, 4) void k_policy(PolicyArgs a) {
    __shared__ RowShared<THREADS> shared;
    policy_row<T, THREADS, MODE, MASKED, KEEP>(a, blockIdx.x, threadIdx.x, shared);
}

// The rows' losses together, in a fixed order.
__device__ __forceinline__ void add_rows(const float *row_loss, int n, float *loss, double *box, int threads) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += threads) sum += row_loss[i];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x) return;
    sum = 0.0;
    for (int w = 0; w < threads / 64; w++) sum += box[w];
    *loss = (float)sum;
}
__global__ __launch_bounds__(256) void k_policy_sum(const float *row_loss, int n, float *loss) {
    __shared__ double box[4];
    add_rows(row_loss, n, loss, box, 256);
}

// Few short rows by one block, a wavefront each at a time, and their sum: one launch less.
constexpr int kFewRows = 64;
template <class T, int MODE, bool MASKED> __global__ __launch_bounds__(1024, 4) void k_policy_few(PolicyArgs a) {
    __shared__ RowShared<64> shared[16];
    __shared__ double box[16];
    const int wave = threadIdx.x >> 6;
    for (int r = wave; r < a.num_rows; r += 16) policy_row<T, 64, MODE, MASKED, 4>(a, r, threadIdx.x & 63, shared[wave]);
    __threadfence_block();
    __syncthreads();
    add_rows(a.row_loss, a.num_rows, a.loss, box, 1024);
}

template <class T, int THREADS, int MODE, bool MASKED, int KEEP> static void launch_rows(const PolicyArgs &a, hipStream_t st) {
    k_policy<T, THREADS, MODE, MASKED, KEEP><<<dim3(a.num_rows), THREADS, 0, st>>>(a);
}

template <class T, int MODE> static logoskg_status launch_policy(const PolicyArgs &a, hipStream_t st) {
    const bool sum = MODE == kLoss || MODE == kLossAndGradient;
    if (sum && a.num_rows <= kFewRows && a.vocab <= 64 * 2 * (16 / (int)sizeof(T))) {
        a.mask ? k_policy_few<T, MODE, true><<<1, 1024, 0, st>>>(a) : k_policy_few<T, MODE, false><<<1, 1024, 0, st>>>(a);
        LKG_HIP(hipGetLastError());
        return LOGOSKG_OK;
    }
    if (a.num_rows) {
        // Threads by the chunks of a row: a wavefront for 4 each (4,096 rows of 2,000 bfloat16 logits 11 us; 128 threads 13, 512 21), 128 or 512
        // for 8 (8,192 rows of 32,000: 192 us with 512, 250 with 1,024), else 1,024, where keeping few chunks is best under masks (2,048 rows of
        // 150,001: 269 us with 2, 345 with 20, most of whose registers are the masks'), and all of long rows without (272 us with 20,
        // 308 with 4; 4,096 rows of 80,000: 278 with 4, 294 with 512 threads).
        const long long chunks = a.vocab / (16 / (int)sizeof(T));
        if (chunks <= 64 * 4) a.mask ? launch_rows<T, 64, MODE, true, 4>(a, st) : launch_rows<T, 64, MODE, false, 4>(a, st);
        else if (chunks <= 128 * 8) a.mask ? launch_rows<T, 128, MODE, true, 8>(a, st) : launch_rows<T, 128, MODE, false, 8>(a, st);
        else if (chunks <= 512 * 8) a.mask ? launch_rows<T, 512, MODE, true, 8>(a, st) : launch_rows<T, 512, MODE, false, 8>(a, st);
        else if (a.mask) launch_rows<T, 1024, MODE, true, 2>(a, st);
        else if (chunks <= 1024 * 10 || chunks > 1024 * 20) launch_rows<T, 1024, MODE, false, 4>(a, st);
        else launch_rows<T, 1024, MODE, false, 20>(a, st);
        LKG_HIP(hipGetLastError());
    }
    if (sum) {
        k_policy_sum<<<1, 256, 0, st>>>(a.row_loss, a.num_rows, a.loss);
        LKG_HIP(hipGetLastError());
    }
    return LOGOSKG_OK;
}
template <class T> static logoskg_status launch_policy(int mode, const PolicyArgs &a, hipStream_t st) {
    return mode == kLogp ? launch_policy<T, kLogp>(a, st) : mode == kLoss ? launch_policy<T, kLoss>(a, st)
         : mode == kLossAndGradient ? launch_policy<T, kLossAndGradient>(a, st) : launch_policy<T, kBackward>(a, st);
}

static const char *policy_args(const logoskg_policy *p, int mode, PolicyArgs *a) {
    if (!p || p->struct_size != sizeof(logoskg_policy)) return "struct_size";
    if (p->dtype < LOGOSKG_F32 || p->dtype > LOGOSKG_F16) return "unknown type";
    if (p->num_rows < 0 || p->vocab < 0 || p->vocab >= (1ll << 31) || p->num_masks < 0 || p->num_masks >= (1ll << 31)) return "a count is out of range";
    if (p->row < 0 || (p->row < p->vocab && p->num_rows > 1)) return "rows overlap";
    if (p->num_rows && ((p->vocab && !p->logits) || !p->target || !p->lse)) return "logits, target or lse is NULL";
    if (!aligned_to(p->logits, p->dtype) || !aligned_to(p->dlogits, p->dtype)) return kUnaligned;
    if (mode != kBackward && p->num_rows && !p->logp) return "logp is NULL";
    if (p->mask && !p->mask_row && p->num_masks < p->num_rows) return "fewer masks than rows";
    if (!(p->scale > 0.f) || p->scale - p->scale != 0.f) return "scale is not above 0";
    if (mode != kLogp) {
        if (!(p->kl >= 0.f) || p->kl - p->kl != 0.f) return "kl is negative";
        if (!(p->clip_low >= 0.f) || !(p->clip_high >= 0.f)) return "a clip is negative";
        if (p->num_rows && !p->advantage) return "advantage is NULL";
        if (p->num_rows && p->kl > 0.f && !p->ref) return "kl without ref";
        if (mode != kBackward && !p->loss) return "loss is NULL";
        if (mode == kBackward && p->num_rows && p->vocab && !p->dlogits) return "dlogits is NULL";
        if (p->dlogits == p->logits && p->dlogits && p->row != p->vocab && p->num_rows > 1) return "dlogits in place of logits with gaps";
    }
    memset(a, 0, sizeof *a);
    a->num_rows = p->num_rows; a->num_masks = (int)p->num_masks; a->vocab = p->vocab; a->row = p->row; a->words = (p->vocab + 63) / 64;
    a->logits = p->logits; a->target = p->target; a->mask = (const u64 *)p->mask; a->mask_row = p->mask_row;
    a->scale = p->scale; a->kl = p->kl; a->low = p->clip_low; a->high = p->clip_high;
    a->advantage = p->advantage; a->old = p->old; a->ref = p->ref; a->weight = p->weight;
    a->logp = p->logp; a->lse = p->lse; a->loss = p->loss; a->dlogits = p->dlogits; a->dloss = p->dloss;
    return nullptr;
}

static long long policy_bytes(const PolicyArgs &a) { return (long long)a.num_rows * 4; }

static logoskg_status policy(const logoskg_policy *p, int mode, const char *call) {
    PolicyArgs a;
    if (mode == kLoss && p && p->dlogits) mode = kLossAndGradient;
    if (const char *why = policy_args(p, mode, &a)) { set_error("%s: %s", call, why); return LOGOSKG_EINVAL; }
    if (mode == kLoss || mode == kLossAndGradient) {
        if (p->workspace_bytes < policy_bytes(a) || (policy_bytes(a) && !p->workspace) || ((uintptr_t)p->workspace & 15)) {
            set_error("%s: the workspace has %lld of %lld bytes, or is not 16-byte aligned", call, (long long)p->workspace_bytes, policy_bytes(a));
            return LOGOSKG_ERANGE;
        }
        a.row_loss = (float *)p->workspace;
    }
    OnDevice on;
    LKG_TRY(on.go(p->device));
    hipStream_t st = (hipStream_t)p->stream;
    if (p->dtype == LOGOSKG_F32) return launch_policy<float>(mode, a, st);
    return p->dtype == LOGOSKG_BF16 ? launch_policy<bf16>(mode, a, st) : launch_policy<fp16>(mode, a, st);
}

}  // namespace lkg

using namespace lkg;

extern "C" logoskg_status logoskg_token_logp(const logoskg_policy *p) { return policy(p, kLogp, "logoskg_token_logp"); }
extern "C" int64_t logoskg_policy_loss_bytes(const logoskg_policy *p) {
    PolicyArgs a;
    if (const char *why = policy_args(p, kLoss, &a)) { set_error("logoskg_policy_loss_bytes: %s", why); return -1; }
    return policy_bytes(a);
}
extern "C" logoskg_status logoskg_policy_loss(const logoskg_policy *p) { return policy(p, kLoss, "logoskg_policy_loss"); }
extern "C" logoskg_status logoskg_policy_loss_backward(const logoskg_policy *p) { return policy(p, kBackward, "logoskg_policy_loss_backward"); }
