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

// One row by a block (or a part of a block) of THREADS threads: a sweep over its logits for the largest and the sum, another for
// the gradient.
template <class T, int THREADS, int MODE> __global__ __launch_bounds__(THREADS) void k_policy(PolicyArgs a) {
    constexpr int V = 16 / sizeof(T), kWaves = THREADS / 64;
    __shared__ float tops[kWaves], sums[kWaves], said[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = blockIdx.x;
    const T *in = (const T *)a.logits + (long long)r * a.row;
    const long long vocab = a.vocab;
    const int target = a.target[r];
    const long long mask_at = !a.mask ? 0 : a.mask_row ? a.mask_row[r] : r;
    const bool closed = a.mask && (mask_at < 0 || mask_at >= a.num_masks);
    const u64 *mask = a.mask && !closed ? a.mask + mask_at * a.words : nullptr;
    const float k = a.scale * kLog2e;
    const long long lead0 = ((16 - ((uintptr_t)in & 15)) & 15) / sizeof(T), lead = lead0 < vocab ? lead0 : vocab;
    const long long chunks = (vocab - lead) / V, tail = lead + chunks * V;
    auto allowed = [&](long long v) { return !closed && (!mask || (mask[v >> 6] >> (v & 63) & 1)); };
    auto bits_of = [&](long long v) -> unsigned {  // of the V ids from v on
        if (closed) return 0;
        if (!mask) return ~0u;
        const int sh = (int)(v & 63);
        u64 m = mask[v >> 6] >> sh;
        if (sh > 64 - V) m |= mask[(v >> 6) + 1] << (64 - sh);
        return (unsigned)m;
    };
    auto counts = [&](float logp) { return target >= 0 && target < vocab && logp != -INFINITY; };
    float lse, logp, slope;
    if (MODE != kBackward) {
        Sum s = {-INFINITY, 0.f};
        auto take = [&](float x) { s.join(x, x == -INFINITY ? 0.f : 1.f, k); };
        if (tid < lead && allowed(tid)) take((float)in[tid]);
        if (tail + tid < vocab && allowed(tail + tid)) take((float)in[tail + tid]);
        for (long long c = tid; c < chunks; c += THREADS) {
            const long long v = lead + c * V;
            const Some<T> x = *(const Some<T> *)(in + v);
            const unsigned bits = bits_of(v);
            float y[V], top = s.top;
#pragma unroll
            for (int e = 0; e < V; e++) {
                y[e] = bits >> e & 1 ? (float)x[e] : -INFINITY;
                top = fmaxf(top, y[e]);
            }
            const float at = top == -INFINITY ? 0.f : top;
            float sum = s.sum * exp2_fast((s.top - at) * k);
#pragma unroll
            for (int e = 0; e < V; e++) sum += exp2_fast((y[e] - at) * k);
            s.top = top, s.sum = sum;
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            const float top = __shfl_xor(s.top, d), sum = __shfl_xor(s.sum, d);
            s.join(top, sum, k);
        }
        if (kWaves > 1) {
            if (lane == 0) tops[wave] = s.top, sums[wave] = s.sum;
            __syncthreads();
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
        row_terms(a, r, logp, counts(logp), loss, slope);
        if (MODE != kBackward) a.row_loss[r] = loss;
        else if (a.dloss) slope *= *a.dloss;
        said[0] = slope * a.scale;
        said[1] = logp;
    }
    if (MODE == kLoss) return;
    __syncthreads();
    slope = said[0];
    logp = said[1];
    T *out = (T *)a.dlogits + (long long)r * vocab;
    const float base = lse == -INFINITY ? 0.f : lse;
    const bool any = slope != 0.f;
    auto share = [&](float x) { return any && x != -INFINITY ? -slope * exp2_fast(__builtin_fmaf(x, a.scale, -base) * kLog2e) : 0.f; };
    if (tid < lead) out[tid] = (T)(allowed(tid) ? share((float)in[tid]) : 0.f);
    if (tail + tid < vocab) out[tail + tid] = (T)(allowed(tail + tid) ? share((float)in[tail + tid]) : 0.f);
    for (long long c = tid; c < chunks; c += THREADS) {
        const long long v = lead + c * V;
        const Some<T> x = *(const Some<T> *)(in + v);
        const unsigned bits = bits_of(v);
        Some<T> y;
#pragma unroll
        for (int e = 0; e < V; e++) y[e] = (T)(bits >> e & 1 ? share((float)x[e]) : 0.f);
        store_some<T>(out + v, y, V);
    }
    __syncthreads();  // (a thread's share of the target is written over)
    if (tid == 0 && any) out[target] = (T)(-slope * expm1f(logp));
}

__global__ __launch_bounds__(256) void k_policy_sum(const float *row_loss, int n, float *loss) {
    __shared__ double box[4];
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) sum += row_loss[i];
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) *loss = (float)(box[0] + box[1] + box[2] + box[3]);
}

template <class T, int MODE> static logoskg_status launch_policy(const PolicyArgs &a, hipStream_t st) {
    if (a.num_rows) {
        if (a.vocab <= 4096) k_policy<T, 64, MODE><<<dim3(a.num_rows), 64, 0, st>>>(a);
        else k_policy<T, 512, MODE><<<dim3(a.num_rows), 512, 0, st>>>(a);
        LKG_HIP(hipGetLastError());
    }
    if (MODE == kLoss || MODE == kLossAndGradient) {
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
