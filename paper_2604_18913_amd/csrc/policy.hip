// The loss of sampled answers over their logits, and its gradient (logoskg_token_logp, logoskg_policy_loss,
// logoskg_policy_loss_backward).
#include "training.h"

namespace lkg {

static_assert(sizeof(logoskg_policy) == 168, "the ctypes binding mirrors this layout");

typedef unsigned long long u64;

struct PolicyArgs {
    int num_rows, num_masks, first;  // first: row of a launch
    long long vocab, row, words;
    const void *logits;
    const int32_t *target, *mask_row;
    const u64 *mask;
    float scale, kl, low, high;
    const float *advantage, *old, *ref, *weight;
    float *logp, *lse, *loss;
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

// What stands beside a row: asked for at its begin, used at its end.
struct Beside { float advantage, old, ref, weight; };
__device__ __forceinline__ Beside beside(const PolicyArgs &a, int r) {
    return Beside{a.advantage[r], a.old ? a.old[r] : 0.f, a.kl > 0.f ? a.ref[r] : 0.f, a.weight ? a.weight[r] : 1.f};
}
// Rows that pad, whose answer cannot be or that weigh nothing do not count: their loss and gradient are 0 whatever stands beside them.
__device__ __forceinline__ bool row_counts(const PolicyArgs &a, const Beside &row, int target, float logp) {
    return target >= 0 && target < a.vocab && logp != -INFINITY && row.weight != 0.f;
}
// A row's loss and what its logp's gradient is, weight included; 0 and 0 for rows that do not count.
__device__ __forceinline__ void row_terms(const PolicyArgs &a, const Beside &row, float logp, bool counts, float &loss, float &slope) {
    loss = slope = 0.f;
    if (!counts) return;
    const float A = row.advantage, w = row.weight;
    if (A != 0.f) {  // (an infinite ratio times 0 is nothing, too)
        const float ratio = a.old ? expf(logp - row.old) : 1.f;
        const float near = fminf(fmaxf(ratio, 1.f - a.low), 1.f + a.high), inside = ratio * A, border = near * A;
        if (inside <= border || inside != inside) loss = -inside, slope = -inside;
        else loss = -border;
    }
    if (a.kl > 0.f) {
        const float d = row.ref - logp, e = expm1f(d);
        loss += a.kl * (e - d);
        slope -= a.kl * e;
    }
    loss *= w;
    slope *= w;
}

// Exponents up to this size, in units of log 2, are made in one step, x k minus a product that is rounded before: 2^-19 of the exponential
// at most.
constexpr float kNear = 64.f;

// x where the bit is set, `other` where it is not: of a bit as a whole word two instructions
__device__ __forceinline__ float by_bit(unsigned bits, int e, float x, float other) {
    const unsigned m = (unsigned)__builtin_amdgcn_sbfe((int)bits, e, 1);
    return __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, x) & m) | (__builtin_bit_cast(unsigned, other) & ~m));
}

// A chunk with -infinity where its bits are not set: pairs of 16-bit elements as a word.
template <class T> __device__ __forceinline__ Some<T> hidden_by(unsigned bits, Some<T> x) {
    constexpr int V = 16 / sizeof(T);
    if (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < V; e++) x[e] = (T)by_bit(bits, e, (float)x[e], -INFINITY);
        return x;
    }
    u32x4 w = __builtin_bit_cast(u32x4, x);
    const unsigned hidden = std::is_same<T, bf16>::value ? 0xff80ff80u : 0xfc00fc00u;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const unsigned lo = (unsigned)__builtin_amdgcn_sbfe((int)bits, 2 * i, 1), hi = (unsigned)__builtin_amdgcn_sbfe((int)bits, 2 * i + 1, 1), m = (lo & 0xffffu) | (hi & 0xffff0000u);
        w[i] = (w[i] & m) | (hidden & ~m);
    }
    return __builtin_bit_cast(Some<T>, w);
}

// Keeps a chunk as it is: of one that is used again the compiler would keep every element in 32 bits instead.
template <class T> __device__ __forceinline__ void keep(Some<T> &x) {
    u32x4 w = __builtin_bit_cast(u32x4, x);
    asm volatile("" : "+v"(w));
    x = __builtin_bit_cast(Some<T>, w);
}

// One row by THREADS threads: a sweep over its logits for the largest and the sum, another for the gradient.  The first KEEP
// chunks of a thread are asked for at once and stay in registers for the second sweep.  WHOLE: they are all that there are; then the
// largest is found first, and the row's mask stands in LDS, from the first whole chunk's ids on.
template <class T, int THREADS, int MODE, bool MASKED, int KEEP, bool WHOLE> struct RowShared {
    static constexpr int kStaged = MASKED && WHOLE ? THREADS * KEEP * (16 / (int)sizeof(T)) / 32 : 1;
    unsigned staged[kStaged];
    float tops[(THREADS + 63) / 64], sums[(THREADS + 63) / 64], said[2];
};
template <class T, int THREADS, int MODE, bool MASKED, int KEEP, bool WHOLE> __device__ __forceinline__ void policy_row(const PolicyArgs &a, int r, int tid, RowShared<T, THREADS, MODE, MASKED, KEEP, WHOLE> &shared) {
    constexpr int V = 16 / sizeof(T), kWaves = THREADS / 64;
    constexpr bool kStaged = MASKED && WHOLE;
    const int lane = tid & 63, wave = tid >> 6;
    float *tops = shared.tops, *sums = shared.sums, *said = shared.said;
    auto all_here = [] {  // (rows of a wavefront or a part of one need no more than its own order)
        if (THREADS <= 64) wave_sync();
        else __syncthreads();
    };
    // (places in a row are 32-bit, in bytes)
    const T *in = (const T *)a.logits + (long long)r * a.row;
    const unsigned vocab = (unsigned)a.vocab;
    const int target = a.target[r];
    Beside row = {};
    if (MODE != kLogp) row = beside(a, r);
    const long long mask_at = !MASKED ? 0 : a.mask_row ? a.mask_row[r] : r;
    const bool closed = MASKED && (mask_at < 0 || mask_at >= a.num_masks);  // (such a row's mask is not read: nothing is allowed)
    const u64 *mask = MASKED && !closed ? a.mask + mask_at * a.words : nullptr;
    const float k = a.scale * kLog2e;
    const unsigned lead0 = (unsigned)((16 - ((uintptr_t)in & 15)) & 15) / sizeof(T), lead = lead0 < vocab ? lead0 : vocab;
    const unsigned chunks = closed ? 0 : (vocab - lead) / V, tail = lead + (vocab - lead) / V * V;
    auto allowed = [&](unsigned v) { return !MASKED || (!closed && (mask[v >> 6] >> (v & 63) & 1)); };
    typedef unsigned short __attribute__((aligned(1))) two_bytes;
    const unsigned last = (unsigned)a.words * 8 - 2;
    auto chunk_at = [&](unsigned c) { return *(const Some<T> *)((const char *)(in + lead) + c * 16u); };
    auto bits_at = [&](unsigned c) -> unsigned {  // of the V ids of chunk c, and others above: the two bytes that they stand in
        if (!MASKED) return ~0u;
        if (kStaged) return ((const unsigned char *)shared.staged)[c * V / 8] >> (c * V % 8);
        const unsigned v = lead + c * V, at = v >> 3 < last ? v >> 3 : last;
        return (unsigned)*(const two_bytes *)((const char *)mask + at) >> (v - 8 * at);
    };
    Some<T> kept[KEEP], nothing;
#pragma unroll
    for (int e = 0; e < V; e++) nothing[e] = (T)-INFINITY;
    // the mask's words first, then the chunks, so that the mask can be put away while those are on their way
    constexpr int kWords = kStaged ? (RowShared<T, THREADS, MODE, MASKED, KEEP, WHOLE>::kStaged + THREADS - 1) / THREADS : 1;
    unsigned lo[kWords], hi[kWords];
    const unsigned staged = closed ? 0 : (chunks * V + 31) / 32;
    if (kStaged) {
        const unsigned *words = (const unsigned *)mask, most = (unsigned)a.words * 2 - 1;  // (of a word behind the last no bit is looked at)
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const unsigned j = tid + i * THREADS;
            if (j < staged) lo[i] = words[j], hi[i] = words[j + 1 < most ? j + 1 : most];
        }
    }
    if (MODE != kBackward) {
#pragma unroll
        for (int i = 0; i < KEEP; i++)
            if (tid + i * THREADS < chunks) kept[i] = chunk_at(tid + i * THREADS);
            else if (WHOLE) kept[i] = nothing;
    }
    if (kStaged) {
#pragma unroll
        for (int i = 0; i < kWords; i++) {
            const unsigned j = tid + i * THREADS;
            if (j < staged) shared.staged[j] = lead == 0 ? lo[i] : lo[i] >> lead | hi[i] << (32 - lead);
        }
        all_here();
    }
    float said_x = (unsigned)target < vocab && allowed(target) ? (float)in[target] : -INFINITY;  // (asked for behind the chunks, here by the row's end)
    asm volatile("" : "+v"(said_x));
    Sum s = {-INFINITY, 0.f};
    float lse, logp, slope;
    // Where lse is far from 0, its rounding would be that of shares and of logp (2^-24 of 1,000: 6e-5 of a share): these are made of the
    // largest and the sum, and the backward, which is given lse alone, makes those again.  (Such rows of 150,001 bfloat16 logits, 2,048 of
    // them: 320 us, others 248; under masks 243 and 208; 8,192 of 32,000 255 and 205.)
    bool far = false;
    if (MODE == kBackward) {
        lse = a.lse[r];
        far = said_x != -INFINITY && !(__builtin_fabsf(lse * kLog2e) < kNear);
    }
    if (MODE != kBackward || far) {
        auto take = [&](float x) { s.join(x, x == -INFINITY ? 0.f : 1.f, k); };
        if ((unsigned)tid < lead && allowed(tid)) take((float)in[tid]);
        if (tail + tid < vocab && allowed(tail + tid)) take((float)in[tail + tid]);
        // N chunks together
        auto take_chunks = [&](auto count, const Some<T> *x, const unsigned *bits) __attribute__((always_inline)) {
            constexpr int N = decltype(count)::value;
            float y[N * V], top = s.top;
#pragma unroll
            for (int e = 0; e < N * V; e++) {
                y[e] = (float)x[e / V][e % V];
                if (MASKED) y[e] = by_bit(bits[e / V], e % V, y[e], -INFINITY);
                top = fmaxf(top, y[e]);
            }
            const float at = top == -INFINITY ? 0.f : top, from = -at * k;
            float sum = s.sum * exp2_fast((s.top - at) * k);
            if (__builtin_expect(__builtin_fabsf(from) < kNear, 1)) {
#pragma unroll
                for (int e = 0; e < N * V; e++) sum += exp2_fast(__builtin_fmaf(y[e], k, from));
            } else {
#pragma unroll
                for (int e = 0; e < N * V; e++) sum += exp2_fast((y[e] - at) * k);
            }
            s.top = top, s.sum = sum;
        };
        if (WHOLE && MODE != kBackward) {  // the largest of all first; what is hidden becomes -infinity in place, for the second sweep too
            float top = s.top;
#pragma unroll
            for (int i = 0; i < KEEP; i++) {
                if (MASKED) kept[i] = hidden_by<T>(bits_at(tid + i * THREADS), kept[i]);
#pragma unroll
                for (int e = 0; e < V; e++) top = fmaxf(top, (float)kept[i][e]);
                keep<T>(kept[i]);
            }
            const float at = top == -INFINITY ? 0.f : top, from = -at * k;
            float sum[4] = {s.sum * exp2_fast((s.top - at) * k), 0.f, 0.f, 0.f};
            if (__builtin_fabsf(from) < kNear) {
#pragma unroll
                for (int i = 0; i < KEEP; i++) {
#pragma unroll
                    for (int e = 0; e < V; e++) sum[e & 3] += exp2_fast(__builtin_fmaf((float)kept[i][e], k, from));
                    keep<T>(kept[i]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < KEEP; i++) {
#pragma unroll
                    for (int e = 0; e < V; e++) sum[e & 3] += exp2_fast(((float)kept[i][e] - at) * k);
                    keep<T>(kept[i]);
                }
            }
            s.top = top, s.sum = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        } else if (MODE != kBackward) {
#pragma unroll
            for (int i = 0; i < KEEP; i++)
                if (tid + i * THREADS < chunks) {
                    const unsigned bits = bits_at(tid + i * THREADS);
                    take_chunks(std::integral_constant<int, 1>{}, &kept[i], &bits);
                }
        }
        constexpr bool kRest = !WHOLE || MODE == kBackward;
        unsigned c = tid + (MODE == kBackward ? 0 : KEEP * THREADS);
        for (; kRest && c + THREADS < chunks; c += 2 * THREADS) {
            const Some<T> x[2] = {chunk_at(c), chunk_at(c + THREADS)};
            const unsigned bits[2] = {bits_at(c), bits_at(c + THREADS)};
            take_chunks(std::integral_constant<int, 2>{}, x, bits);
        }
        if (kRest && c < chunks) {
            const Some<T> x = chunk_at(c);
            const unsigned bits = bits_at(c);
            take_chunks(std::integral_constant<int, 1>{}, &x, &bits);
        }
#pragma unroll
        for (int d = THREADS < 64 ? THREADS / 2 : 32; d > 0; d >>= 1) {
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
        if (MODE != kBackward) far = !(__builtin_fabsf(lse * kLog2e) < kNear);
        if (tid == 0) {
            logp = 0.f;
            if ((unsigned)target < vocab) logp = said_x == -INFINITY ? -INFINITY : (said_x - s.top) * a.scale - total;
            if (MODE != kBackward) {
                a.logp[r] = logp;
                a.lse[r] = lse;
            }
        }
    } else if (tid == 0) {
        logp = said_x == -INFINITY ? -INFINITY : __builtin_fmaf(said_x, a.scale, -lse);
    }
    if (MODE == kLogp) return;
    if (tid == 0) {
        float loss;
        const bool counts = row_counts(a, row, target, logp);
        row_terms(a, row, logp, counts, loss, slope);
        if (MODE == kBackward && a.dloss) slope *= *a.dloss;  // (it may be infinite or NaN, and this NaN of a row that does not count)
        said[0] = slope * a.scale;
        said[1] = counts ? logp : -INFINITY;
    }
    if (MODE == kLoss) return;
    all_here();
    slope = said[0];
    logp = said[1];
    T *out = (T *)a.dlogits + (long long)r * vocab;
    if (logp == -INFINITY || slope == 0.f) {  // zeros, whatever the logits are; behind this the target is an id
        const unsigned lead1 = (unsigned)((16 - ((uintptr_t)out & 15)) & 15) / sizeof(T), before = lead1 < vocab ? lead1 : vocab, whole = (vocab - before) / V, behind = before + whole * V;
        if ((unsigned)tid < before) out[tid] = (T)0.f;
        if (behind + tid < vocab) out[behind + tid] = (T)0.f;
        for (unsigned c = tid; c < whole; c += THREADS) *(Some<T> *)((char *)(out + before) + c * 16u) = Some<T>{};
        return;
    }
    constexpr int kKept = MODE == kBackward ? 0 : KEEP;
    auto write_row = [&](auto far) __attribute__((always_inline)) {
        const float from = far ? -__log2f(s.sum) : -lse * kLog2e;
        auto share = [&](float x) { return exp2_fast(__builtin_fmaf(far ? x - s.top : x, k, from)) * -slope; };
        constexpr bool kHide = MASKED && !(WHOLE && kKept > 0);  // (else it is hidden already)
        auto write_chunk = [&](unsigned c, const Some<T> &x) __attribute__((always_inline)) {
            const unsigned bits = kHide ? bits_at(c) : 0;
            Some<T> y;
#pragma unroll
            for (int e = 0; e < V; e++) {
                const float z = share((float)x[e]);
                y[e] = (T)(kHide ? by_bit(bits, e, z, 0.f) : z);
            }
            *(typename Loose<T>::type *)((char *)(out + lead) + c * 16u) = y;
        };
        if ((unsigned)tid < lead) out[tid] = (T)(allowed(tid) ? share((float)in[tid]) : 0.f);
        if (tail + tid < vocab) out[tail + tid] = (T)(allowed(tail + tid) ? share((float)in[tail + tid]) : 0.f);
#pragma unroll
        for (int i = 0; i < kKept; i++)
            if (tid + i * THREADS < chunks) write_chunk(tid + i * THREADS, kept[i]);
        unsigned c = tid + kKept * THREADS;
        for (; (!WHOLE || kKept == 0) && c + THREADS < chunks; c += 2 * THREADS) {
            const Some<T> x[2] = {chunk_at(c), chunk_at(c + THREADS)};
            write_chunk(c, x[0]), write_chunk(c + THREADS, x[1]);
        }
        if ((!WHOLE || kKept == 0) && c < chunks) write_chunk(c, chunk_at(c));
    };
    if (far) write_row(std::true_type{});
    else write_row(std::false_type{});
    auto written = [&] {  // before others write over it
        if (THREADS <= 64) __threadfence_block();
        all_here();
    };
    written();
    if (MASKED && WHOLE && kKept > 0 && !(lse - lse == 0.f && slope - slope == 0.f)) {  // what is hidden has come through the products as NaN
        for (unsigned v = tid; v < vocab; v += THREADS)
            if (!allowed(v)) out[v] = (T)0.f;
        written();
    }
    if (tid == 0) out[target] = (T)(-slope * expm1f(logp));
}

template <class T, int THREADS, int MODE, bool MASKED, int KEEP, bool WHOLE> __global__ __launch_bounds__(THREADS, 4) void k_policy(PolicyArgs a) {
    __shared__ RowShared<T, THREADS, MODE, MASKED, KEEP, WHOLE> shared;
    policy_row<T, THREADS, MODE, MASKED, KEEP, WHOLE>(a, a.first + blockIdx.x, threadIdx.x, shared);
}

// The rows' losses, made again of their logp, and their sum in a fixed order.  (One block's: 2 us, of 500,000 rows 165, and 325
// where a thread asks for one row at a time.)
template <int THREADS> __device__ __forceinline__ void add_rows(const PolicyArgs &a, double *box) {
    double sum = 0.0;
    auto add = [&](int target, float logp, const Beside &row) {
        float loss, slope;
        row_terms(a, row, logp, row_counts(a, row, target, logp), loss, slope);
        sum += loss;
    };
    int r = threadIdx.x;
    constexpr int kTogether = 8;
    for (; r < a.num_rows - (kTogether - 1) * THREADS; r += kTogether * THREADS) {  // asked for together: one block has all the rows
        int target[kTogether];
        float logp[kTogether];
        Beside row[kTogether];
#pragma unroll
        for (int i = 0; i < kTogether; i++) target[i] = a.target[r + i * THREADS], logp[i] = a.logp[r + i * THREADS], row[i] = beside(a, r + i * THREADS);
#pragma unroll
        for (int i = 0; i < kTogether; i++) add(target[i], logp[i], row[i]);
    }
    for (; r < a.num_rows; r += THREADS) add(a.target[r], a.logp[r], beside(a, r));
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x) return;
    sum = 0.0;
    for (int w = 0; w < THREADS / 64; w++) sum += box[w];
    *a.loss = (float)sum;
}
__global__ __launch_bounds__(1024) void k_policy_sum(PolicyArgs a) {
    __shared__ double box[16];
    add_rows<1024>(a, box);
}

// Short rows, 16 lanes each.  Few of them by one block, their sum with them: one launch less.  (64 rows of 500 logits 7.5 us; a
// wavefront each, four rows one after the other, 15.2; a block each, and the sum behind them, 4.4 and 3.5, and the host's 3 of a
// launch.  Many rows: 2,000,000 of 64 logits 850 us with a wavefront each, 290 so; from 500 logits on they are alike.)
constexpr int kShortLanes = 16, kShortChunks = 8, kFewRows = 1024 / kShortLanes;
template <class T, int MODE, bool MASKED, int THREADS, bool SUM> __global__ __launch_bounds__(THREADS, 4) void k_policy_short(PolicyArgs a) {
    constexpr int L = kShortLanes;
    __shared__ RowShared<T, L, MODE, MASKED, kShortChunks, true> shared[THREADS / L];
    __shared__ double box[THREADS / 64];
    const int r = a.first + blockIdx.x * (THREADS / L) + threadIdx.x / L;
    if (r < a.num_rows) policy_row<T, L, MODE, MASKED, kShortChunks, true>(a, r, threadIdx.x % L, shared[threadIdx.x / L]);
    if (!SUM) return;
    __threadfence_block();
    __syncthreads();
    add_rows<THREADS>(a, box);
}

// A block a row, in launches of fewer than 2^32 threads.
template <class T, int THREADS, int MODE, bool MASKED, int KEEP, bool WHOLE> static void launch_rows(PolicyArgs a, hipStream_t st) {
    launch_ranges(a.num_rows, 1, [&](long long first, long long n) {
        a.first = (int)first;
        k_policy<T, THREADS, MODE, MASKED, KEEP, WHOLE><<<dim3((unsigned)n), THREADS, 0, st>>>(a);
    }, (long long)UINT32_MAX / THREADS);
}
template <class T, int THREADS, int MODE, int KEEP> static void launch_rows(const PolicyArgs &a, hipStream_t st) {
    a.mask ? launch_rows<T, THREADS, MODE, true, KEEP, true>(a, st) : launch_rows<T, THREADS, MODE, false, KEEP, true>(a, st);
}
template <class T, int MODE> static void launch_short_rows(PolicyArgs a, hipStream_t st) {
    constexpr int kRows = 256 / kShortLanes;
    launch_ranges(a.num_rows, kRows, [&](long long first, long long n) {
        a.first = (int)first;
        const dim3 blocks((unsigned)((n + kRows - 1) / kRows));
        a.mask ? k_policy_short<T, MODE, true, 256, false><<<blocks, 256, 0, st>>>(a) : k_policy_short<T, MODE, false, 256, false><<<blocks, 256, 0, st>>>(a);
    });
}

template <class T, int MODE> static logoskg_status launch_policy(const PolicyArgs &a, hipStream_t st) {
    const bool sum = MODE == kLoss || MODE == kLossAndGradient;
    const long long chunks = a.vocab / (16 / (int)sizeof(T));
    if (sum && a.num_rows <= kFewRows && chunks <= kShortLanes * kShortChunks) {
        a.mask ? k_policy_short<T, MODE, true, 1024, true><<<1, 1024, 0, st>>>(a) : k_policy_short<T, MODE, false, 1024, true><<<1, 1024, 0, st>>>(a);
        LKG_HIP(hipGetLastError());
        return LOGOSKG_OK;
    }
    if (a.num_rows) {
        // By the chunks of a row.  Whole rows in registers where they are short or no mask takes its share of instructions: 8,192 rows of
        // 32,000 bfloat16 logits under masks 208 us (264 in two sweeps), 2,048 rows of 150,001 without 284 (317), 4,096 of 80,000 without
        // 261 (272).  Long rows under masks in two sweeps over memory, two blocks of a unit in turn: 4,096 of 80,000 298 us (318 in registers,
        // where one block fits and its loads, exponentials and stores take turns), 2,048 of 150,001 332 (334).
        if (chunks <= kShortLanes * kShortChunks) launch_short_rows<T, MODE>(a, st);
        else if (chunks <= 64 * 4) launch_rows<T, 64, MODE, 4>(a, st);
        else if (chunks <= 256 * 4) launch_rows<T, 256, MODE, 4>(a, st);
        else if (chunks <= 256 * 16) launch_rows<T, 256, MODE, 16>(a, st);
        else if (a.mask) launch_rows<T, 1024, MODE, true, 2, false>(a, st);
        else if (chunks <= 1024 * 10) launch_rows<T, 1024, MODE, false, 10, true>(a, st);
        else if (chunks <= 1024 * 20) launch_rows<T, 1024, MODE, false, 20, true>(a, st);
        else launch_rows<T, 1024, MODE, false, 4, false>(a, st);
        LKG_HIP(hipGetLastError());
    }
    if (sum) {
        k_policy_sum<<<1, 1024, 0, st>>>(a);
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
    // (rows are counted in 32 bits, by steps of up to 2^13 behind the last)
    if (p->num_rows < 0 || p->num_rows > INT32_MAX - (1 << 16) || p->vocab < 0 || p->vocab * size_of(p->dtype) >= (1ll << 32) - (1 << 20) || p->vocab >= (1ll << 31) - (1 << 16) || p->num_masks < 0 || p->num_masks >= (1ll << 31)) return "a count is out of range";
    if (p->row < 0 || (p->row < p->vocab && p->num_rows > 1)) return "rows overlap";
    if (p->num_rows && ((p->vocab && !p->logits) || !p->target || !p->lse)) return "logits, target or lse is NULL";
    if (!aligned_to(p->logits, p->dtype) || !aligned_to(p->dlogits, p->dtype)) return kUnaligned;
    if (mode != kBackward && p->num_rows && !p->logp) return "logp is NULL";
    if (p->mask && !p->mask_row && p->num_masks < p->num_rows) return "fewer masks than rows";
    if (!(p->scale > 0.f) || p->scale - p->scale != 0.f) return "scale is not above 0";
    if (p->scale > 2e38f) return "scale is above 2e38";  // (times log2 e it is finite)
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

static logoskg_status policy(const logoskg_policy *p, int mode, const char *call) {
    PolicyArgs a;
    if (mode == kLoss && p && p->dlogits) mode = kLossAndGradient;
    if (const char *why = policy_args(p, mode, &a)) { set_error("%s: %s", call, why); return LOGOSKG_EINVAL; }
    OnDevice on;
    LKG_TRY(on.go(p->device));
    hipStream_t st = (hipStream_t)p->stream;
    if (p->dtype == LOGOSKG_F32) return launch_policy<float>(mode, a, st);
    return p->dtype == LOGOSKG_BF16 ? launch_policy<bf16>(mode, a, st) : launch_policy<fp16>(mode, a, st);
}

}  // namespace lkg

using namespace lkg;

extern "C" logoskg_status logoskg_token_logp(const logoskg_policy *p) { return policy(p, kLogp, "logoskg_token_logp"); }
extern "C" logoskg_status logoskg_policy_loss(const logoskg_policy *p) { return policy(p, kLoss, "logoskg_policy_loss"); }
extern "C" logoskg_status logoskg_policy_loss_backward(const logoskg_policy *p) { return policy(p, kBackward, "logoskg_policy_loss_backward"); }
