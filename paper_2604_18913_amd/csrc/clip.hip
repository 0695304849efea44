// The norm of a step's gradients together, and the gradients brought to it (logoskg_clip_gradients).
#include "training.h"

#include <algorithm>
#include <new>
#include <vector>

namespace lkg {

static_assert(sizeof(logoskg_gradient) == 32, "the ctypes binding mirrors this layout");

constexpr int kClipList = 64;           // tensors of a launch: they travel in its arguments
constexpr long long kClipChunk = 8192;  // elements
constexpr int kClipBlocks = 2048;       // of a launch, at most
constexpr int kClipEach = 4096;         // sums that every block adds up again, which spares a launch
constexpr int kClipTop = 2;             // doubles in front of the blocks' sums: the factor

struct ClipArgs {
    int count, first;        // of the list; place of the launch's first block among the sums
    long long chunks;        // of all tensors of the launch
    double *sums;
    const void *grad[kClipList];
    void *out[kClipList];
    long long n[kClipList];
    int begin[kClipList + 1];       // first chunk of each
    unsigned char type[kClipList], out_type[kClipList];
};
static_assert(sizeof(ClipArgs) < 4000, "a launch's arguments");

__device__ __forceinline__ int tensor_of(const ClipArgs &a, long long chunk) {
    int lo = 0, hi = a.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.begin[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// The squares of a chunk in 64 bits: no size of a gradient overflows, and the sum of billions keeps its bits.  Memory bounds this and the
// scaling: 770 million bfloat16 gradients (1.54 GB) 304 us, and 826 into 32 bits (4.6 GB), 5.1 and 5.6 TB/s.  (The second pass from behind, where caches
// may have a part: nothing; all loads of a chunk before its squares: 304 -> 336.)
template <class T> __device__ __forceinline__ double squares(const T *g, long long n, int tid) {
    constexpr int V = 16 / sizeof(T);
    double sum = 0.0;
    for (long long i = (long long)tid * V; i < n; i += 256 * V) {
        const Some<T> x = load_some<T>(g + i, n - i < V ? (int)(n - i) : V);
#pragma unroll
        for (int e = 0; e < V; e++) sum += (double)(float)x[e] * (double)(float)x[e];
    }
    return sum;
}

__device__ __forceinline__ double block_sum(double sum, double *box) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) box[threadIdx.x >> 6] = sum;
    __syncthreads();
    return box[0] + box[1] + box[2] + box[3];
}

__global__ __launch_bounds__(256) void k_clip_squares(ClipArgs a) {
    __shared__ double box[4];
    double sum = 0.0;
    for (long long c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int t = tensor_of(a, c);
        const long long from = (c - a.begin[t]) * kClipChunk, n = a.n[t] - from < kClipChunk ? a.n[t] - from : kClipChunk;
        if (a.type[t] == LOGOSKG_F32) sum += squares((const float *)a.grad[t] + from, n, threadIdx.x);
        else if (a.type[t] == LOGOSKG_BF16) sum += squares((const bf16 *)a.grad[t] + from, n, threadIdx.x);
        else sum += squares((const fp16 *)a.grad[t] + from, n, threadIdx.x);
    }
    sum = block_sum(sum, box);
    if (threadIdx.x == 0) a.sums[kClipTop + a.first + blockIdx.x] = sum;
}

// The norm and the factor of the blocks' sums, in every thread.
__device__ __forceinline__ double factor_of(const double *sums, int n, float max_norm, float scale, double *box, double &norm) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < n; i += 256) sum += sums[kClipTop + i];
    norm = sqrt(block_sum(sum, box)) * fabs((double)scale);
    return norm <= (double)max_norm ? (double)scale : (double)scale * ((double)max_norm / norm);
}
__global__ __launch_bounds__(256) void k_clip_norm(double *sums, int n, float max_norm, float scale, float *norm) {
    __shared__ double box[4];
    double got, by = factor_of(sums, n, max_norm, scale, box, got);
    if (threadIdx.x == 0) *norm = (float)got, sums[0] = by;
}

// The factor in 32 bits: `by` alone, or where it is below the normal numbers, which would leave it few bits, 2^-100 and 2^100 times it in turn.
// (Gradients below 2^-26 lose bits by 2^-100; their product is below 2^-152 and 0.)
struct Factor { float first, by; };
template <class T, class O> __device__ __forceinline__ void scaled(const T *g, O *out, long long n, Factor f, int tid) {
    constexpr int V = 16 / (sizeof(T) > sizeof(O) ? sizeof(T) : sizeof(O));  // elements at a time: 16 bytes of the wider type
    typedef T from __attribute__((ext_vector_type(V), aligned(sizeof(T))));
    typedef O to __attribute__((ext_vector_type(V), aligned(sizeof(O))));
    for (long long i = (long long)tid * V; i < n; i += 256 * V) {
        if (n - i >= V) {
            const from x = *(const from *)(g + i);
            to y;
#pragma unroll
            for (int e = 0; e < V; e++) y[e] = (O)((float)x[e] * f.first * f.by);
            *(to *)(out + i) = y;
        } else {
            for (int e = 0; e < n - i; e++) out[i + e] = (O)((float)g[i + e] * f.first * f.by);
        }
    }
}

template <class T> __device__ __forceinline__ void scaled_to(const ClipArgs &a, int t, long long from, long long n, Factor f) {
    const T *g = (const T *)a.grad[t] + from;
    if (a.out_type[t] == LOGOSKG_F32) scaled(g, (float *)a.out[t] + from, n, f, threadIdx.x);
    else if (a.out_type[t] == LOGOSKG_BF16) scaled(g, (bf16 *)a.out[t] + from, n, f, threadIdx.x);
    else scaled(g, (fp16 *)a.out[t] + from, n, f, threadIdx.x);
}

// (n: the number of sums that every block adds up itself, or 0: the factor is made)
__global__ __launch_bounds__(256) void k_clip_scale(ClipArgs a, int n, float max_norm, float scale, float *norm) {
    __shared__ double box[4];
    double got, factor = n ? factor_of(a.sums, n, max_norm, scale, box, got) : a.sums[0];
    if (n && blockIdx.x == 0 && a.first == 0 && threadIdx.x == 0) *norm = (float)got;
    const bool small = fabs(factor) < 0x1p-126 && factor != 0.0;
    const Factor f = {small ? 0x1p-100f : 1.f, (float)(small ? factor * 0x1p100 : factor)};
    for (long long c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int t = tensor_of(a, c);
        if (f.first * f.by == 1.f && a.grad[t] == a.out[t] && a.type[t] == a.out_type[t]) continue;  // (they are what they become)
        const long long from = (c - a.begin[t]) * kClipChunk, n = a.n[t] - from < kClipChunk ? a.n[t] - from : kClipChunk;
        if (a.type[t] == LOGOSKG_F32) scaled_to<float>(a, t, from, n, f);
        else if (a.type[t] == LOGOSKG_BF16) scaled_to<bf16>(a, t, from, n, f);
        else scaled_to<fp16>(a, t, from, n, f);
    }
}

static const char *bad_gradients(const logoskg_gradient *list, int64_t count) {
    if (count < 0 || count > (1 << 24) || (count && !list)) return "list is NULL, or a count is out of range";
    for (int64_t i = 0; i < count; i++) {
        const logoskg_gradient &g = list[i];
        if (g.dtype < LOGOSKG_F32 || g.dtype > LOGOSKG_F16 || g.out_dtype < LOGOSKG_F32 || g.out_dtype > LOGOSKG_F16) return "unknown type";
        if (g.n < 0 || g.n > (1ll << 42)) return "a count is out of range";
        if (g.n && (!g.grad || !g.out)) return "grad or out is NULL";
        if (g.n && (!aligned_to(g.grad, g.dtype) || !aligned_to(g.out, g.out_dtype))) return kUnaligned;
    }
    return nullptr;
}

// Whether an array that is written shares memory with another array (its own gradient may be it, element for element).
static bool shared(const logoskg_gradient *list, int64_t count) {
    struct Range { uintptr_t from, to; int64_t of; bool written; };
    std::vector<Range> all;
    all.reserve(2 * (size_t)count);
    for (int64_t i = 0; i < count; i++) {
        const logoskg_gradient &g = list[i];
        if (!g.n) continue;
        const bool same = g.grad == g.out && g.dtype == g.out_dtype;
        all.push_back({(uintptr_t)g.out, (uintptr_t)g.out + (uintptr_t)g.n * size_of(g.out_dtype), i, true});
        if (!same) all.push_back({(uintptr_t)g.grad, (uintptr_t)g.grad + (uintptr_t)g.n * size_of(g.dtype), i, false});
    }
    std::sort(all.begin(), all.end(), [](const Range &x, const Range &y) { return x.from < y.from; });
    uintptr_t end = 0, written_end = 0;  // of the ranges so far, and of those that are written
    for (const Range &r : all) {
        if (r.from < (r.written ? end : written_end)) return true;
        end = std::max(end, r.to);
        if (r.written) written_end = std::max(written_end, r.to);
    }
    return false;
}

// f(arguments, blocks) for every launch: up to kClipList tensors each; the number of sums.
template <class F> static long long each_launch(const logoskg_gradient *list, int64_t count, F f) {
    long long first = 0;
    for (int64_t i = 0; i < count;) {
        ClipArgs a;
        a.count = 0;
        long long chunks = 0;
        for (; i < count && a.count < kClipList; i++) {
            const logoskg_gradient &g = list[i];
            if (!g.n) continue;
            const long long more = (g.n + kClipChunk - 1) / kClipChunk;
            if (chunks + more >= (1ll << 31)) break;
            const int t = a.count++;
            a.grad[t] = g.grad; a.out[t] = g.out; a.n[t] = g.n;
            a.type[t] = (unsigned char)g.dtype; a.out_type[t] = (unsigned char)g.out_dtype;
            a.begin[t] = (int)chunks;
            chunks += more;
        }
        if (!a.count) continue;
        a.chunks = chunks;
        a.first = (int)first;
        const int blocks = (int)std::min<long long>(chunks, kClipBlocks);
        if (!f(a, blocks)) return -1;
        first += blocks;
    }
    return first;
}

}  // namespace lkg

using namespace lkg;

extern "C" int64_t logoskg_clip_gradients_bytes(const logoskg_gradient *list, int64_t count) {
    if (const char *why = bad_gradients(list, count)) { set_error("logoskg_clip_gradients_bytes: %s", why); return -1; }
    return (kClipTop + each_launch(list, count, [](const ClipArgs &, int) { return true; })) * 8;
}

extern "C" logoskg_status logoskg_clip_gradients(int32_t device, const logoskg_gradient *list, int64_t count, float max_norm, float scale,
                                                 float *norm, void *workspace, int64_t workspace_bytes, void *stream) {
    const char *why = bad_gradients(list, count);
    if (!why && !(max_norm >= 0.f)) why = "max_norm is negative";
    if (!why && !(scale - scale == 0.f)) why = "scale is not finite";
    if (!why && !norm) why = "norm is NULL";
    if (!why && ((uintptr_t)workspace & 15)) why = "the workspace is not 16-byte aligned";
    try {
        if (!why && shared(list, count)) why = "arrays that are written share memory";
    } catch (const std::bad_alloc &) {
        set_error("logoskg_clip_gradients: no host memory");
        return LOGOSKG_ENOMEM;
    }
    if (why) { set_error("logoskg_clip_gradients: %s", why); return LOGOSKG_EINVAL; }
    const int64_t need = logoskg_clip_gradients_bytes(list, count);
    if (workspace_bytes < need || !workspace) {
        set_error("logoskg_clip_gradients: the workspace has %lld of %lld bytes", (long long)workspace_bytes, (long long)need);
        return LOGOSKG_ERANGE;
    }
    OnDevice on;
    LKG_TRY(on.go(device));
    hipStream_t st = (hipStream_t)stream;
    double *sums = (double *)workspace;
    hipError_t went = hipSuccess;
    const long long n = each_launch(list, count, [&](ClipArgs &a, int blocks) {
        a.sums = sums;
        k_clip_squares<<<dim3(blocks), 256, 0, st>>>(a);
        return (went = hipGetLastError()) == hipSuccess;
    });
    LKG_HIP(went);
    const bool each = n > 0 && n <= kClipEach;
    if (!each) {
        k_clip_norm<<<1, 256, 0, st>>>(sums, (int)n, max_norm, scale, norm);
        LKG_HIP(hipGetLastError());
    }
    each_launch(list, count, [&](ClipArgs &a, int blocks) {
        a.sums = sums;
        k_clip_scale<<<dim3(blocks), 256, 0, st>>>(a, each ? (int)n : 0, max_norm, scale, norm);
        return (went = hipGetLastError()) == hipSuccess;
    });
    LKG_HIP(went);
    return LOGOSKG_OK;
}
