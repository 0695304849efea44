// Gradients of the attention of a ragged batch (logoskg_attend_backward).
//
// With p = 2^(y - lse), dP = dO V^T and delta = sum of p dP of a row (= dO . O), the gradient of the score y is
// dy = p (dP - delta), that of the product z: dz = dy scale (1 - tanh^2); dV = p^T dO, dK = dz^T Q, dQ = dz K, and a
// bucket's bias gets the sum of its dy.  Two kernels make p and dP again: first one that keeps rows and passes over their
// keys (dQ), then one that keeps keys and passes over the rows that see them (dK, dV, biases): seven products for five, and
// in return no sum depends on the order in which blocks arrive, and none is kept in memory in between.
//
// O comes in 16 bits, and dO . O carries its rounding: the first kernel, which begins with dO . O of its rows, adds up a row's
// dy, which is what delta lacks, and leaves delta with it to the second (a bucket's sum of many dy would show it most).  Its own dQ
// has it where rows see few keys (kFewSeen); a row whose biases hide all but a few keys of several tiles is not told from others.
// p and dz are rounded to the 16 bits that the matrix instructions take, sums are held in 32: dQ, dK and dV carry two
// roundings, this one of every term and their own, sqrt 2 of what rounding the exact gradient alone gives (bfloat16: 0.0025 for
// 0.0017 of the norm).  In float16 a dz below 2^-14 loses bits and one below 2^-25 all: losses are scaled, as that type asks.
//
// Both kernels work as the forward does: products of the next and of the last tile between the elements of this one, and
// tiles that ask for nothing special (all visible, one bias, scores in the range of the tanh's polynomial) are spared the
// rest.  A special tile's elements are made beforehand in a form that the common steps leave as they are.
#include "attend.h"

namespace lkg {

// What an element's steps take, from its products z and dP: w = z times the polynomial (or z near0), p = 2^(w + fma(lse, lse_share,
// b)), dy = p (dP - delta_share delta), dz = dy (curve w^2 + slope).  Special tiles come with w + shift in z and with
// (dP - delta) slope in dP.
struct Steps {
    float near0, near1, near2, near3, b, lse_share, delta_share, curve, slope;
};
template <bool CAP> __device__ __forceinline__ Steps plain_steps(const AttArgs &a, float b) {
    Steps x;
    x.near0 = CAP ? a.score.near[0] : a.score.k, x.near1 = a.score.near[1], x.near2 = a.score.near[2], x.near3 = a.score.near[3];
    x.b = b, x.lse_share = -1.f, x.delta_share = 1.f, x.curve = CAP ? a.curve : 0.f, x.slope = a.scale;
    return x;
}
__device__ __forceinline__ Steps special_steps() { return Steps{1.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 1.f}; }

template <bool CAP> __device__ __forceinline__ float element_w(const Steps &x, float z) {
    if (!CAP) return z;
    const float zz = z * z;
    float w = __builtin_fmaf(zz, x.near3, x.near2);
    w = __builtin_fmaf(zz, w, x.near1);
    w = __builtin_fmaf(zz, w, x.near0);
    return z * w;
}
template <bool CAP> __device__ __forceinline__ float element_dz(const Steps &x, float dy, float w) {
    return dy * (CAP ? __builtin_fmaf(w * w, x.curve, x.slope) : x.slope);
}

// An element on its way through the steps (first_of): w, p, dy, dz, a stage each step
constexpr int kStages = 6;
struct Element {
    float square, w, p, dz;
    template <bool CAP> __device__ __forceinline__ void step(int stage, const Steps &x, float z, float dp, float shift, float delta, float &sum) {
        if (stage == 0 && CAP) {
            square = z * z;
            w = __builtin_fmaf(square, x.near3, x.near2);
            here(w);
        }
        if (stage == 1 && CAP) {
            w = __builtin_fmaf(square, w, x.near1);
            w = __builtin_fmaf(square, w, x.near0);
            here(w);
        }
        if (stage == 2) {
            if (CAP) w *= z;
            p = CAP ? w + shift : __builtin_fmaf(z, x.near0, shift);
            here(p);
        }
        if (stage == 3) {
            p = exp2_fast(p);
            dz = __builtin_fmaf(delta, -x.delta_share, dp);
            here(p);
            here(dz);
        }
        if (stage == 4) {
            dz *= p;  // (dy)
            square = CAP ? w * w : 0.f;
            here(dz);
        }
        if (stage == 5) {
            sum += dz;
            dz *= CAP ? __builtin_fmaf(square, x.curve, x.slope) : x.slope;
            here(dz);
        }
    }
};
template <class E> __device__ __forceinline__ typename Vec8<E>::type chunk_of(const unsigned *pairs) {
    return as8<E>(u32x4{pairs[0], pairs[1], pairs[2], pairs[3]});
}

// A special element: y and its slope from the product; `far`: which may be of any size
template <bool CAP> __device__ __forceinline__ void score_of(const AttArgs &a, const Steps &x, bool far, float z, float &y, float &slope) {
    if (!CAP) {
        y = z * x.near0;
        slope = x.slope;
    } else if (far) {
        float share;
        y = any_capped(a.score, z, share);
        slope = a.slope * (share * (1.f - share));
    } else {
        y = element_w<CAP>(x, z);
        slope = __builtin_fmaf(y * y, x.curve, x.slope);
    }
}
// What is special about a tile: varied biases alone, whose elements need no look at what a row sees; hidden keys; products that
// are not near (in dK, dV kEdge takes these too, eight elements at a time, for want of registers).  Without biases one kind is for all.
enum { kVaried, kEdge, kFar };
constexpr float kHiddenLse = 1e15f;    // of a row that sees nothing, or is none: p = 0 the same way

// the first row that sees one of the keys from kb on
__device__ __forceinline__ int first_row(const AttArgs &a, const AttDoc &doc, long long kb) {
    if (!a.causal || kb < doc.prefix) return 0;
    const long long i = kb - ((long long)doc.keys - doc.rows);
    return i < 0 ? 0 : i > doc.rows ? doc.rows : (int)i;
}

// ---------------------------------------------------------------- order
// Blocks by their work, most first, for k_att_dkdv (key blocks) and k_att_dq (row blocks): where there are more of them than
// units, long ones that begin late leave the others idle.  One block each; a wavefront goes over a document's blocks, three
// times: the largest, how many of each of 512 classes, and each into its class's places (in whichever order: what a block
// computes does not depend on its turn).  Offsets that do not ascend may name a block twice or never, but none outside.
__global__ __launch_bounds__(1024) void k_att_order(AttArgs a) {
    constexpr int kBins = 512;
    __shared__ unsigned bins[kBins];
    __shared__ int largest;
    const bool of_rows = blockIdx.x != 0;
    const int64_t *off = of_rows ? a.q_off : a.k_off;
    const long long total = of_rows ? a.num_rows : a.num_keys, n = of_rows ? a.row_blocks : a.key_blocks;
    const int mult = of_rows ? a.group : 1, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int *order = of_rows ? a.row_order : a.key_order;
    const float by_group = 1.f / a.group;  // (a row or two off is no matter here)
    if (tid < kBins) bins[tid] = 0;
    if (tid == 0) largest = 1;
    for (long long i = tid; i < n; i += 1024) order[i] = (int)i;
    __syncthreads();
    auto each = [&](auto f) {
        for (int d = wave; d < a.num_docs; d += 16) {
            const AttDoc doc = att_doc(a, d);
            const long long base = first_block(off, d, total, mult, kAttRowsShift), end = d + 1 == a.num_docs ? n : first_block(off, d + 1, total, mult, kAttRowsShift);
            for (long long b = (d == 0 ? 0 : base) + lane; b < end && b < n; b += 64) {
                const long long x = (b - base) << kAttRowsShift, rows = (long long)doc.rows * a.group;
                int tiles = 0;
                if (of_rows && x >= 0 && x < rows) tiles = (doc.seen((int)((float)(x + kAttRows < rows ? x + kAttRows - 1 : rows - 1) * by_group), a.causal) >> 6) + 1;
                if (!of_rows && x >= 0 && x < doc.keys) tiles = ((doc.rows - first_row(a, doc, x)) >> 6) + 1;
                f(b, tiles);
            }
        }
        __syncthreads();
    };
    each([&](long long, int tiles) { atomicMax(&largest, tiles); });
    const float by_most = (kBins - 1) / (float)largest;
    auto bin_of = [&](int tiles) { return kBins - 1 - (int)((float)tiles * by_most); };
    each([&](long long, int tiles) { atomicAdd(&bins[bin_of(tiles)], 1u); });
    if (wave == 0) {  // how many lie before a class
        unsigned mine[kBins / 64], sum = 0;
#pragma unroll
        for (int i = 0; i < kBins / 64; i++) mine[i] = sum, sum += bins[lane * (kBins / 64) + i];
        unsigned before = sum;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const unsigned x = __shfl_up(before, s);
            if (lane >= s) before += x;
        }
#pragma unroll
        for (int i = 0; i < kBins / 64; i++) bins[lane * (kBins / 64) + i] = before - sum + mine[i];
    }
    __syncthreads();
    each([&](long long b, int tiles) {
        const unsigned at = atomicAdd(&bins[bin_of(tiles)], 1u);
        if (at < n) order[at] = (int)b;
    });
}

// ---------------------------------------------------------------- dQ
// One block: 128 rows as in the forward, keys in tiles of 64: K through a ring of four buffers (read by rows for the next
// tile's scores, by columns for the last tile's dQ), V through two.  Heads above 64 have registers for one wavefront a
// unit, whose matrix instructions follow from four chains; smaller ones for two.  4 documents of up to 4,096 rows and keys (32 / 8
// heads of 128, bfloat16, cap, bias): 690 us, 520 TFLOP/s of its three products.
constexpr int kGradTile = 64;
constexpr int kFewSeen = 16;  // with n keys what delta lacks is some 1 / sqrt n of the roundings of dz and dQ

template <class E, int DP, bool CAP, bool BIAS>
__global__ __launch_bounds__(kAttThreads, DP == 64 ? 2 : 1) void k_att_dq(AttArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    typedef typename Vec8<E>::type Chunk;
    constexpr int kTile = kGradTile * DP * 2, kSteps = DP / 16, kOut = DP / 32, kUnder = 32 * DP * 2;  // kUnder: to a tile's second 32 rows
    int *kpos = (int *)(lds + 6 * kTile);       // [4][kGradTile]  (LDS begins with four buffers of K, two of V)
    float *table = (float *)(kpos + 4 * kGradTile);
    const int M = a.score.max_distance, G = a.group;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int head = blockIdx.x % a.kv_heads;
    const unsigned turn = blockIdx.x / a.kv_heads;  // (the last rows of a document see most)
    const long long block = a.row_order ? a.row_order[turn] : a.row_blocks - 1 - turn;
    const int d = document_of(a.q_off, a.num_docs, a.num_rows, G, kAttRowsShift, block, lane);
    const AttDoc doc = att_doc(a, d);
    const long long first = (block - first_block(a.q_off, d, a.num_rows, G, kAttRowsShift)) << kAttRowsShift;
    const long long vrows = (long long)doc.rows * G;
    each_spare<kAttRows>(doc.row0 * a.group, vrows, a.num_rows * a.group, d, a.num_docs, block, first, tid, [&](long long at) {
        const long long spare = at / a.group * a.heads + head * a.group + at % a.group;
        clear_row((E *)a.dq + spare * a.dim, a.dim);
    });
    if (first >= vrows || first < 0) return;

    const long long vr = first + wave * 32 + (lane & 31);
    const bool mine = vr < vrows;
    const long long vr_in = mine ? vr : vrows - 1;
    const int row = (int)(vr_in / G), g = (int)(vr_in % G), h = head * G + g;
    const int seen = mine ? doc.seen(row, a.causal) : 0;
    const int least = doc.seen((int)(first / G), a.causal);
    const long long last_v = first + kAttRows < vrows ? first + kAttRows - 1 : vrows - 1;
    const int most = doc.seen((int)(last_v / G), a.causal);
    const long long place = (doc.row0 + row) * a.heads + h;
    const E *qrow = (const E *)a.q + (doc.row0 + row) * a.q_row + (long long)h * a.q_head;
    const E *orow = (const E *)a.dout + place * a.dim;
    Chunk q[kSteps], o[kSteps];
#pragma unroll
    for (int kk = 0; kk < kSteps; kk++) {
        q[kk] = row_chunk<E>(qrow, mine, kk, a.dim, lane);
        o[kk] = row_chunk<E>(orow, mine, kk, a.dim, lane);
    }
    float delta = 0.f;
#pragma unroll
    for (int kk = 0; kk < kSteps; kk++) {
        const Chunk x = row_chunk<E>((const E *)a.out + place * a.dim, mine, kk, a.dim, lane);
#pragma unroll
        for (int i = 0; i < 8; i++) delta = __builtin_fmaf((float)x[i], (float)o[kk][i], delta);
    }
    delta = halves_sum(delta);
    float lse = mine ? a.lse[place] : -INFINITY;
    lse = lse == -INFINITY ? kHiddenLse : lse * kLog2e;
    const float *my_table = table + g * (2 * M + 1);
    int q_low = 0, q_high = 0;
    Places places = {0, 0, 0};
    if (BIAS) {
        const int q_pos = a.q_pos ? a.q_pos[doc.row0 + row] : row + (doc.keys - doc.rows);
        places = places_of_keys(q_pos, M, lds_place(my_table));
        q_low = __builtin_amdgcn_readfirstlane(wave_min(q_pos));
        q_high = __builtin_amdgcn_readfirstlane(wave_max(q_pos));
        bias_to_lds<E>(table, a.score, head * G, G, tid, kAttThreads);
    }
    const char *kbase = (const char *)a.k + (doc.key0 * a.k_row + (long long)head * a.k_head) * 2;
    const char *vbase = (const char *)a.v + (doc.key0 * a.v_row + (long long)head * a.v_head) * 2;
    f32x16 dq[kOut], s[2] = {zero16(), zero16()}, dp[2] = {zero16(), zero16()};
#pragma unroll
    for (int i = 0; i < kOut; i++) dq[i] = zero16();
    Chunk z[4];
#pragma unroll
    for (int i = 0; i < 4; i++) z[i] = as8<E>(u32x4{0, 0, 0, 0});
    float size = 0.f, lacks = 0.f;

    TileLoad<kGradTile, DP> kload, vload;
    kload.begin(kbase, (unsigned)a.k_row * 2, 0, doc.keys, a.dim, tid);
    vload.begin(vbase, (unsigned)a.v_row * 2, 0, doc.keys, a.dim, tid);
    u32x4 kx[TileLoad<kGradTile, DP>::kChunks], vx[TileLoad<kGradTile, DP>::kChunks];
    const unsigned tiles = lds_place(lds), my_rows = rows_place<DP>(lane) + tiles, my_columns = columns_place<DP>(lane) + tiles;
    auto k_buffer = [](int t) { return (unsigned)(t & 3) * kTile; };
    auto v_buffer = [](int t) { return (unsigned)(4 + (t & 1)) * kTile; };
    int kp = 0;
    auto fetch = [&](int t) {
        kload.load(kx);
        vload.load(vx);
        if (BIAS && wave == 0) {
            int j = t * kGradTile + lane;
            j = j < doc.keys ? j : doc.keys - 1;
            kp = a.k_pos && doc.keys > 0 ? a.k_pos[doc.key0 + j] : j;
        }
    };
    auto stage = [&](int t) {
        kload.store(tiles + k_buffer(t), kx);
        vload.store(tiles + v_buffer(t), vx);
        if (BIAS && wave == 0) kpos[(t & 3) * kGradTile + lane] = kp;
    };
    bool varied = false;
    float b = 0.f;
    auto look_at = [&](int pos) {  // one bias for all distances of a tile?
        const int y = distance_place(pos, q_high, M), w = distance_place(pos, q_low, M), y0 = __builtin_amdgcn_readfirstlane(y);
        varied = wave_any(y != y0 || w != y0);
        b = my_table[y0];
    };
    const int tiles_n = (most + kGradTile - 1) / kGradTile;
    if (tiles_n > 0) {
        fetch(0);
        stage(0);
        fetch(1);
        stage(1);
        kload.clear(tiles + k_buffer(3));  // (round 0 multiplies it with zeros)
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2 * kSteps; i++) {
            s[i & 1] = mfma(rows_chunk<E>(my_rows + (i & 1) * kUnder, i >> 1), q[i >> 1], s[i & 1]);
            dp[i & 1] = mfma(rows_chunk<E>(my_rows + v_buffer(0) + (i & 1) * kUnder, i >> 1), o[i >> 1], dp[i & 1]);
        }
#pragma unroll
        for (int r = 0; r < 32; r++) size = fmaxf(size, __builtin_fabsf(s[r / 16][r % 16]));
        if (BIAS) look_at(kpos[lane]);
        if (tiles_n == 1 || least <= kFewSeen) {
            // The dy of few keys nearly cancel (one key's is 0), and what delta lacks would be most of them.  It is added up first
            // for the rows that see no keys behind this tile, in blocks that have some with few.
            float lack = 0.f;
            const Steps x = plain_steps<CAP>(a, 0.f);
            auto add_up = [&](auto far) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 8; j++) {
                    const int at = 8 * j + 4 * half;
                    const u32x4 p4 = BIAS ? *(const u32x4 *)(kpos + at) : u32x4{0, 0, 0, 0};
                    float bias[4];
#pragma unroll
                    for (int e = 0; e < 4; e++) bias[e] = BIAS ? float_at(place_of_key(places, (int)p4[e])) : 0.f;
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int u = j / 4, r = 4 * (j % 4) + e;
                        float y, slope;
                        score_of<CAP>(a, x, decltype(far)::value, s[u][r], y, slope);
                        y += bias[e] - lse;
                        if (at + e < seen) lack = __builtin_fmaf(exp2_fast(y), dp[u][r] - delta, lack);
                    }
                    if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            };
            if (CAP && wave_any(size > a.score.most)) add_up(std::true_type{});
            else add_up(std::false_type{});
            lack = halves_sum(lack);
            if (seen <= kGradTile) delta += lack;
        }
        __syncthreads();
    }
    for (int t = 0; t < tiles_n; t++) {
        const bool edge = (t + 1) * kGradTile > least, far = wave_any(size > a.score.most), plain = !edge && !far && !varied;
        Steps x = plain_steps<CAP>(a, b);
        auto special = [&](auto kind) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < 2; u++) {
                float bias[16];
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    const u32x4 p4 = BIAS ? *(const u32x4 *)(kpos + (t & 3) * kGradTile + 32 * u + 8 * j + 4 * half) : u32x4{0, 0, 0, 0};
#pragma unroll
                    for (int e = 0; e < 4; e++) bias[4 * j + e] = BIAS ? float_at(place_of_key(places, (int)p4[e])) : 0.f;
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int r = 0; r < 16; r++) {
                    float away = dp[u][r] - delta;
                    if (decltype(kind)::value == kVaried) {
                        const float w = element_w<CAP>(x, s[u][r]);
                        float y = bias[r] - lse;
                        y = CAP ? y + w : __builtin_fmaf(w, x.near0, y);
                        s[u][r] = y;
                        dp[u][r] = element_dz<CAP>(x, away, w);
                    } else {
                        float y, slope;
                        score_of<CAP>(a, x, decltype(kind)::value == kFar, s[u][r], y, slope);
                        y += bias[r] - lse;
                        if (t * kGradTile + 32 * u + 8 * (r / 4) + 4 * half + r % 4 >= seen) y = kHidden, away = 0.f;
                        s[u][r] = y < kHidden ? kHidden : y;
                        dp[u][r] = away * slope;
                    }
                    lacks = __builtin_fmaf(exp2_fast(s[u][r]), away, lacks);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        if (!plain) {
            if (CAP && (!BIAS || far)) special(std::integral_constant<int, kFar>{});
            else if (!BIAS || edge) special(std::integral_constant<int, kEdge>{});
            else special(std::integral_constant<int, kVaried>{});
            x = special_steps();
        }
        const unsigned kt = my_rows + k_buffer(t + 1), vt = my_rows + v_buffer(t + 1), ct = my_columns + k_buffer(t - 1);
        constexpr int kAll = 6 * kSteps, kAhead = 4, kRing = 5;
        Chunk piece[kRing];
        auto piece_of = [&](int at) {
            if (at < 2 * kSteps) return columns_chunk<E, DP>(ct, 16 * (at / kOut), at % kOut);
            const int i = at - 2 * kSteps;  // four chains, one after the other: scores and dP of either half
            return rows_chunk<E>((i & 1 ? vt : kt) + (i >> 1 & 1) * kUnder, i >> 2);
        };
#pragma unroll
        for (int i = 0; i < kAhead; i++) piece[i] = piece_of(i);
        f32x16 next_s[2] = {zero16(), zero16()}, next_dp[2] = {zero16(), zero16()};
        float sum = 0.f;
        Element el[32];
        unsigned dz_pair[16];
        const float shift = __builtin_fmaf(lse, x.lse_share, x.b);
        in_turn<kAll + kStages - 1>([&](auto step) __attribute__((always_inline)) {
            constexpr int at = decltype(step)::value;
            __builtin_amdgcn_sched_barrier(0);
            if (at + kAhead < kAll) piece[(at + kAhead) % kRing] = piece_of(at + kAhead);
            if (at < 2 * kSteps) dq[at % kOut] = mfma(piece[at % kRing], z[at / kOut & 3], dq[at % kOut]);
            else if (at < kAll) {
                constexpr int i = at - 2 * kSteps, u = i >> 1 & 1;
                if (i & 1) next_dp[u] = mfma(piece[at % kRing], o[i >> 2], next_dp[u]);
                else next_s[u] = mfma(piece[at % kRing], q[i >> 2], next_s[u]);
            }
#pragma unroll
            for (int stage = 0; stage < kStages; stage++)
#pragma unroll
                for (int e = first_of<kAll>(at - stage); e < first_of<kAll>(at - stage + 1); e++) {
                    el[e].step<CAP>(stage, x, s[e / 16][e % 16], dp[e / 16][e % 16], shift, delta, sum);
                    if (stage == kStages - 1 && (e & 1)) {
                        dz_pair[e / 2] = rounded2<E>(el[e - 1].dz, el[e].dz);
                        here(dz_pair[e / 2]);
                    }
                }
            here(sum);
            if (BIAS && at == kAll / 4) look_at(kpos[((t + 1) & 3) * kGradTile + lane]);
            if (at == 0) fetch(t + 2);
            if (at == kAll / 2) stage(t + 2);  // (its buffers: of K of t - 2, of V of t, read last in the round before)
        });
        __builtin_amdgcn_sched_barrier(0);
        if (plain) lacks += sum;
        size = 0.f;
#pragma unroll
        for (int u = 0; u < 2; u++) {
            s[u] = next_s[u];
            dp[u] = next_dp[u];
        }
#pragma unroll
        for (int i = 0; i < 4; i++) z[i] = chunk_of<E>(dz_pair + 4 * i);
#pragma unroll
        for (int r = 0; r < 32; r++) size = fmaxf(size, __builtin_fabsf(s[r / 16][r % 16]));
        __syncthreads();
    }
    if (tiles_n > 0) {
        const unsigned ct = my_columns + k_buffer(tiles_n - 1);
#pragma unroll
        for (int i = 0; i < 4 * kOut; i++) dq[i % kOut] = mfma(columns_chunk<E, DP>(ct, 16 * (i / kOut), i % kOut), z[i / kOut], dq[i % kOut]);
    }
    lacks = halves_sum(lacks);
    if (!mine) return;
    if (half == 0) a.delta[place] = delta + lacks;
    write_row<E, DP>(dq, 1.f, (E *)a.dq + place * a.dim, a.dim, half);
}

// ---------------------------------------------------------------- dK, dV, biases
// One block: 128 keys of (document, key head), 32 per wavefront, key = lane, K and V in registers as the B of S = Q K^T and
// dP = dO V^T.  The rows that see them pass in tiles of 64 of one head, one head of the group after the other, through three
// buffers in LDS, where they are read by rows for these two products and by columns for dV^T += dO^T p and dK^T += Q^T dz;
// a round's first half is the last tile's columns, whose buffer then takes the tile after the next.  A lane adds its dy to its
// own column of [buckets][64] in LDS ([buckets][32] and one half of the wavefront after the other where there is no room: no
// two lanes add to an address at a time, so the sums have an order), those of a tile of one bias all at once; a head's
// columns are added up when its rows are through.
//
// dK, dV, K, V and the products fill both halves of the registers: one wavefront a unit, and what it waits for is its own
// time.  The batch of k_att_dq: 1,145 us, 420 TFLOP/s of its four products; matrix units busy for 24 % of the time, vector units for
// half, LDS for half.  It takes as long as the longest document's first key blocks, which see all 4,096 rows of four heads.
template <class E, int DP, bool CAP, bool BIAS>
__global__ __launch_bounds__(kAttThreads, 1) void k_att_dkdv(AttArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    typedef typename Vec8<E>::type Chunk;
    constexpr int kTile = kGradTile * DP * 2, kSteps = DP / 16, kOut = DP / 32, kUnder = 32 * DP * 2;
    const int G = a.group, M = a.score.max_distance, places_n = 2 * M + 1, nb = a.score.num_buckets;
    float *lses = (float *)(lds + 6 * kTile), *deltas = lses + 4 * kGradTile;  // [4][kGradTile] of the rows  (LDS begins with three times Q, dO)
    int *qpos = (int *)(deltas + 4 * kGradTile);
    const int cols = a.bias_columns;
    float *sums = (float *)(qpos + 4 * kGradTile);            // [4 wavefronts][nb][cols]
    float *aside = sums + (BIAS ? 4 * nb * cols : 0);         // [4 wavefronts][64]
    float *total = aside + (BIAS ? 256 : 0);                  // [2][4 wavefronts][nb]
    int *column = (int *)(total + (BIAS ? 8 * nb : 0));                // [places_n] where a distance's bucket begins, in bytes
    float *table = (float *)(column + (BIAS ? places_n : 0));  // [group][places_n]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int head = blockIdx.x % a.kv_heads;
    const unsigned turn = blockIdx.x / a.kv_heads;  // the first keys of a document are seen by most rows: first
    const long long block = a.key_order ? a.key_order[turn] : turn;
    const int d = document_of(a.k_off, a.num_docs, a.num_keys, 1, kAttRowsShift, block, lane);
    const AttDoc doc = att_doc(a, d);
    const long long kb = (block - first_block(a.k_off, d, a.num_keys, 1, kAttRowsShift)) << kAttRowsShift;
    float *part = BIAS ? a.bias_part + (block * a.heads + head * G) * nb : nullptr;
    each_spare<kAttRows>(doc.key0, doc.keys, a.num_keys, d, a.num_docs, block, kb, tid, [&](long long at) {
        clear_row((E *)a.dk + (at * a.kv_heads + head) * a.dim, a.dim);
        clear_row((E *)a.dv + (at * a.kv_heads + head) * a.dim, a.dim);
    });
    if (kb >= doc.keys || kb < 0) {
        if (BIAS)
            for (int i = tid; i < G * nb; i += kAttThreads) part[i] = 0.f;
        return;
    }

    const int key = (int)kb + wave * 32 + (lane & 31);
    const bool mine = key < doc.keys;
    const E *krow = (const E *)a.k + (doc.key0 + key) * a.k_row + (long long)head * a.k_head;
    const E *vrow = (const E *)a.v + (doc.key0 + key) * a.v_row + (long long)head * a.v_head;
    Chunk k[kSteps], v[kSteps];
#pragma unroll
    for (int kk = 0; kk < kSteps; kk++) {
        k[kk] = row_chunk<E>(krow, mine, kk, a.dim, lane);
        v[kk] = row_chunk<E>(vrow, mine, kk, a.dim, lane);
    }
    int k_low = 0, k_high = 0;
    Places places = {0, 0, 0};  // in `column`; a head's biases lie the same way
    const unsigned to_table = (unsigned)((char *)table - (char *)column), my_sums = lds_place(sums) + (wave * nb * cols + (lane & (cols - 1))) * 4;
    if (BIAS) {
        const int in = mine ? key : doc.keys - 1, k_pos = a.k_pos ? a.k_pos[doc.key0 + in] : in;
        places = places_of_rows(k_pos, M, lds_place(column));
        k_low = __builtin_amdgcn_readfirstlane(wave_min(k_pos));
        k_high = __builtin_amdgcn_readfirstlane(wave_max(k_pos));
        bias_to_lds<E>(table, a.score, head * G, G, tid, kAttThreads);
        for (int i = tid; i < places_n; i += kAttThreads) {
            int b = a.score.buckets[i];
            column[i] = (b < 0 ? 0 : b >= nb ? nb - 1 : b) * cols * 4;
        }
        for (int i = tid; i < nb * cols; i += kAttThreads) ((f32x4 *)sums)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // (Read, added and written: nobody else has the address meanwhile.  An atomic addition of 64 floats keeps LDS busy for 192 clocks.)
    auto add_at = [&](unsigned place, float x) {
        typedef __attribute__((address_space(3))) float lds_float;
        lds_float *at = (lds_float *)(uintptr_t)place;
        *at = *at + x;
    };
    // keys that are none (and where halves go one after the other, the other half) add to a place of their own that nobody reads
    const unsigned my_aside = lds_place(aside) + tid * 4;
    auto add_each = [&](int bucket, float x) {
        if (cols == 64) add_at(mine ? my_sums + bucket : my_aside, x);
        else {
            add_at(mine && half == 0 ? my_sums + bucket : my_aside, x);
            add_at(mine && half == 1 ? my_sums + bucket : my_aside, x);
        }
    };

    f32x16 dk[kOut], dv[kOut], s[2] = {zero16(), zero16()}, dp[2] = {zero16(), zero16()};
#pragma unroll
    for (int i = 0; i < kOut; i++) dk[i] = zero16(), dv[i] = zero16();
    Chunk p[4], z[4];
#pragma unroll
    for (int i = 0; i < 4; i++) p[i] = z[i] = as8<E>(u32x4{0, 0, 0, 0});
    float size = 0.f;

    const int kend = doc.keys < kb + kAttRows ? doc.keys : (int)kb + kAttRows;
    const int from = first_row(a, doc, kb);
    const int per = (doc.rows - from + kGradTile - 1) / kGradTile, tiles_n = per * G;  // tiles of a head, of all

    TileLoad<kGradTile, DP> qload, oload;
    qload.begin((const char *)a.q, (unsigned)a.q_row * 2, 0, 0, a.dim, tid);
    oload.begin((const char *)a.dout, (unsigned)a.heads * a.dim * 2, 0, 0, a.dim, tid);
    u32x4 qx[TileLoad<kGradTile, DP>::kChunks], ox[TileLoad<kGradTile, DP>::kChunks];
    const unsigned tiles = lds_place(lds), my_rows = rows_place<DP>(lane) + tiles, my_columns = columns_place<DP>(lane) + tiles;
    float my_lse = 0.f, my_delta = 0.f;
    int my_pos = 0, fetch_g = 0, fetch_at = 0;
    auto fetch = [&]() {  // the next tile (behind the last head's: rows that there are none of)
        const int h = head * G + (fetch_g < G ? fetch_g : G - 1), r0 = fetch_g < G ? from + fetch_at * kGradTile : doc.rows;
        if (fetch_at == 0) {
            qload.go_to((const char *)a.q + (doc.row0 * a.q_row + (long long)h * a.q_head) * 2, r0, doc.rows, a.dim);
            oload.go_to((const char *)a.dout + (doc.row0 * a.heads + h) * a.dim * 2, r0, doc.rows, a.dim);
        }
        qload.load(qx);
        oload.load(ox);
        if (wave == 0) {
            const int row = r0 + lane;
            const bool in = row < doc.rows;
            const long long at = in ? (doc.row0 + row) * a.heads + h : 0;
            const float lse = in ? a.lse[at] : -INFINITY;
            my_lse = lse == -INFINITY ? kHiddenLse : lse * kLog2e;
            my_delta = in ? a.delta[at] : 0.f;
            if (BIAS) {
                const int near = in ? row : doc.rows - 1;
                my_pos = a.q_pos ? a.q_pos[doc.row0 + near] : near + (doc.keys - doc.rows);
            }
        }
        if (++fetch_at == per) fetch_at = 0, fetch_g++;
    };
    auto stage = [&](int t, unsigned buffer) {
        qload.store(tiles + buffer, qx);
        oload.store(tiles + buffer + kTile, ox);
        if (wave == 0) {
            const int at = (t & 3) * kGradTile + lane;
            lses[at] = my_lse;
            deltas[at] = my_delta;
            if (BIAS) qpos[at] = my_pos;
        }
    };
    // The columns of a head that is through: a wavefront adds up its own, half of a bucket's columns a lane (16 bytes at a time,
    // from another place for each bucket, so that lanes read different banks), and clears them; the four sums are joined behind
    // one barrier, in two places by turns, so that none has to wait for the readers.
    auto finish = [&](int g) {
        float *mine4 = total + (g & 1) * 4 * nb;
        wave_sync();
        for (int b0 = 0; b0 < nb; b0 += 32) {
            const int b = b0 + (lane & 31), quads = cols >> 3;
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
            if (b < nb) {
                f32x4 *at = (f32x4 *)(sums + (wave * nb + b) * cols) + half * quads;
#pragma unroll 4
                for (int i = 0; i < quads; i++) {
                    const int c = (i + b) & (quads - 1);
                    const f32x4 x = at[c];
                    at[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < 4; e++) sum[e] += x[e];
                }
            }
            const float all = halves_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
            if (b < nb && half == 0) mine4[wave * nb + b] = all;
        }
        __syncthreads();
        if (tid < nb) part[g * nb + tid] = (mine4[tid] + mine4[nb + tid]) + (mine4[2 * nb + tid] + mine4[3 * nb + tid]);
    };
    bool varied = false;
    float b = 0.f;
    int bucket = 0;
    auto look_at = [&](int pos, int g) {  // one bias for all distances of a tile? (rows of a head, a lane each)
        const int y = distance_place(k_low, pos, M), w = distance_place(k_high, pos, M), y0 = __builtin_amdgcn_readfirstlane(y);
        varied = wave_any(y != y0 || w != y0);
        b = table[g * places_n + y0];
        bucket = column[y0];
    };
    unsigned last = 4 * kTile, now = 0, after = 2 * kTile;  // buffers of the tiles t - 1, t, t + 1
    if (tiles_n > 0) {
        fetch();
        stage(0, now);
        fetch();
        stage(1, after);
        qload.clear(tiles + last);  // (round 0 multiplies them with zeros)
        oload.clear(tiles + last + kTile);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2 * kSteps; i++) {
            s[i & 1] = mfma(rows_chunk<E>(my_rows + (i & 1) * kUnder, i >> 1), k[i >> 1], s[i & 1]);
            dp[i & 1] = mfma(rows_chunk<E>(my_rows + kTile + (i & 1) * kUnder, i >> 1), v[i >> 1], dp[i & 1]);
        }
#pragma unroll
        for (int r = 0; r < 32; r++) size = fmaxf(size, __builtin_fabsf(s[r / 16][r % 16]));
        if (BIAS) look_at(qpos[lane], 0);
        __syncthreads();
    }
    int g = 0, at_tile = 0;  // of the tile in work
    for (int t = 0; t < tiles_n; t++) {
        const int r0 = from + at_tile * kGradTile;
        const bool edge = doc.seen(r0, a.causal) < kend, far = wave_any(size > a.score.most), plain = !edge && !far && !varied;
        const float *lse = lses + (t & 3) * kGradTile, *delta = deltas + (t & 3) * kGradTile;
        const int bucket_now = bucket;
        Steps x = plain_steps<CAP>(a, b);
        auto special = [&](auto kind) __attribute__((always_inline)) {
            const unsigned to_head = to_table + g * places_n * 4;
#pragma unroll
            for (int part = 0; part < 4; part++) {
                // eight rows' look-ups, then their elements, then their additions: one wait each
                const int u = part >> 1, j0 = 2 * (part & 1);
                unsigned place[8];
                float bias[8], dy[8];
                int bucket_of[8];
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    if (!BIAS) break;
                    const u32x4 p4 = *(const u32x4 *)(qpos + (t & 3) * kGradTile + 32 * u + 8 * (j0 + j) + 4 * half);
#pragma unroll
                    for (int e = 0; e < 4; e++) place[4 * j + e] = place_of_row(places, (int)p4[e]);
                }
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    bias[i] = BIAS ? float_at(place[i] + to_head) : 0.f;
                    if (BIAS) bucket_of[i] = int_at(place[i]);
                }
                __builtin_amdgcn_sched_barrier(0);
                float ys[8], slopes[8];
                if (decltype(kind)::value != kVaried) {
                    if (CAP && (!BIAS || far)) {
#pragma unroll
                        for (int i = 0; i < 8; i++) score_of<CAP>(a, x, true, s[u][4 * j0 + i], ys[i], slopes[i]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; i++) score_of<CAP>(a, x, false, s[u][4 * j0 + i], ys[i], slopes[i]);
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; j++) {
                    const int at = 32 * u + 8 * (j0 + j) + 4 * half;
                    const f32x4 lse4 = *(const f32x4 *)(lse + at), delta4 = *(const f32x4 *)(delta + at);
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const int r = 4 * (j0 + j) + e;
                        float away = dp[u][r] - delta4[e];
                        if (decltype(kind)::value == kVaried) {
                            const float w = element_w<CAP>(x, s[u][r]);
                            float y = bias[4 * j + e] - lse4[e];
                            y = CAP ? y + w : __builtin_fmaf(w, x.near0, y);
                            s[u][r] = y;
                            dp[u][r] = element_dz<CAP>(x, away, w);
                        } else {
                            float y, slope;
                            y = ys[4 * j + e], slope = slopes[4 * j + e];
                            y += bias[4 * j + e] - lse4[e];
                            if (key >= doc.seen(r0 + at + e, a.causal)) y = kHidden, away = 0.f;
                            s[u][r] = y < kHidden ? kHidden : y;
                            dp[u][r] = away * slope;
                        }
                        dy[4 * j + e] = exp2_fast(s[u][r]) * away;
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if (BIAS) add_each(bucket_of[i], dy[i]);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        if (!plain) {
            if (!BIAS || edge || far) special(std::integral_constant<int, kEdge>{});
            else special(std::integral_constant<int, kVaried>{});
            x = special_steps();
        }
        const unsigned rt = my_rows + after, ct = my_columns + last;
        constexpr int kAll = 8 * kSteps, kAhead = 4, kRing = 5;
        Chunk piece[kRing];
        auto piece_of = [&](int at) {
            if (at < 4 * kSteps) return columns_chunk<E, DP>(ct + (at & 1 ? 0 : kTile), 16 * (at / 2 / kOut), at / 2 % kOut);  // dO and Q in turn
            const int i = at - 4 * kSteps;
            return rows_chunk<E>(rt + (i & 1 ? kTile : 0) + (i >> 1 & 1) * kUnder, i >> 2);
        };
        f32x16 next_s[2] = {zero16(), zero16()}, next_dp[2] = {zero16(), zero16()};
        float sum = 0.f;
        f32x4 l4[2], d4[2];  // of four rows, and the four before them
        Element el[32];
        unsigned p_pair[16], dz_pair[16];
        in_turn<kAll + kStages - 1>([&](auto step) __attribute__((always_inline)) {
            constexpr int at = decltype(step)::value;
            __builtin_amdgcn_sched_barrier(0);
            if (at % (kAll / 2) == 0 && at < kAll) {
                if (at == 0) fetch();  // (tile t + 2)
                else {
                    __syncthreads();  // the last tile's columns are read
                    stage(t + 2, last);
                }
#pragma unroll
                for (int i = 0; i < kAhead; i++) piece[(at + i) % kRing] = piece_of(at + i);
            }
            if (at + kAhead < kAll && (at + kAhead) % (kAll / 2) >= kAhead) piece[(at + kAhead) % kRing] = piece_of(at + kAhead);
            if (at % (kAll / 8) == 0 && at < kAll) {
                l4[at / (kAll / 8) & 1] = *(const f32x4 *)(lse + 8 * (8 * at / kAll) + 4 * half);
                d4[at / (kAll / 8) & 1] = *(const f32x4 *)(delta + 8 * (8 * at / kAll) + 4 * half);
            }
            if (at < 4 * kSteps) {
                constexpr int i = at / 2;
                if (at & 1) dk[i % kOut] = mfma(piece[at % kRing], z[i / kOut & 3], dk[i % kOut]);
                else dv[i % kOut] = mfma(piece[at % kRing], p[i / kOut & 3], dv[i % kOut]);
            } else if (at < kAll) {
                constexpr int i = at - 4 * kSteps, u = i >> 1 & 1;
                if (i & 1) next_dp[u] = mfma(piece[at % kRing], v[i >> 2], next_dp[u]);
                else next_s[u] = mfma(piece[at % kRing], k[i >> 2], next_s[u]);
            }
#pragma unroll
            for (int stage = 0; stage < kStages; stage++)
#pragma unroll
                for (int e = first_of<kAll>(at - stage); e < first_of<kAll>(at - stage + 1); e++) {
                    const float shift = stage == 2 ? __builtin_fmaf(l4[e / 4 & 1][e % 4], x.lse_share, x.b) : 0.f;
                    el[e].step<CAP>(stage, x, s[e / 16][e % 16], dp[e / 16][e % 16], shift, d4[e / 4 & 1][e % 4], sum);
                    if (stage == kStages - 1 && (e & 1)) {
                        p_pair[e / 2] = rounded2<E>(el[e - 1].p, el[e].p);
                        dz_pair[e / 2] = rounded2<E>(el[e - 1].dz, el[e].dz);
                        here(p_pair[e / 2]);
                        here(dz_pair[e / 2]);
                    }
                }
            if (BIAS) here(sum);
            if (BIAS && at == kAll / 4) look_at(qpos[((t + 1) & 3) * kGradTile + lane], at_tile + 1 < per ? g : g + 1 < G ? g + 1 : g);
        });
        __builtin_amdgcn_sched_barrier(0);
        if (BIAS && plain) add_each(bucket_now, sum);
#pragma unroll
        for (int i = 0; i < 4; i++) p[i] = chunk_of<E>(p_pair + 4 * i), z[i] = chunk_of<E>(dz_pair + 4 * i);
        size = 0.f;
#pragma unroll
        for (int u = 0; u < 2; u++) {
            s[u] = next_s[u];
            dp[u] = next_dp[u];
        }
#pragma unroll
        for (int r = 0; r < 32; r++) size = fmaxf(size, __builtin_fabsf(s[r / 16][r % 16]));
        const unsigned free_now = last;
        last = now;
        now = after;
        after = free_now;
        __syncthreads();
        if (++at_tile == per) {
            if (BIAS) finish(g);
            at_tile = 0, g++;
        }
    }
    if (tiles_n > 0) {
        const unsigned ct = my_columns + last;
#pragma unroll
        for (int i = 0; i < 4 * kOut; i++) {
            dv[i % kOut] = mfma(columns_chunk<E, DP>(ct + kTile, 16 * (i / kOut), i % kOut), p[i / kOut], dv[i % kOut]);
            dk[i % kOut] = mfma(columns_chunk<E, DP>(ct, 16 * (i / kOut), i % kOut), z[i / kOut], dk[i % kOut]);
        }
    } else if (BIAS) {
        for (int i = tid; i < G * nb; i += kAttThreads) part[i] = 0.f;
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

// dbias[head][bucket] = the blocks' parts, one after the other in 1024 / num_buckets strands
template <class E> __global__ __launch_bounds__(1024) void k_att_dbias(AttArgs a) {
    __shared__ float strand[1024];
    const int nb = a.score.num_buckets, h = blockIdx.x, strands = 1024 / nb, b = threadIdx.x % nb, s = threadIdx.x / nb;
    float sum = 0.f;
    if (s < strands)
        for (long long i = s; i < a.key_blocks; i += strands) sum += a.bias_part[(i * a.heads + h) * nb + b];
    strand[threadIdx.x] = sum;
    __syncthreads();
    if (s != 0) return;
    for (int i = 1; i < strands; i++) sum += strand[i * nb + b];
    ((E *)a.dbias)[h * nb + b] = (E)sum;
}

// Ordered where the blocks of either kernel are more than the units, the documents more than a few, whose blocks come most
// first by themselves and share caches, and most of them longer than a block: the order is made by one block per side, document by
// document, and blocks that are all alike have none.  Forward and backward, us without / with:
//   documents of uneven lengths (16 / 4 heads of 128, up to 700 tokens and 1,500 entities): 4 (176 blocks) 390 / 391, 8 (456)
//   618 / 567, 16 (840) 861 / 733, 64 (3,276) 2,837 / 2,681; text and entities attending to each other, 2,000: 4 (564) 739 / 743,
//   8 (1,104) 866 / 882, 16 (2,236) 1,373 / 1,210; up to 400: 16 (188 blocks) 147 / 147, 32 (348) 207 / 179
//   1,024 documents by the blocks of both kernels to a document: 2.2 987 / 1,084, 3.0 1,349 / 1,304, 3.4 1,746 / 1,722, 5.3
//   3,803 / 3,567; of 8 / 8 heads of 64: 2.2 780 / 934, 3.0 1,410 / 1,464, 3.7 1,906 / 1,922, 4.0 2,310 / 2,273, 5.7 4,344 / 4,252
static bool ordered(const AttArgs &a) {
    return a.num_docs >= 8 && a.num_rows && a.num_keys && 3 * (a.row_blocks + a.key_blocks) >= 10ll * a.num_docs &&
           (a.row_blocks > a.key_blocks ? a.row_blocks : a.key_blocks) * a.kv_heads > 256;
}
static int64_t delta_bytes(const AttArgs &a) { return (a.num_rows * a.heads * 4 + 15) / 16 * 16; }
static int64_t backward_bytes(const AttArgs &a) {
    return delta_bytes(a) + (a.score.bias ? a.key_blocks * a.heads * (int64_t)a.score.num_buckets * 4 : 0) + (ordered(a) ? (a.row_blocks + a.key_blocks) * 4 : 0);
}

template <class E, int DP, bool CAP, bool BIAS> static logoskg_status launch_backward(const AttArgs &a, hipStream_t st) {
    const size_t places = BIAS ? 2 * a.score.max_distance + 1 : 0, table = a.group * places * 4;
    if (a.num_rows) {
        size_t bytes = 6 * kGradTile * DP * 2 + 4 * kGradTile * 4 + table;
        LKG_TRY(allow_lds(k_att_dq<E, DP, CAP, BIAS>, bytes));
        k_att_dq<E, DP, CAP, BIAS><<<dim3((unsigned)(a.row_blocks * a.kv_heads)), kAttThreads, bytes, st>>>(a);
        LKG_HIP(hipGetLastError());
    }
    if (a.num_keys) {
        AttArgs b = a;
        size_t bytes = 6 * kGradTile * DP * 2 + 3 * 4 * kGradTile * 4 + table + places * 4 + (BIAS ? 1024 + 32 * (size_t)a.score.num_buckets : 0);
        static_assert(6 * kGradTile * 128 * 2 + 3 * 4 * kGradTile * 4 + (LOGOSKG_BIAS_PLACES + 2 * LOGOSKG_MAX_DISTANCE + 1) * 4 + 1024 +
                      LOGOSKG_MAX_BUCKETS * (32 + 4 * 32 * 4) <= kLds, "the largest biases fit, with 32 columns a bucket");
        b.bias_columns = bytes + (size_t)4 * a.score.num_buckets * 64 * 4 <= kLds ? 64 : 32;
        if (BIAS) bytes += (size_t)4 * a.score.num_buckets * b.bias_columns * 4;
        LKG_TRY(allow_lds(k_att_dkdv<E, DP, CAP, BIAS>, bytes));
        k_att_dkdv<E, DP, CAP, BIAS><<<dim3((unsigned)(a.key_blocks * a.kv_heads)), kAttThreads, bytes, st>>>(b);
        LKG_HIP(hipGetLastError());
    }
    return LOGOSKG_OK;
}

template <class E> static logoskg_status backward(const AttArgs &a, hipStream_t st) {
    if (a.key_order) {
        k_att_order<<<dim3(2), 1024, 0, st>>>(a);
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
    if (a.key_blocks * a.kv_heads >= (1ll << 31)) { set_error("logoskg_attend_backward: too many rows"); return LOGOSKG_EINVAL; }
    if (a.num_keys == 0) a.key_blocks = 0;
    if (ordered(a)) a.key_order = (int *)(a.bias_part + (a.score.bias ? a.key_blocks * a.heads * (int64_t)a.score.num_buckets : 0)), a.row_order = a.key_order + a.key_blocks;
    LKG_HIP(hipSetDevice(in->device));
    return in->dtype == LOGOSKG_BF16 ? backward<bf16>(a, (hipStream_t)in->stream) : backward<fp16>(a, (hipStream_t)in->stream);
}
