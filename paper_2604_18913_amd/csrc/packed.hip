// Keys and values by entity in 4 bits: into that form and back, and few tokens of every query attending to a list of such rows
// (logoskg_pack_entities, logoskg_unpack_entities, logoskg_read_packed).
#include "read.h"
#include "training.h"

#include <algorithm>

namespace lkg {

static_assert(sizeof(logoskg_pack) == 104, "the ctypes binding mirrors this layout");

typedef unsigned long long u64;

// ---------------------------------------------------------------- rows
struct PackArgs {
    int kv_heads, dim, groups, pad;  // groups: of a head; pad: bytes behind the last group
    long long num_rows;
    void *keys, *values;
    long long key_row, key_head, value_row, value_head;
    char *packed;
    long long packed_row;
};

__host__ __device__ __forceinline__ int row_bytes_of(int kv_heads, int groups) { return (40 * kv_heads * groups + 15) / 16 * 16; }

template <class T> struct Eight { typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T)))); };

// of this lane and the one beside it, and of those two and the other two of four
template <int PERM> __device__ __forceinline__ float quad(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), PERM, 0xf, 0xf, true)); }
__device__ __forceinline__ float quad_min(float x) { x = fminf(x, quad<0xb1>(x)); return fminf(x, quad<0x4e>(x)); }
__device__ __forceinline__ float quad_max(float x) { x = fmaxf(x, quad<0xb1>(x)); return fmaxf(x, quad<0x4e>(x)); }
__device__ __forceinline__ float quad_sum(float x) { x += quad<0xb1>(x); return x + quad<0x4e>(x); }

// Four lanes' codes of a group of 32 elements, eight each (x: those of this lane, `in`: whether there are any), and its scale and base.
struct Codes { unsigned word, scale_base; };
__device__ __forceinline__ Codes codes_of(const float (&x)[8], bool in) {
    float lo = INFINITY, hi = -INFINITY, odd = 0.f;
    if (in) {
#pragma unroll
        for (int e = 0; e < 8; e++) lo = fminf(lo, x[e]), hi = fmaxf(hi, x[e]), odd = __builtin_fmaf(x[e], 0.f, odd);
    }
    lo = quad_min(lo), hi = quad_max(hi), odd = quad_sum(odd);
    // both rounded to the nearest bfloat16, off by up to 2^-8 of themselves: of the scale, over 15 steps, that is a ninth of half a step; of the
    // base it is as much of the group's offset, which is more than a step where that is 17 times the range
    const bf16 scale = (bf16)((hi - lo) / 15.f), base = (bf16)lo;
    const float s = (float)scale, b = (float)base;
    Codes got = {0, (unsigned)__builtin_bit_cast(unsigned short, scale) | (unsigned)__builtin_bit_cast(unsigned short, base) << 16};
    if (!(odd + (s - s) + (b - b) == 0.f)) {
        got.scale_base = 0x7fc07fc0u;  // NaN
        return got;
    }
    // (x - b) / s to the nearest whole number, halves to even ones, without a division: by a reciprocal, whose error matters next to
    // halves alone, where the rest x - b - c s (c s has 12 bits, so that the rest is exact there) says on which side it is.  Scales that
    // have no normal reciprocal are divided by.
    float c[8], rest = 0.f;
    if (s > 1e-37f && s < 1e37f) {
        const float inv = 1.f / s, half = 0.5f * s;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            const float d = x[e] - b;
            c[e] = __builtin_rintf(d * inv);
            rest = fmaxf(rest, __builtin_fabsf(__builtin_fmaf(-c[e], s, d)));
        }
        if (wave_any(rest >= half)) {
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float d = x[e] - b, r = __builtin_fmaf(-c[e], s, d), size = __builtin_fabsf(r);
                if (size > half || (size == half && ((int)c[e] & 1))) c[e] += r > 0.f ? 1.f : -1.f;
            }
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) c[e] = s > 0.f ? __builtin_rintf((x[e] - b) / s) : 0.f;
    }
    if (in) {  // four codes a time as a whole number of 16 bits, which 32-bit floats hold
        float two[2] = {0.f, 0.f};
#pragma unroll
        for (int e = 7; e >= 0; e--) two[e >> 2] = __builtin_fmaf(two[e >> 2], 16.f, __builtin_amdgcn_fmed3f(c[e], 0.f, 15.f));
        got.word = (unsigned)two[0] | (unsigned)two[1] << 16;
    }
    return got;
}

// What a thread of k_pack and k_unpack does: four lanes per group of 32 elements, blocks of whole rows (or of a part of a long one's
// groups at a time).  f(row, head, group, lane of the four)
template <class F> __device__ __forceinline__ void each_group(const PackArgs &a, F f) {
    const int items = a.kv_heads * a.groups, q = threadIdx.x >> 2, c = threadIdx.x & 3;
    const int rows = items < 64 ? 64 / items : 1, sub = items < 64 ? q / items : 0;
    if (sub >= rows) return;
    for (int item = items < 64 ? q % items : q; item < items; item += 64) {
        const int h = item / a.groups, g = item % a.groups;
        for (long long r = (long long)blockIdx.x * rows + sub; r < a.num_rows; r += (long long)gridDim.x * rows) f(r, h, g, c);
    }
}

// A row's keys, then its values, of a group.  Memory bounds it: 407,000 rows of 8 heads of 128 in bfloat16 (2.2 GB) 518 us, 4.2 TB/s.
template <class T> __global__ __launch_bounds__(256) void k_pack(PackArgs a) {
    each_group(a, [&](long long r, int h, int g, int c) __attribute__((always_inline)) {
        const int at = 32 * g + 8 * c;
        const bool in = at < a.dim;
        typename Eight<T>::type k = {}, v = {};
        if (in) {
            k = *(const typename Eight<T>::type *)((const T *)a.keys + r * a.key_row + h * a.key_head + at);
            v = *(const typename Eight<T>::type *)((const T *)a.values + r * a.value_row + h * a.value_head + at);
        }
        float x[8], y[8];
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = (float)k[e], y[e] = (float)v[e];
        const Codes kc = codes_of(x, in), vc = codes_of(y, in);
        char *row = a.packed + r * a.packed_row;
        const int all = a.kv_heads * a.groups;
        ((unsigned *)row)[h * 4 * a.groups + c * a.groups + g] = kc.word;
        ((unsigned *)row)[4 * all + (h * a.groups + g) * 4 + c] = vc.word;
        if (c < 2) ((unsigned *)row)[8 * all + (h * a.groups + g) * 2 + c] = c == 0 ? kc.scale_base : vc.scale_base;
        if (a.pad && c < 2 && h == a.kv_heads - 1 && g == a.groups - 1) ((unsigned *)row)[10 * all + c] = 0;
    });
}

__device__ __forceinline__ float low_half(unsigned x) { return __builtin_bit_cast(float, x << 16); }         // a bfloat16 in 32 bits
__device__ __forceinline__ float high_half(unsigned x) { return __builtin_bit_cast(float, x & 0xffff0000u); }

// (the same rows 393 us, 5.6 TB/s)
template <class T> __global__ __launch_bounds__(256) void k_unpack(PackArgs a) {
    each_group(a, [&](long long r, int h, int g, int c) __attribute__((always_inline)) {
        const int at = 32 * g + 8 * c, all = a.kv_heads * a.groups;
        if (at >= a.dim) return;
        const unsigned *row = (const unsigned *)(a.packed + r * a.packed_row);
        const unsigned kw = row[h * 4 * a.groups + c * a.groups + g], vw = row[4 * all + (h * a.groups + g) * 4 + c];
        const unsigned kp = row[8 * all + (h * a.groups + g) * 2], vp = row[8 * all + (h * a.groups + g) * 2 + 1];
        typename Eight<T>::type k, v;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            k[e] = (T)__builtin_fmaf(low_half(kp), (float)(kw >> (4 * e) & 15), high_half(kp));
            v[e] = (T)__builtin_fmaf(low_half(vp), (float)(vw >> (4 * e) & 15), high_half(vp));
        }
        *(typename Eight<T>::type *)((T *)a.keys + r * a.key_row + h * a.key_head + at) = k;
        *(typename Eight<T>::type *)((T *)a.values + r * a.value_row + h * a.value_head + at) = v;
    });
}

// ---------------------------------------------------------------- attention
__device__ __forceinline__ f32x4 mfma16(Vec8<bf16>::type a, Vec8<bf16>::type b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mfma16(Vec8<fp16>::type a, Vec8<fp16>::type b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Eight codes c of a word as 16 + c in 16 bits: a code's four bits become the highest of the mantissa of 16.  Codes 0 and 4,
// 1 and 5, .. stand side by side.
// (`sixteens`: twice 16, in a vector register, so that "and" and "or" are one instruction, which takes one constant.)
template <class E> constexpr unsigned kSixteens = std::is_same<E, bf16>::value ? 0x41804180u : 0x4c004c00u;
template <class E> __device__ __forceinline__ typename Vec8<E>::type codes8(unsigned w, unsigned sixteens) {
    if (std::is_same<E, bf16>::value) {
        const unsigned m = 0x00780078u;
        return as8<E>(u32x4{(w << 3 & m) | sixteens, (w >> 1 & m) | sixteens, (w >> 5 & m) | sixteens, (w >> 9 & m) | sixteens});
    }
    const unsigned m = 0x03c003c0u;
    return as8<E>(u32x4{(w << 6 & m) | sixteens, (w << 2 & m) | sixteens, (w >> 2 & m) | sixteens, (w >> 6 & m) | sixteens});
}

// acc + the sum of two neighbours
__device__ __forceinline__ float both_added(Pair<bf16>::type x, float acc) { return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(Pair<short>::type, x), Pair<short>::type{0x3f80, 0x3f80}, acc, false); }
__device__ __forceinline__ float both_added(Pair<fp16>::type x, float acc) { return __builtin_amdgcn_fdot2(x, Pair<fp16>::type{(fp16)1.f, (fp16)1.f}, acc, false); }

__device__ __forceinline__ float quarters_max(float x) { x = fmaxf(x, __shfl_xor(x, 16)); return fmaxf(x, __shfl_xor(x, 32)); }
__device__ __forceinline__ float quarters_sum(float x) { x += __shfl_xor(x, 16); return x + __shfl_xor(x, 32); }

struct PackedArgs {
    ReadArgs r;
    long long row_bytes;              // stride
    int heads_in, rows_in, streams;   // of a block: key heads, groups of 16 rows, wavefronts that share a head's tiles
    int row_groups, ways;             // of 16 / ways rows
    int table_words;                  // of biases, per key head
};

constexpr int kPackedTile = 64;  // entries of a wavefront at a time

// Bytes of a wavefront's piece of LDS: values' codes, scales and bases, ids and places of biases.
constexpr int piece_bytes(int groups) { return kPackedTile * (16 * groups + 16 * groups + 4); }

// N scores of a lane under a cap, in place: by the near form where all of the wavefront's are near, as cap_scores.
template <int N> __device__ __forceinline__ void cap_some(const ScoreArgs &s, float (&z)[N]) {
    float size = 0.f;
#pragma unroll
    for (int e = 0; e < N; e++) size = fmaxf(size, __builtin_fabsf(z[e]));
    const bool far = wave_any(size > s.most);
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; e++) y[e] = near_capped(s, z[j + e]);
        if (far) {
#pragma unroll
            for (int e = 0; e < 4; e++) y[e] = any_capped(s, z[j + e]);
        }
#pragma unroll
        for (int e = 0; e < 4; e++) z[j + e] = y[e];
    }
}

// One block: 2^shift entries of a list, some key heads and groups of 16 / WAYS rows (token, head of the group); a wavefront has
// one of each, and every so manieth tile of 64 entries.  With x = base + scale c (a group of 32 elements),
//     q.k = sum over groups of scale (q . c) + base (sum of q),      out = sum of (p scale) c + p base :
// the matrix instructions take the codes as they are, as 16 + c (see codes8), and the scales stay in 32 bits: those of the keys
// are factors of a group's product (which begins at -16 times the sum of q), those of the values go into the weights, which are
// rounded to 16 bits for the second product (as p itself is elsewhere).  16 + c would let that rounding weigh as much as the
// code is large: the sum of the rounded weights times 23.5 is taken off, which makes it c - 7.5, and 7.5 scale goes to the base.
//
// Keys go from memory into the registers that the instruction reads; values' codes lie in LDS as they come, and the transposing
// 4-bit read gives a lane one element of 16 entries.
//
// The instructions' 16 columns are rows of q.  Eight rows or fewer leave columns empty, and with them most of the lanes' work
// between the two products: then the columns stand WAYS times for the rows, each time for other entries of the tile (16
// neighbours of every 16 WAYS).  A lane keeps of the first product what is its own entries', its weights stand in the
// second one's operand beside zeros, and the ways' sums are joined at the end.
//
// 1,024 lists of up to 3,000 entries, four tokens, 16 / 8 heads of 64: 327 us, of which the loads alone take 292 and the lines that they bring
// (0.8 GB) 166 at a copy's rate.  The eight heads of a row ask for its lines at eight times; vector instructions (450 for 64 entries of eight rows) and
// matrix instructions take 60 % of the cycles, the rest are waits that four wavefronts leave.  Rows fetched by the block together, straight into
// LDS, come in 163, but hold the wavefronts to one step (331 in all; 64 lists of up to 20,000, 32 / 8 heads of 128: 262, so 204); a barrier
// before every fetch, so that heads share lines, 359; two heads a wavefront, with half as many lines asked for, the same.
template <class E, int NG, int WAYS, bool CAP, bool BIAS>
__global__ __launch_bounds__(512, NG <= 2 ? 4 : 2) void k_read_packed(PackedArgs pa) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const ReadArgs &a = pa.r;
    constexpr int kBytes = 16 * NG, kOut = 2 * NG, kPiece = piece_bytes(NG), kRows = 16 / WAYS, kTiles = 4 / WAYS, kMine = 16 / WAYS;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, quarter = lane >> 4;
    const int way = col / kRows, my = 16 * way + 4 * quarter;  // a lane's entries of a tile: my .. my + 3 of every 16 WAYS
    const int units = pa.heads_in * pa.rows_in, unit = wave % units, stream = wave / units;
    char *codes = lds + wave * kPiece;
    float *params = (float *)(codes + kPackedTile * kBytes);  // [NG][key scale, key base, value scale, value base][64]
    int *places = (int *)(params + 4 * NG * kPackedTile);
    float *tables = (float *)(lds + pa.streams * units * kPiece);
    const int head_groups = a.kv_heads / pa.heads_in;
    // the key heads of a block's entries one behind the other on one of the card's eight dies, which blocks take turns with
    const unsigned turn = blockIdx.x >> 3;
    const int first_head = (int)(turn % head_groups) * pa.heads_in, head = first_head + unit % pa.heads_in;
    const long long block = a.first + (long long)(turn / head_groups) * 8 + (blockIdx.x & 7);
    if (block >= a.blocks) return;
    const int d = document_of(a.off, a.num_queries, a.num_entries, 1, a.shift, block, lane);
    const long long b0 = first_block(a.off, d, a.num_entries, 1, a.shift);
    const long long e0 = taken_into(a.off[d], a.num_entries), e1 = taken_into(a.off[d + 1], a.num_entries);
    const long long len = e1 > e0 ? e1 - e0 : 0, from = (block - b0) << a.shift;
    if (from < 0 || (from > 0 && from >= len)) return;
    const bool alone = len <= (1ll << a.shift);
    const int n = (int)(len - from < (1ll << a.shift) ? len - from : 1ll << a.shift);
    const int32_t *entity = a.entity ? a.entity + e0 + from : nullptr;
    const uint8_t *hop = a.hop ? a.hop + e0 + from : nullptr;

    const char *rows = (const char *)a.keys;
    const int all = a.kv_heads * NG;
    const unsigned row_bytes = (unsigned)pa.row_bytes;
    auto id_of = [&](int t) {
        const int at = t * kPackedTile + lane;
        if (at >= n) return -1;
        const long long id = entity ? entity[at] : e0 + from + at;
        return id >= 0 && id < a.num_entities ? (int)id : -1;
    };
    auto hop_of = [&](int t) {
        const int at = t * kPackedTile + lane;
        return hop && at < n ? (int)hop[at] : 0;
    };
    // Rows of the tile of codes: row 16 h + j holds the entry whose weight is element j of quarter h in the second product's
    // operands (two steps of eight, see below).
    auto entry_of = [](int p) {
        const int h = p >> 4, j = p & 15, r = j & 3, sub = WAYS == 2 ? 2 * (j >> 2 & 1) + (j >> 3) : j >> 2;
        return 16 * sub + 4 * h + r;
    };
    unsigned k[4][NG];
    u32x4 v[NG];
    u64 param[NG];
    // (of global memory: loads of a place that may be LDS too are waited for with every read of LDS)
    typedef const __attribute__((address_space(1))) char global_bytes;
    typedef const __attribute__((address_space(1))) unsigned global_words;
    typedef const __attribute__((address_space(1))) u32x4 global_chunk;
    typedef const __attribute__((address_space(1))) u64 global_pair;
    // A lane makes the place of its own entry's row; the others get it by shuffles.  (The first row stands in for entries that are left
    // out: their scales, bases and weights are 0.)
    auto row_of = [&](u64 own, int entry) {
        const unsigned lo = (unsigned)__shfl((int)(unsigned)own, entry), hi = (unsigned)__shfl((int)(unsigned)(own >> 32), entry);
        return (global_bytes *)((u64)hi << 32 | lo);
    };
    auto own_row = [&](int id) { return (u64)(uintptr_t)rows + (u64)(unsigned)(id < 0 ? 0 : id) * row_bytes; };
    auto fetch_keys = [&](u64 own) {
#pragma unroll
        for (int t = 0; t < 4; t++) {
            global_words *at = (global_words *)(row_of(own, 16 * t + col) + head * kBytes) + quarter * NG;
#pragma unroll
            for (int i = 0; i < NG; i++) k[t][i] = at[i];
        }
    };
    auto fetch = [&](u64 own) {
#pragma unroll
        for (int i = 0; i < NG; i++) {
            const int chunk = i * 64 + lane;
            v[i] = *(global_chunk *)(row_of(own, entry_of(chunk / NG)) + 16 * all + head * kBytes + chunk % NG * 16);
        }
#pragma unroll
        for (int i = 0; i < NG; i++) param[i] = *(global_pair *)((global_bytes *)(uintptr_t)own + 32 * all + (head * NG + i) * 8);
    };
    const int tiles = a.num_entities > 0 ? (n + kPackedTile - 1) / kPackedTile : 0;
    int id = id_of(stream), next_id = id_of(stream + pa.streams), now_hop = 0, next_hop = 0;
    if (BIAS) now_hop = hop_of(stream), next_hop = hop_of(stream + pa.streams);
    u64 own = own_row(id);
    if (stream < tiles) fetch(own), fetch_keys(own);

    const int row_group = blockIdx.y * pa.rows_in + unit / pa.heads_in, vr = row_group * kRows + col % kRows;
    const bool mine = vr < a.rows;
    const int token = mine ? vr / a.group : 0, g = mine ? vr % a.group : 0;
    const long long place = ((long long)d * a.tokens + token) * a.heads + head * a.group + g;
    typename Vec8<E>::type q[NG];
    float q_sum[NG];  // of a group's elements
#pragma unroll
    for (int i = 0; i < NG; i++) {
        const int c = 32 * i + 8 * quarter;
        u32x4 x = {0, 0, 0, 0};
        if (mine && c < a.dim) x = *(const u32x4 *)((const E *)a.q + place * a.dim + c);
        const typename Vec8<E>::type y = as8<E>(x);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) sum += (float)y[e];
        q_sum[i] = quarters_sum(sum);
        q[i] = __builtin_shufflevector(y, y, 0, 4, 1, 5, 2, 6, 3, 7);
    }
    const int q_pos = a.q_pos ? a.q_pos[d] : 0, M = a.score.max_distance;
    const float *my_table = tables + (unit % pa.heads_in) * pa.table_words + g * (2 * M + 1);
    if (BIAS) {  // of the block's heads, one behind the other
        bias_to_lds<E>(tables, a.score, first_head * a.group, pa.heads_in * a.group, tid, blockDim.x);
        __syncthreads();
    }
    f32x4 o[kOut];
    float base_sum[NG], weight_sum[NG];
#pragma unroll
    for (int i = 0; i < kOut; i++) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NG; i++) base_sum[i] = weight_sum[i] = 0.f;
    float m = kLowest, l = 0.f;
    float unit_scale = std::is_same<E, bf16>::value ? 1.f : 0.f;  // of the weights: see below
    unsigned sixteens = kSixteens<E>;
    here(sixteens);
    // of the second product's two steps, the lanes and halves of registers that a weight stands in
    const unsigned keep[2] = {WAYS == 1 ? ~0u : WAYS == 2 ? (way == 0 ? ~0u : 0u) : way == 0 ? 0xffffu : way == 1 ? 0xffff0000u : 0u,
                              WAYS == 1 ? ~0u : WAYS == 2 ? (way == 1 ? ~0u : 0u) : way == 2 ? 0xffffu : way == 3 ? 0xffff0000u : 0u};
    // chunks of a row of the tile of codes change places, so that the 16 rows that a read goes down lie in different banks
    constexpr int kTurn = NG == 4 ? 3 : NG == 2 ? 1 : 0;
    const unsigned codes_at = lds_place(codes) + (16 * quarter + col) * kBytes + ((NG == 4 ? col >> 2 : col >> 3) & kTurn) * 16;
    char *codes_to = codes + lane / NG * kBytes + ((lane % NG) ^ ((lane >> 4) & kTurn)) * 16;

    for (int t = stream; t < tiles; t += pa.streams) {
        const u64 seen = __ballot(id >= 0);
        if (!std::is_same<E, bf16>::value) {
            // float16 holds weights down to 2^-24 only: they are multiplied by a power of two by which the values' largest scale so far
            // is about 1
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < NG; i++) top = id < 0 ? 0.f : fmaxf(top, __builtin_fabsf(low_half((unsigned)(param[i] >> 32))));
            if (wave_any(top * unit_scale > 1024.f || (unit_scale == 0.f && top > 0.f))) {
#pragma unroll
                for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
                int power = 127 - (int)(__builtin_bit_cast(unsigned, top) >> 23 & 255);
                power = power < -100 ? -100 : power > 100 ? 100 : power;
                const float now = __builtin_bit_cast(float, (unsigned)(power + 127) << 23), change = unit_scale > 0.f ? now / unit_scale : 1.f;
#pragma unroll
                for (int i = 0; i < kOut; i++) o[i] *= change;
#pragma unroll
                for (int i = 0; i < NG; i++) weight_sum[i] *= change;
                unit_scale = now;
            }
        }
#pragma unroll
        for (int i = 0; i < NG; i++) *(u32x4 *)(NG == 3 ? codes + (i * 64 + lane) * 16 : codes_to + i * 1024) = v[i];
#pragma unroll
        for (int i = 0; i < NG; i++) {
            const unsigned kp = id < 0 ? 0u : (unsigned)param[i], vp = id < 0 ? 0u : (unsigned)(param[i] >> 32);
            const float vs = low_half(vp);
            params[(4 * i + 0) * 64 + lane] = low_half(kp);
            params[(4 * i + 1) * 64 + lane] = high_half(kp);
            params[(4 * i + 2) * 64 + lane] = vs * unit_scale;
            params[(4 * i + 3) * 64 + lane] = __builtin_fmaf(7.5f, vs, high_half(vp));
        }
        if (BIAS) places[lane] = distance_place(now_hop, q_pos, M);
        wave_sync();
        id = next_id;
        now_hop = next_hop;
        own = own_row(id);
        if (t + pa.streams < tiles) fetch(own);
        next_id = id_of(t + 2 * pa.streams);
        if (BIAS) next_hop = hop_of(t + 2 * pa.streams);
        float s[kMine];
#pragma unroll
        for (int b = 0; b < kTiles; b++) {
            float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NG; i++) {  // a group's product, and its scale and base
                const float begin = -16.f * q_sum[i];
                f32x4 z = mfma16(codes8<E>(k[WAYS * b][i], sixteens), q[i], f32x4{begin, begin, begin, begin});
#pragma unroll
                for (int x = 1; x < WAYS; x++) {
                    const f32x4 other = mfma16(codes8<E>(k[WAYS * b + x][i], sixteens), q[i], f32x4{begin, begin, begin, begin});
#pragma unroll
                    for (int e = 0; e < 4; e++) z[e] = way == x ? other[e] : z[e];
                }
                const f32x4 ks = *(const f32x4 *)(params + (4 * i + 0) * 64 + 16 * WAYS * b + my);
                const f32x4 kb = *(const f32x4 *)(params + (4 * i + 1) * 64 + 16 * WAYS * b + my);
#pragma unroll
                for (int e = 0; e < 4; e++) y[e] = __builtin_fmaf(ks[e], z[e], __builtin_fmaf(kb[e], q_sum[i], y[e]));
            }
#pragma unroll
            for (int e = 0; e < 4; e++) {
                here(y[e]);  // (else the compiler makes all scores behind the next branch, with what they are made of in registers until then)
                s[4 * b + e] = y[e];
            }
        }
        if (t + pa.streams < tiles) fetch_keys(own);
        if (CAP) cap_some(a.score, s);
#pragma unroll
        for (int b = 0; b < kTiles; b++) {
            int4 at = {0, 0, 0, 0};
            if (BIAS) at = *(const int4 *)(places + 16 * WAYS * b + my);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if (!CAP) s[4 * b + e] *= a.score.k;
                if (BIAS) s[4 * b + e] += my_table[e == 0 ? at.x : e == 1 ? at.y : e == 2 ? at.z : at.w];
            }
        }
        if (seen != ~0ull) {
#pragma unroll
            for (int b = 0; b < kTiles; b++) {
                const unsigned open = (unsigned)(seen >> (16 * WAYS * b + my));
#pragma unroll
                for (int e = 0; e < 4; e++) s[4 * b + e] = open >> e & 1 ? s[4 * b + e] : -INFINITY;
            }
        }
        float top = kLowest;
#pragma unroll
        for (int e = 0; e < kMine; e++) top = fmaxf(top, s[e]);
        top = quarters_max(top);
        if (wave_any(top > m)) {
            const float up = fmaxf(m, top), shrink = exp2_fast(m - up);
            m = up;
            l *= shrink;
#pragma unroll
            for (int i = 0; i < kOut; i++) o[i] *= shrink;
#pragma unroll
            for (int i = 0; i < NG; i++) weight_sum[i] *= shrink, base_sum[i] *= shrink;
        }
#pragma unroll
        for (int e = 0; e < kMine; e++) {
            s[e] = exp2_fast(s[e] - m);
            l += s[e];
        }
        typedef int v2i __attribute__((ext_vector_type(2)));
        typedef __attribute__((address_space(3))) v2i lds2;
#pragma unroll
        for (int i = 0; i < NG; i++) {
            u32x4 w[2];  // of the second product's two steps; element 2 r (+ 1) is entry r of a neighbourhood of 16 (of the next)
            f32x4 ws[kTiles];
#pragma unroll
            for (int b = 0; b < kTiles; b++) {
                const f32x4 vs = *(const f32x4 *)(params + (4 * i + 2) * 64 + 16 * WAYS * b + my);
                const f32x4 vb = *(const f32x4 *)(params + (4 * i + 3) * 64 + 16 * WAYS * b + my);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    base_sum[i] = __builtin_fmaf(s[4 * b + e], vb[e], base_sum[i]);
                    ws[b][e] = s[4 * b + e] * vs[e];
                }
            }
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if (WAYS == 1) {
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        const unsigned x = rounded2<E>(ws[2 * j % kTiles][e], ws[(2 * j + 1) % kTiles][e]);
                        weight_sum[i] = both_added(__builtin_bit_cast(typename Pair<E>::type, x), weight_sum[i]);  // (of w[j][e] it would take w[j][0])
                        w[j][e] = x;
                    }
                } else {
                    const unsigned x = rounded2<E>(ws[0][e], ws[kTiles - 1][e]);
                    const unsigned once = WAYS == 2 ? x : x & 0xffffu;
                    weight_sum[i] = both_added(__builtin_bit_cast(typename Pair<E>::type, once), weight_sum[i]);
                    w[0][e] = x & keep[0];
                    w[1][e] = x & keep[1];
                }
            }
#pragma unroll
            for (int j = 2 * i; j < 2 * i + 2; j++) {
                const v2i x = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds2 *)(uintptr_t)((codes_at ^ (NG == 3 ? 0 : i << 4)) + (NG == 3 ? i << 4 : 0) + (j & 1) * 8));
                o[j] = mfma16(codes8<E>((unsigned)x[0], sixteens), as8<E>(w[0]), o[j]);
                o[j] = mfma16(codes8<E>((unsigned)x[1], sixteens), as8<E>(w[1]), o[j]);
            }
        }
        wave_sync();
    }
    // the output of this wavefront's entries: element 16 j + 4 quarter + e of the lane's row
    const float back = unit_scale > 0.f ? 1.f / unit_scale : 1.f;
    l = quarters_sum(l);
#pragma unroll
    for (int i = 0; i < NG; i++) base_sum[i] = quarters_sum(base_sum[i]), weight_sum[i] = -23.5f * quarters_sum(weight_sum[i]);
#pragma unroll
    for (int j = 0; j < kOut; j++)
#pragma unroll
        for (int e = 0; e < 4; e++) o[j][e] = __builtin_fmaf(o[j][e] + weight_sum[j / 2], back, base_sum[j / 2]);
#pragma unroll
    for (int x = kRows; x < 16; x <<= 1) {  // the ways' sums together
        const float om = __shfl_xor(m, x), ol = __shfl_xor(l, x), up = fmaxf(m, om), mine_by = exp2_fast(m - up), other_by = exp2_fast(om - up);
        l = l * mine_by + ol * other_by;
#pragma unroll
        for (int j = 0; j < kOut; j++)
#pragma unroll
            for (int e = 0; e < 4; e++) o[j][e] = o[j][e] * mine_by + __shfl_xor(o[j][e], x) * other_by;
        m = up;
    }
    if (pa.streams > 1) {  // joined with the others that have the same rows, in their order
        __syncthreads();
        float *box = (float *)(lds + wave * kPiece);
        if (stream > 0) {
#pragma unroll
            for (int j = 0; j < kOut; j++) *(f32x4 *)(box + (j * 64 + lane) * 4) = o[j];
            if (quarter == 0) box[kOut * 256 + col] = m, box[kOut * 256 + 16 + col] = l;
        }
        __syncthreads();
        if (stream > 0) return;
        for (int w = 1; w < pa.streams; w++) {
            const float *other = (const float *)(lds + (wave + w * units) * kPiece);
            const float om = other[kOut * 256 + col], ol = other[kOut * 256 + 16 + col];
            const float up = fmaxf(m, om), mine_by = exp2_fast(m - up), other_by = exp2_fast(om - up);
            m = up;
            l = l * mine_by + ol * other_by;
#pragma unroll
            for (int j = 0; j < kOut; j++) o[j] = o[j] * mine_by + *(const f32x4 *)(other + (j * 64 + lane) * 4) * other_by;
        }
    }
    if (!mine || way > 0) return;
    if (alone) {
        const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
        for (int j = 0; j < kOut; j++) {
            const int c = 16 * j + 4 * quarter;
            if (c >= a.dim) continue;
            typename Vec4<E>::type x;
#pragma unroll
            for (int e = 0; e < 4; e++) x[e] = (E)(o[j][e] * inv);
            *(typename Vec4<E>::type *)((E *)a.out + place * a.dim + c) = x;
        }
        if (quarter == 0) a.lse[place] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
    } else {
        const long long at = (block * a.tokens + token) * a.heads + head * a.group + g;
#pragma unroll
        for (int j = 0; j < kOut; j++) {
            const int c = 16 * j + 4 * quarter;
            if (c < a.dim) *(f32x4 *)(a.part_o + at * a.dim + c) = o[j];
        }
        if (quarter == 0) a.part_ml[2 * at] = m, a.part_ml[2 * at + 1] = l;
    }
}

static logoskg_status packed_args(const logoskg_entity_read *r, PackedArgs *pa, const char *call) {
    if (!r || r->struct_size != sizeof(logoskg_entity_read)) { set_error("%s: struct_size", call); return LOGOSKG_EINVAL; }
    const char *why = bad_heads(r->dtype, r->heads, r->kv_heads, r->dim);
    if (!why) why = bad_score(r->score, r->heads, r->kv_heads);
    if (!why && (r->num_queries < 0 || r->tokens < 1 || r->tokens > 65535 || r->num_entries < 0 || r->num_entities < 0)) why = "a count is out of range";
    if (!why && r->num_entities >= (1ll << 31)) why = "num_entities is 2^31 or more";
    if (!why && !r->entity && r->num_entities < r->num_entries) why = "fewer rows than entries";
    if (!why && r->num_queries && (!r->off || !r->q || !r->out || !r->lse)) why = "off, q, out or lse is NULL";
    if (!why && r->num_entries && r->num_entities && !r->keys) why = "the table is NULL";
    if (!why && (r->values || r->key_head || r->value_row || r->value_head)) why = "values or strides beside a packed table";
    if (!why && (((uintptr_t)r->q | (uintptr_t)r->keys | (uintptr_t)r->out | (uintptr_t)r->workspace) & 15)) why = "an array is not 16-byte aligned";
    if (!why && (r->key_row & 15 || r->key_row < 0 || r->key_row > (1ll << 31) || (r->num_entities > 1 && r->key_row < row_bytes_of(r->kv_heads, (r->dim + 31) / 32)))) why = "the rows' stride is no multiple of 16, or rows overlap";
    if (why) { set_error("%s: %s", call, why); return LOGOSKG_EINVAL; }
    memset(pa, 0, sizeof *pa);
    ReadArgs *a = &pa->r;
    a->num_queries = r->num_queries; a->tokens = r->tokens; a->heads = r->heads; a->kv_heads = r->kv_heads;
    a->group = r->heads / r->kv_heads; a->dim = r->dim; a->rows = a->tokens * a->group;
    a->num_entries = r->num_entries; a->num_entities = r->num_entities;
    a->off = r->off; a->entity = r->entity; a->q_pos = r->q_pos; a->hop = r->hop;
    a->q = r->q; a->keys = r->keys; pa->row_bytes = r->key_row;
    a->score = score_args(r->score);
    a->out = r->out; a->lse = r->lse;
    // A block's eight wavefronts: as many key heads as divide theirs, whose rows lie side by side (64 lists of up to 20,000 entries, 32 / 8
    // heads of 128: 340 us with two in a block, 204 with eight), and have room for their biases; then groups of rows; then streams of
    // tiles.  Fewer heads where blocks would not do for the card (one list of 900: 12.4 us with eight, 9.5 with one).
    pa->ways = a->rows <= 4 ? 4 : a->rows <= 8 ? 2 : 1;
    pa->row_groups = (a->rows * pa->ways + 15) / 16;
    pa->table_words = a->score.bias ? a->group * (2 * a->score.max_distance + 1) : 0;
    const int groups = (a->dim + 31) / 32, piece = piece_bytes(groups), room = (groups <= 2 ? 80 : 150) << 10;  // (two blocks of a unit, or one)
    long long each = 0;  // blocks per 2^shift entries
    for (int h = 8; h >= 1; h--) {
        if (a->kv_heads % h || (h > 1 && 8 * piece + h * pa->table_words * 4 > room)) continue;
        pa->heads_in = h;
        pa->rows_in = 8 / h < pa->row_groups ? 8 / h : pa->row_groups;
        each = (a->kv_heads / h) * (long long)((pa->row_groups + pa->rows_in - 1) / pa->rows_in);
        if (((a->num_entries >> 6) + a->num_queries) * each >= 256) break;
    }
    // Blocks of 64 entries, larger ones (up to 4,096) where there are more than eight rounds of them: a block's begin costs as much as some tiles
    a->shift = 6;
    // Few entries go to one block a list, whose wavefronts share it, and nothing is joined behind, a launch and a workspace less: up to 4,096, where an
    // average list is a tile or two for each of the wavefronts that share it (and where those are one or two, 512 each).  (One token, 32 / 8 heads of 128, a call and on the GPU: one list of 200 14.7
    // and 10.6 us, so 10.0 and 8.6; 16 of 250 14.8 and 12.8, so 11.6 and 11.3; one of 900 would be 14.8 and 12.6, 14.7 and 14.5, of 4,000 22 and 34.
    // Of heads of 64 one of 900 14.5 and 10.4, so 10.2 and 9.3.)
    const int spare = 8 / (pa->heads_in * pa->rows_in);  // wavefronts to a list
    const long long few = std::min<long long>(spare >= 4 ? 4096 : 512 * spare, (long long)(groups <= 2 ? 128 : 64) * spare * a->num_queries);
    while (a->num_entries <= few && a->num_entries >> a->shift > 0) a->shift++;
    while (a->shift < 12 && (a->num_entries >> a->shift) * each > (groups <= 2 ? 4096 : 2048)) a->shift++;
    const int tiles = 1 << (a->shift - 6);
    pa->streams = tiles < spare ? tiles : spare;
    a->blocks = (a->num_entries >> a->shift) + a->num_queries;
    if ((a->blocks + 8) * (a->kv_heads / pa->heads_in) >= (1ll << 31) || pa->row_groups > 65535 || (long long)a->num_queries * a->tokens * a->heads >= (1ll << 32)) { set_error("%s: too many rows", call); return LOGOSKG_EINVAL; }
    return LOGOSKG_OK;
}

template <class E, int NG, int WAYS, bool CAP, bool BIAS> static logoskg_status launch_packed(PackedArgs pa, hipStream_t st) {
    ReadArgs &a = pa.r;
    const int waves = pa.heads_in * pa.rows_in * pa.streams;
    const size_t bytes = (size_t)waves * piece_bytes(NG) + (size_t)pa.heads_in * pa.table_words * 4;
    LKG_TRY(allow_lds(k_read_packed<E, NG, WAYS, CAP, BIAS>, bytes));
    const unsigned row_blocks = (unsigned)((pa.row_groups + pa.rows_in - 1) / pa.rows_in);
    each_eight_blocks(a, a.kv_heads / pa.heads_in, waves * 64, [&](unsigned blocks) { k_read_packed<E, NG, WAYS, CAP, BIAS><<<dim3(blocks, row_blocks), waves * 64, bytes, st>>>(pa); });
    LKG_HIP(hipGetLastError());
    return LOGOSKG_OK;
}
template <class E, int NG, int WAYS> static logoskg_status launch_packed(const PackedArgs &pa, hipStream_t st) {
    const bool cap = pa.r.score.c > 0, bias = pa.r.score.bias != nullptr;
    return cap ? bias ? launch_packed<E, NG, WAYS, true, true>(pa, st) : launch_packed<E, NG, WAYS, true, false>(pa, st)
               : bias ? launch_packed<E, NG, WAYS, false, true>(pa, st) : launch_packed<E, NG, WAYS, false, false>(pa, st);
}
template <class E, int NG> static logoskg_status read_packed(const PackedArgs &pa, hipStream_t st) {
    return pa.ways == 4 ? launch_packed<E, NG, 4>(pa, st) : pa.ways == 2 ? launch_packed<E, NG, 2>(pa, st) : launch_packed<E, NG, 1>(pa, st);
}
template <class E> static logoskg_status read_packed(const PackedArgs &pa, hipStream_t st) {
    const ReadArgs &a = pa.r;
    const int groups = (a.dim + 31) / 32;
    LKG_TRY((groups == 1 ? read_packed<E, 1>(pa, st) : groups == 2 ? read_packed<E, 2>(pa, st) : groups == 3 ? read_packed<E, 3>(pa, st) : read_packed<E, 4>(pa, st)));
    return launch_join<E>(a, st);
}

static const char *pack_args(const logoskg_pack *p, PackArgs *a) {
    if (!p || p->struct_size != sizeof(logoskg_pack)) return "struct_size";
    if (p->dtype < LOGOSKG_F32 || p->dtype > LOGOSKG_F16) return "unknown type";
    if (logoskg_packed_row_bytes(p->kv_heads, p->dim) == 0) return "dim is no multiple of 8 up to 128, or kv_heads out of range";
    if (p->num_rows < 0 || p->num_rows > (1ll << 31)) return "a count is out of range";
    if (p->num_rows && (!p->keys || !p->values || !p->packed)) return "keys, values or packed is NULL";
    if (!aligned_to(p->keys, p->dtype) || !aligned_to(p->values, p->dtype)) return kUnaligned;
    if (p->key_row < 0 || p->key_head < 0 || p->value_row < 0 || p->value_head < 0) return "a stride is negative";
    if (((uintptr_t)p->packed & 15) || p->packed_row & 15 || p->packed_row < 0 || (p->num_rows > 1 && p->packed_row < logoskg_packed_row_bytes(p->kv_heads, p->dim)))
        return "packed is not 16-byte aligned, its stride no multiple of 16, or its rows overlap";
    memset(a, 0, sizeof *a);
    a->kv_heads = p->kv_heads; a->dim = p->dim; a->groups = (p->dim + 31) / 32;
    a->pad = row_bytes_of(a->kv_heads, a->groups) - 40 * a->kv_heads * a->groups;
    a->num_rows = p->num_rows; a->keys = p->keys; a->values = p->values;
    a->key_row = p->key_row; a->key_head = p->key_head; a->value_row = p->value_row; a->value_head = p->value_head;
    a->packed = (char *)p->packed; a->packed_row = p->packed_row;
    return nullptr;
}

static logoskg_status pack(const logoskg_pack *p, bool back, const char *call) {
    PackArgs a;
    if (const char *why = pack_args(p, &a)) { set_error("%s: %s", call, why); return LOGOSKG_EINVAL; }
    if (a.num_rows == 0) return LOGOSKG_OK;
    OnDevice on;
    LKG_TRY(on.go(p->device));
    hipStream_t st = (hipStream_t)p->stream;
    const int items = a.kv_heads * a.groups, rows = items < 64 ? 64 / items : 1;
    const long long blocks = (a.num_rows + rows - 1) / rows;
    const long long most = back ? 1 << 20 : 1 << 14;  // (packing 407,000 rows: 527 us with 16,384 blocks, 554 with 4,096, 632 with one a row; back 400, 440 and 390)
    const dim3 grid((unsigned)(blocks > most ? most : blocks));
    if (p->dtype == LOGOSKG_F32) back ? k_unpack<float><<<grid, 256, 0, st>>>(a) : k_pack<float><<<grid, 256, 0, st>>>(a);
    else if (p->dtype == LOGOSKG_BF16) back ? k_unpack<bf16><<<grid, 256, 0, st>>>(a) : k_pack<bf16><<<grid, 256, 0, st>>>(a);
    else back ? k_unpack<fp16><<<grid, 256, 0, st>>>(a) : k_pack<fp16><<<grid, 256, 0, st>>>(a);
    LKG_HIP(hipGetLastError());
    return LOGOSKG_OK;
}

}  // namespace lkg

using namespace lkg;

extern "C" int64_t logoskg_packed_row_bytes(int32_t kv_heads, int32_t dim) {
    return kv_heads < 1 || kv_heads > 65536 || dim < 8 || dim > 128 || dim % 8 ? 0 : row_bytes_of(kv_heads, (dim + 31) / 32);
}

extern "C" logoskg_status logoskg_pack_entities(const logoskg_pack *p) { return pack(p, false, "logoskg_pack_entities"); }
extern "C" logoskg_status logoskg_unpack_entities(const logoskg_pack *p) { return pack(p, true, "logoskg_unpack_entities"); }

extern "C" int64_t logoskg_read_packed_bytes(const logoskg_entity_read *r) {
    PackedArgs pa;
    return packed_args(r, &pa, "logoskg_read_packed_bytes") == LOGOSKG_OK ? part_bytes(pa.r) : -1;
}

extern "C" logoskg_status logoskg_read_packed(const logoskg_entity_read *r) {
    PackedArgs pa;
    LKG_TRY(packed_args(r, &pa, "logoskg_read_packed"));
    ReadArgs &a = pa.r;
    if (r->workspace_bytes < part_bytes(a) || (part_bytes(a) && !r->workspace)) {
        set_error("logoskg_read_packed: the workspace has %lld of %lld bytes", (long long)r->workspace_bytes, (long long)part_bytes(a));
        return LOGOSKG_ERANGE;
    }
    if (a.num_queries == 0) return LOGOSKG_OK;
    a.part_o = (float *)r->workspace;
    a.part_ml = a.part_o + (part_bytes(a) ? a.blocks * a.tokens * a.heads * a.dim : 0);
    OnDevice on;
    LKG_TRY(on.go(r->device));
    return r->dtype == LOGOSKG_BF16 ? read_packed<bf16>(pa, (hipStream_t)r->stream) : read_packed<fp16>(pa, (hipStream_t)r->stream);
}
