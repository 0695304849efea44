// Attention of a ragged batch with capped scores, a learned distance bias and a prefix + causal mask (logoskg_attend).
#include "attend.h"

namespace lkg {

// One block: 128 rows of (document, key head), where a row is a (row of q, head of the group) pair, so that the heads that
// share a key head share its tiles.  A wavefront holds 32 rows: lane l works for row l % 32 and half of the keys, so a row's
// maximum and sum are its own registers and one exchange with the other half.  Keys pass in tiles of 64 through two buffers
// for K and two for V in LDS: S^T = K Q^T, p = 2^(y - m), O^T += V^T P^T with m the running maximum.
//
// The vector units bound this: a score costs them about twelve issue slots (a tanh among them), its products four.  So the
// products of the next tile's scores and of the last tile's values are issued between the exponentials of this one, one
// matrix instruction a step, and a tile is spared what costs most when nothing special is asked of it: all its keys are visible, all
// its distances read one bias (text far from the row, which is most of a long document), the scores are in the range of the
// tanh's polynomial, and the maximum does not move by more than 8.  m need not be the true maximum: p stays below 2^8 and
// is summed in 32 bits.  (The test takes b - m: against m + 8 it would lose the scores beside a bias of large size.)  Other tiles get their y - m first, with m the maximum again, which takes them twice as long.
//
// 4 documents of up to 8,192 rows and keys (32 / 8 heads of 128, bfloat16, cap, bias; two fifths of the pairs are between
// entities, whose distances vary): 2,130 us, 680 TFLOP/s of the 1,370 that a product of 16,384^3 reaches here; text alone, whose
// tiles are plain, without a cap: 860.  By the counters the matrix units are busy for 36 % of the time (4 x 4,096 rows),
// LDS banks collide for 2 %.  p is rounded to 16 bits as the matrix instruction takes it, the sum l is of the unrounded ones.
//
// A document's own hidden keys are multiplied with p = 0: infinities and NaN in their values reach the rows of their tile.
constexpr int kKeys = 64;

template <class E, int DP, bool CAP, bool BIAS>
__global__ __launch_bounds__(kAttThreads, 2) void k_attend(AttArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    typedef typename Vec8<E>::type Chunk;
    constexpr int kTile = kKeys * DP * 2, kSteps = DP / 16, kOut = DP / 32;
    int *kpos = (int *)(lds + 4 * kTile);              // [4][kKeys]  (LDS begins with K, K, V, V)
    float *table = (float *)(kpos + 4 * kKeys);        // [group][2 M + 1]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int head = blockIdx.x % a.kv_heads;
    const long long block = a.row_blocks - 1 - blockIdx.x / a.kv_heads;  // the last rows of a document see most: first
    const int d = document_of(a.q_off, a.num_docs, a.num_rows, a.group, kAttRowsShift, block, lane);
    const AttDoc doc = att_doc(a, d);
    const long long first = (block - first_block(a.q_off, d, a.num_rows, a.group, kAttRowsShift)) << kAttRowsShift;
    const long long vrows = (long long)doc.rows * a.group;
    each_spare<kAttRows>(doc.row0 * a.group, vrows, a.num_rows * a.group, d, a.num_docs, block, first, tid, [&](long long at) {
        const long long spare = at / a.group * a.heads + head * a.group + at % a.group;
        clear_row((E *)a.out + spare * a.dim, a.dim);
        a.lse[spare] = -INFINITY;
    });
    if (first >= vrows || first < 0) return;

    const long long vr = first + wave * 32 + (lane & 31);
    const bool mine = vr < vrows;
    const long long vr_in = mine ? vr : vrows - 1;
    const int row = (int)(vr_in / a.group), g = (int)(vr_in % a.group);
    const int seen = mine ? doc.seen(row, a.causal) : 0;
    // of the block's first and last row
    const int least = doc.seen((int)(first / a.group), a.causal);
    const long long last_v = first + kAttRows < vrows ? first + kAttRows - 1 : vrows - 1;
    const int most = doc.seen((int)(last_v / a.group), a.causal);

    const int h = head * a.group + g;
    const E *qrow = (const E *)a.q + (doc.row0 + row) * a.q_row + (long long)h * a.q_head;
    Chunk q[kSteps];
#pragma unroll
    for (int kk = 0; kk < kSteps; kk++) q[kk] = row_chunk<E>(qrow, mine, kk, a.dim, lane);
    const int M = a.score.max_distance;
    const float *my_table = table + g * (2 * M + 1);
    int q_low = 0, q_high = 0;  // the wavefront's lowest and highest position
    Places places = {0, 0, 0};
    if (BIAS) {
        const int q_pos = a.q_pos ? a.q_pos[doc.row0 + row] : row + (doc.keys - doc.rows);
        places = places_of_keys(q_pos, M, lds_place(my_table));
        q_low = __builtin_amdgcn_readfirstlane(wave_min(q_pos));
        q_high = __builtin_amdgcn_readfirstlane(wave_max(q_pos));
        bias_to_lds<E>(table, a.score, head * a.group, a.group, tid, kAttThreads);
    }

    const char *kbase = (const char *)a.k + (doc.key0 * a.k_row + (long long)head * a.k_head) * 2;
    const char *vbase = (const char *)a.v + (doc.key0 * a.v_row + (long long)head * a.v_head) * 2;
    f32x16 o[kOut], s[2] = {zero16(), zero16()};
    Chunk p[4];  // of the last tile, 16 keys each
#pragma unroll
    for (int i = 0; i < 4; i++) p[i] = as8<E>(u32x4{0, 0, 0, 0});
#pragma unroll
    for (int i = 0; i < kOut; i++) o[i] = zero16();
    float m = kLowest, l = 0.f, size = 0.f;  // size: the largest product of the tile, without its sign

    TileLoad<kKeys, DP> kload, vload;
    kload.begin(kbase, (unsigned)a.k_row * 2, 0, doc.keys, a.dim, tid);
    vload.begin(vbase, (unsigned)a.v_row * 2, 0, doc.keys, a.dim, tid);
    const unsigned tiles = lds_place(lds), my_rows = rows_place<DP>(lane) + tiles, my_columns = columns_place<DP>(lane) + tiles + 2 * kTile;
    auto buffer = [](int t) { return (unsigned)(t & 1) * kTile; };
    u32x4 x[TileLoad<kKeys, DP>::kChunks];
    int kp = 0;
    const int tiles_n = (most + kKeys - 1) / kKeys;
    auto fetch_pos = [&](int t) {
        if (BIAS && tid < kKeys) {
            int j = t * kKeys + tid;
            j = j < doc.keys ? j : doc.keys - 1;
            kp = a.k_pos && doc.keys > 0 ? a.k_pos[doc.key0 + j] : j;
        }
    };
    auto stage_pos = [&](int t) {
        if (BIAS && tid < kKeys) kpos[(t & 3) * kKeys + tid] = kp;
    };
    // Round t makes the scores of tile t + 1 and the output of tile t - 1.  K of tile t + 2 and V of tile t come in meanwhile,
    // one after the other through the same registers.
    if (tiles_n > 0) {
        kload.load(x);
        kload.store(tiles, x);
        fetch_pos(0);
        stage_pos(0);
        kload.load(x);
        kload.store(tiles + kTile, x);
        fetch_pos(1);
        stage_pos(1);
        kload.load(x);
        fetch_pos(2);
        stage_pos(2);
        fetch_pos(3);
        vload.clear(tiles + 2 * kTile + buffer(1));  // (round 0 multiplies it with zeros)
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kSteps; kk++)
#pragma unroll
            for (int u = 0; u < 2; u++) s[u] = mfma(rows_chunk<E>(my_rows + u * 32 * DP * 2, kk), q[kk], s[u]);
#pragma unroll
        for (int r = 0; r < 32; r++) size = fmaxf(size, __builtin_fabsf(s[r / 16][r % 16]));
        __syncthreads();
    }
    // one bias for all distances of a tile? (the wavefront's keys, a lane each, from its lowest and its highest row)
    bool varied = false;
    float b = 0.f;
    auto look_at = [&](int pos) {
        const int y = distance_place(pos, q_high, M), z = distance_place(pos, q_low, M), y0 = __builtin_amdgcn_readfirstlane(y);
        varied = wave_any(y != y0 || z != y0);
        b = my_table[y0];
    };
    if (BIAS && tiles_n > 0) look_at(kpos[lane]);
    for (int t = 0; t < tiles_n; t++) {
        const bool edge = (t + 1) * kKeys > least;  // some row does not see all of the tile
        const bool far = wave_any(size > a.score.most);
        const bool plain = !edge && !far && !varied && !wave_any(__builtin_fmaf(size, a.score.slope, b - m) > 8.f);
        // p = 2^(w + shift), w = z times the polynomial of `near` (CAP) or z near[0]; the other way leaves y - m in z
        float shift = b - m, near0 = CAP ? a.score.near[0] : a.score.k, near1 = a.score.near[1], near2 = a.score.near[2], near3 = a.score.near[3];
        float shrink = 1.f;
        if (!plain) {
            const int *kpt = kpos + (t & 3) * kKeys;
            float top = kLowest;
            if (!edge && !far) {
#pragma unroll
                for (int u = 0; u < 2; u++)
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        float y = BIAS ? float_at(place_of_key(places, kpt[32 * u + 8 * (r / 4) + 4 * half + r % 4])) : 0.f;
                        const float z = s[u][r];
                        if (CAP) {
                            const float zz = z * z;
                            float w = __builtin_fmaf(zz, near3, near2);
                            w = __builtin_fmaf(zz, w, near1);
                            w = __builtin_fmaf(zz, w, near0);
                            y = __builtin_fmaf(z, w, y);
                        } else y = __builtin_fmaf(z, near0, y);
                        s[u][r] = y;
                        top = fmaxf(top, y);
                        if (r % 8 == 7) __builtin_amdgcn_sched_barrier(0);  // (no more in registers than these)
                    }
            } else {
#pragma unroll
                for (int u = 0; u < 2; u++)
                    if (CAP) cap_scores<1>(a.score, s[u]);
#pragma unroll
                for (int u = 0; u < 2; u++)
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        const int at = 32 * u + 8 * (r / 4) + 4 * half + r % 4;
                        float y = CAP ? s[u][r] : s[u][r] * a.score.k;
                        if (BIAS) y += float_at(place_of_key(places, kpt[at]));
                        y = t * kKeys + at < seen ? y : -INFINITY;
                        s[u][r] = y;
                        top = fmaxf(top, y);
                        if (r % 8 == 7) __builtin_amdgcn_sched_barrier(0);  // (no more in registers than these)
                    }
            }
            top = halves_max(top);
            if (wave_any(top > m + 8.f)) {
                const float up = fmaxf(m, top);
                shrink = exp2_fast(m - up);
                m = up;
                l *= shrink;
            }
#pragma unroll
            for (int u = 0; u < 2; u++)
#pragma unroll
                for (int r = 0; r < 16; r++) s[u][r] -= m;
            if (CAP && (edge || far)) {  // (2^-1e15 is 0; its square is finite, where that of the infinity of a hidden key is not)
#pragma unroll
                for (int u = 0; u < 2; u++)
#pragma unroll
                    for (int r = 0; r < 16; r++) s[u][r] = s[u][r] < -1e15f ? -1e15f : s[u][r];
            }
            shift = 0.f, near0 = 1.f, near1 = near2 = near3 = 0.f;
        }
        const unsigned kt = my_rows + buffer(t + 1), vt = my_columns + buffer(t - 1);
        // First the output, whose weights' registers then take the new ones, and the scores of the next tile those of this
        // one's: everything fits 256 registers, two wavefronts to a unit.
        constexpr int kAll = 4 * kSteps, kAhead = 3, kStages = 4;
        Chunk piece[4];
        auto piece_of = [&](int at) __attribute__((always_inline)) {
            if (at < 2 * kSteps) return columns_chunk<E, DP>(vt, 16 * (at / kOut), at % kOut);
            return rows_chunk<E>(kt + (at & 1) * 32 * DP * 2, (at - 2 * kSteps) >> 1);
        };
#pragma unroll
        for (int i = 0; i < kAhead; i++) piece[i] = piece_of(i);
        f32x16 next[2] = {zero16(), zero16()};
        float square[32], w[32];  // (few of them at a time)
        unsigned packed[16];
        in_turn<kAll + kStages - 1>([&](auto step) __attribute__((always_inline)) {
            constexpr int at = decltype(step)::value;
            __builtin_amdgcn_sched_barrier(0);
            if (at + kAhead < kAll) piece[(at + kAhead) & 3] = piece_of(at + kAhead);
            if (at < 2 * kSteps) o[at % kOut] = mfma(piece[at & 3], p[at / kOut & 3], o[at % kOut]);
            else if (at < kAll) next[at & 1] = mfma(piece[at & 3], q[(at - 2 * kSteps) >> 1], next[at & 1]);  // (behind the last tile: of what the buffer holds, not used)
#pragma unroll
            for (int e = first_of<kAll>(at); e < first_of<kAll>(at + 1); e++) {
                const float z = s[e / 16][e % 16];
                if (CAP) {
                    square[e] = z * z;
                    w[e] = __builtin_fmaf(square[e], near3, near2);
                    here(w[e]);
                }
            }
#pragma unroll
            for (int e = first_of<kAll>(at - 1); e < first_of<kAll>(at); e++)
                if (CAP) {
                    w[e] = __builtin_fmaf(square[e], w[e], near1);
                    w[e] = __builtin_fmaf(square[e], w[e], near0);
                    here(w[e]);
                }
#pragma unroll
            for (int e = first_of<kAll>(at - 2); e < first_of<kAll>(at - 1); e++) {
                w[e] = exp2_fast(__builtin_fmaf(s[e / 16][e % 16], CAP ? w[e] : near0, shift));
                here(w[e]);
            }
#pragma unroll
            for (int e = first_of<kAll>(at - 3); e < first_of<kAll>(at - 2); e++) {
                l += w[e];
                if (e & 1) {
                    packed[e / 2] = rounded2<E>(w[e - 1], w[e]);
                    here(packed[e / 2]);
                }
            }
            here(l);
            if (BIAS && at == kAll / 4) look_at(kpos[((t + 1) & 3) * kKeys + lane]);
            if (at == 0) {
                kload.store(tiles + buffer(t), x);  // K of t + 2, where that of t was (read in the last round)
                vload.load(x);
            }
            if (at == kAll / 2 + 2) {
                vload.store(tiles + 2 * kTile + buffer(t), x);  // V of t, where that of t - 2 was
                kload.load(x);
            }
        });
        __builtin_amdgcn_sched_barrier(0);
        if (wave_any(shrink != 1.f)) {
#pragma unroll
            for (int i = 0; i < kOut; i++) o[i] *= shrink;
        }
#pragma unroll
        for (int i = 0; i < 4; i++) p[i] = as8<E>(u32x4{packed[4 * i], packed[4 * i + 1], packed[4 * i + 2], packed[4 * i + 3]});
        s[0] = next[0];
        s[1] = next[1];
        size = 0.f;
#pragma unroll
        for (int r = 0; r < 32; r++) size = fmaxf(size, __builtin_fabsf(s[r / 16][r % 16]));
        __syncthreads();
        if (BIAS) {
            stage_pos(t + 3);  // (seen from the barrier of the next round on)
            fetch_pos(t + 4);
        }
    }
    if (tiles_n > 0) {
        const unsigned vt = my_columns + buffer(tiles_n - 1);
#pragma unroll
        for (int i = 0; i < 4 * kOut; i++) o[i % kOut] = mfma(columns_chunk<E, DP>(vt, 16 * (i / kOut), i % kOut), p[i / kOut], o[i % kOut]);
    }
    l = halves_sum(l);
    if (!mine) return;
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;  // (a NaN stays one)
    const long long place = (doc.row0 + row) * a.heads + h;
    write_row<E, DP>(o, inv, (E *)a.out + place * a.dim, a.dim, half);
    if (half == 0) a.lse[place] = l == 0.f ? -INFINITY : (m + __log2f(l)) * kLn2;
}

// Few rows: one block is 32 rows of (document, key head), and its four wavefronts take every fourth tile of 32 keys and
// join at the end, so that a short prompt before many keys is spread over four times the units and each of them does a
// quarter of the keys.  As in the read of entity lists, keys go from memory into the registers that the matrix
// instruction reads and values through the wavefront's own piece of LDS; no wavefront waits for another.
constexpr int kFewKeys = 32;

template <class E, int DP, bool CAP, bool BIAS>
__global__ __launch_bounds__(kAttThreads, 2) void k_attend_few(AttArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int kTile = kFewKeys * DP * 2, kSteps = DP / 16, kOut = DP / 32, kRow = DP / 8;  // kRow: chunks of a row
    float *table = (float *)(lds + 4 * kTile);  // [group][2 M + 1]
    __shared__ __attribute__((aligned(16))) int kpos[4][kFewKeys];
    __shared__ float wave_m[4][32], wave_l[4][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int head = blockIdx.x % a.kv_heads;
    const long long block = a.few_blocks - 1 - blockIdx.x / a.kv_heads;  // the last rows of a document see most: first
    const int d = document_of(a.q_off, a.num_docs, a.num_rows, a.group, kFewShift, block, lane);
    const AttDoc doc = att_doc(a, d);
    const long long first = (block - first_block(a.q_off, d, a.num_rows, a.group, kFewShift)) << kFewShift;
    const long long vrows = (long long)doc.rows * a.group;
    each_spare<1 << kFewShift>(doc.row0 * a.group, vrows, a.num_rows * a.group, d, a.num_docs, block, first, tid, [&](long long at) {
        const long long spare = at / a.group * a.heads + head * a.group + at % a.group;
        clear_row((E *)a.out + spare * a.dim, a.dim);
        a.lse[spare] = -INFINITY;
    });
    if (first >= vrows || first < 0) return;

    const long long vr = first + (lane & 31);
    const bool mine = vr < vrows;
    const long long vr_in = mine ? vr : vrows - 1;
    const int row = (int)(vr_in / a.group), g = (int)(vr_in % a.group), h = head * a.group + g;
    const int seen = mine ? doc.seen(row, a.causal) : 0;
    const int least = doc.seen((int)(first / a.group), a.causal);  // of the block's first row, and of its last
    const int most = doc.seen((int)((first + 31 < vrows ? first + 31 : vrows - 1) / a.group), a.causal);
    const int tiles_n = (most + kFewKeys - 1) / kFewKeys;

    const E *keys = (const E *)a.k + doc.key0 * a.k_row + (long long)head * a.k_head;
    const E *values = (const E *)a.v + doc.key0 * a.v_row + (long long)head * a.v_head;
    u32x4 k[kSteps], v[kSteps];
    int kp = 0;
    auto fetch = [&](int t) {
        const long long j = (long long)t * kFewKeys + (lane & 31);
        const E *krow = keys + j * a.k_row;
#pragma unroll
        for (int kk = 0; kk < kSteps; kk++) k[kk] = __builtin_bit_cast(u32x4, row_chunk<E>(krow, j < doc.keys, kk, a.dim, lane));
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            const int at = i * 64 + lane, c = (at % kRow) * 8;
            const long long r = (long long)t * kFewKeys + at / kRow;
            v[i] = r < doc.keys && c < a.dim ? *(const u32x4 *)(values + r * a.v_row + c) : u32x4{0, 0, 0, 0};
        }
        if (BIAS) {
            const int in = j < doc.keys ? (int)j : doc.keys - 1;
            kp = a.k_pos ? a.k_pos[doc.key0 + in] : in;
        }
    };
    if (wave < tiles_n) fetch(wave);
    const E *qrow = (const E *)a.q + (doc.row0 + row) * a.q_row + (long long)h * a.q_head;
    typename Vec8<E>::type q[kSteps];
#pragma unroll
    for (int kk = 0; kk < kSteps; kk++) q[kk] = row_chunk<E>(qrow, mine, kk, a.dim, lane);
    Places places = {0, 0, 0};
    if (BIAS) {
        const int M = a.score.max_distance;
        places = places_of_keys(a.q_pos ? a.q_pos[doc.row0 + row] : row + (doc.keys - doc.rows), M, lds_place(table + g * (2 * M + 1)));
        bias_to_lds<E>(table, a.score, head * a.group, a.group, tid, kAttThreads);
        __syncthreads();
    }
    f32x16 o[kOut];
#pragma unroll
    for (int i = 0; i < kOut; i++) o[i] = zero16();
    float m = kLowest, l = 0.f;
    char *vt = lds + wave * kTile;
    const unsigned my_columns = columns_place<DP>(lane) + lds_place(vt);

    for (int t = wave; t < tiles_n; t += 4) {
        f32x16 s = zero16();
#pragma unroll
        for (int kk = 0; kk < kSteps; kk++) s = mfma(as8<E>(k[kk]), q[kk], s);
#pragma unroll
        for (int i = 0; i < kSteps; i++) {
            const int at = i * 64 + lane, r = at / kRow, c = at % kRow;
            *(u32x4 *)(vt + r * (DP * 2) + ((c ^ spread<DP>(r)) << 4)) = v[i];
        }
        if (BIAS && lane < kFewKeys) kpos[wave][lane] = kp;
        wave_sync();
        if (t + 4 < tiles_n) fetch(t + 4);
        const bool edge = (t + 1) * kFewKeys > least;
        if (CAP) cap_scores<4>(a.score, s);
        float top = kLowest;
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const u32x4 p4 = BIAS ? *(const u32x4 *)(kpos[wave] + 8 * j + 4 * half) : u32x4{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int r = 4 * j + e;
                float y = CAP ? s[r] : s[r] * a.score.k;
                if (BIAS) y += float_at(place_of_key(places, (int)p4[e]));
                if (edge) y = t * kFewKeys + 8 * j + 4 * half + e < seen ? y : -INFINITY;
                s[r] = y;
                top = fmaxf(top, y);
            }
        }
        top = halves_max(top);
        if (wave_any(top > m)) {
            const float up = fmaxf(m, top), shrink = exp2_fast(m - up);
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
    if (wave != 0 || !mine) return;
    const long long place = (doc.row0 + row) * a.heads + h;
    const float sum = all.sum, inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    write_row<E, DP>(o, inv, (E *)a.out + place * a.dim, a.dim, half);
    if (half == 0) a.lse[place] = sum == 0.f ? -INFINITY : (all.top + __log2f(sum)) * kLn2;
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
    if (!why && (a->q_row < 0 || a->k_row < 0 || a->v_row < 0 || a->k_row >= kMostStride || a->v_row >= kMostStride || a->q_row >= kMostStride)) why = "a row stride is negative or too large";
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
    o->few_blocks = (a->num_rows * o->group >> kFewShift) + a->num_docs;
    o->key_blocks = (a->num_keys >> kAttRowsShift) + a->num_docs;
    o->scale = a->score.scale;
    o->curve = o->score.c > 0 ? (float)(-(double)a->score.scale / ((double)o->score.c * o->score.c)) : 0.f;
    o->slope = 4.f * a->score.scale;
    if (o->row_blocks * a->kv_heads > kMaxBlocks) { set_error("%s: too many rows", call); return LOGOSKG_EINVAL; }
    return LOGOSKG_OK;
}

// Blocks of 128 rows x key heads up to which rows are few (k_attend / k_attend_few, us, with cap and bias and without):
//   heads of 128   16 blocks: 33 rows before 300 entities 24.4 / 13.5 and 14.7 / 10.5, before 5,000 204 / 77 and 98 / 60
//                  128: 500 rows before 300 entities 34 / 27 and 23.7 / 23.1, before 2,000 94 / 62 and 54 / 57
//                  168: 16 documents of 24 rows before 1,000 50 / 32 and 26.5 / 28.6; 256: 1,000 rows before 2,000 96 / 120, 66 / 106
//   heads of 64    192: 3,000 rows before 300 entities 74 / 49 and 51 / 41; 432: 32 documents of 200 rows 31 / 23 and 17.2 / 18.5
constexpr long long few_blocks_most(int DP) { return DP == 64 ? 256 : 128; }

template <class E, int DP, bool CAP, bool BIAS> static logoskg_status launch_attend(const AttArgs &a, hipStream_t st) {
    const size_t table = BIAS ? (size_t)a.group * (2 * a.score.max_distance + 1) * 4 : 0;
    if (a.row_blocks * a.kv_heads <= few_blocks_most(DP)) {
        const size_t few = 4 * kFewKeys * DP * 2 + table;
        LKG_TRY(allow_lds(k_attend_few<E, DP, CAP, BIAS>, few));
        k_attend_few<E, DP, CAP, BIAS><<<dim3((unsigned)(a.few_blocks * a.kv_heads)), kAttThreads, few, st>>>(a);
        LKG_HIP(hipGetLastError());
        return LOGOSKG_OK;
    }
    size_t bytes = 4 * kKeys * DP * 2 + 4 * kKeys * 4 + table;
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
