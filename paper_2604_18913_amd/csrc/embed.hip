// Rows of a table by the ids of retrieved lists, and their gradient summed by entity (logoskg_embed_entities,
// logoskg_embed_entities_backward).
#include "training.h"

namespace lkg {

static_assert(sizeof(logoskg_embedding) == 80 && sizeof(logoskg_embedding_grad) == 104, "the ctypes binding mirrors these layouts");

struct EmbedArgs {
    long long num_ids, num_entities, dim, row;
    float scale;
    const int32_t *ids;
    const void *table;
    void *out;
};

constexpr int kEmbedPieces = 4;  // of a thread

// Where a lane begins whose V elements from c on would end behind the row: at the last V of it, some of which the lane before has too
// and makes the same of.  (Element by element such ends take the whole wavefront eight times as many instructions: gradients of 200,000
// rows of 333 in bfloat16 180 us, so 110.)
__device__ __forceinline__ long long ends_at(long long c, long long dim, int V) { return c + V > dim && dim >= V ? dim - V : c; }

// The output is one run of pieces of 16 bytes, `pieces` to a row; a thread moves kEmbedPieces, a block's threads lie side by side.  Memory
// bounds it: 590,000 rows of 512 in bfloat16 (1.45 GB with the table's) 297 us, 4.9 TB/s.  (A group of lanes per row leaves some of them without
// work: 200,000 rows of 328 in 32 bits 104 us, so 92.)
template <class T> __global__ __launch_bounds__(256) void k_embed(EmbedArgs a, unsigned pieces, unsigned inverse) {
    constexpr int V = 16 / sizeof(T);
    const long long begin = (long long)blockIdx.x * (256 * kEmbedPieces), first = begin / pieces;
    const unsigned from = (unsigned)(begin - first * pieces) + threadIdx.x;
    long long row[kEmbedPieces], id[kEmbedPieces], c[kEmbedPieces];
#pragma unroll
    for (int r = 0; r < kEmbedPieces; r++) {
        const unsigned at = from + r * 256;
        unsigned q = __umulhi(at, inverse);  // at / pieces, or one less
        q += at - q * pieces >= pieces;
        row[r] = first + q;
        c[r] = ends_at((long long)(at - q * pieces) * V, a.dim, V);
        id[r] = row[r] < a.num_ids ? a.ids[row[r]] : -1;
    }
    const int count = a.dim < V ? (int)a.dim : V;
    Some<T> x[kEmbedPieces];
#pragma unroll
    for (int r = 0; r < kEmbedPieces; r++) {
        const bool in = id[r] >= 0 && id[r] < a.num_entities;
        x[r] = in ? load_some<T>((const T *)a.table + id[r] * a.row + c[r], count) : Some<T>{};
    }
#pragma unroll
    for (int r = 0; r < kEmbedPieces; r++) {
        if (row[r] >= a.num_ids) continue;
        const bool in = id[r] >= 0 && id[r] < a.num_entities;
        Some<T> y;
#pragma unroll
        for (int e = 0; e < V; e++) y[e] = in ? (T)((float)x[r][e] * a.scale) : (T)0.f;
        store_some<T>((T *)a.out + row[r] * a.dim + c[r], y, count);
    }
}

// ---------------------------------------------------------------- gradient
// The ids are sorted with their places (by counting, or by stable passes of a radix sort, so that equal ids keep the order of the list); ids
// outside the table become num_entities and come last.  Then every run of equal ids is a sum of rows of dout: chunks of the sorted
// list are added up by groups of lanes, and runs that cross chunks are joined from the chunks' parts, in their order.
struct GradArgs {
    long long num_ids, num_entities, dim, row, chunks;
    int accumulate, chunk, tile, tiles, bits;
    int gaps;  // whether rows without an id are cleared between the sums, and not before
    float scale;
    const int32_t *ids;
    const void *dout;
    void *dtable;
    unsigned *key[2], *place[2];  // of the sort: from one to the other and back
    unsigned *count, *total;      // [tiles][digits], [digits]
    float *part;                  // [chunks][2][dim]: of the run that comes in from the chunk before, and of the one that goes on
    unsigned *gap_pieces;         // how many there are of ..
    uint2 *gap;                   // .. pieces of long gaps: first row and the one behind
};

constexpr int kMostChunk = 64, kFewParts = 16;  // entries of the sorted list; parts of a run that 16 lanes join
constexpr int kGapRows = 32, kGapPiece = 512, kGapBlocks = 1024;  // rows without an id that the sums' kernel clears between two ids; rows of a piece of more; blocks for those
constexpr int kFewIds = 12288, kMostDigitBits = 11;

__device__ __forceinline__ unsigned key_of(const GradArgs &a, long long i) {
    const int id = a.ids[i];
    return (unsigned)id < a.num_entities ? (unsigned)id : (unsigned)a.num_entities;
}

// Lanes of the wavefront that have this lane's digit.
__device__ __forceinline__ unsigned long long alike(unsigned digit, int bits, bool in) {
    unsigned long long m = __ballot(in);
    for (int b = 0; b < bits; b++) {
        const unsigned long long set = __ballot(digit >> b & 1);
        m &= digit >> b & 1 ? set : ~set;
    }
    return m;
}

// Exclusive sums over a block's threads; `all`: the sum of all.  `box`: THREADS / 64 words of LDS.
template <int THREADS> __device__ __forceinline__ unsigned block_before(unsigned x, unsigned *box, unsigned &all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned y = x;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const unsigned z = __shfl_up(y, s);
        if (lane >= s) y += z;
    }
    __syncthreads();
    if (lane == 63) box[wave] = y;
    __syncthreads();
    unsigned before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; w++) {
        if (w == wave) before = all;
        all += box[w];
    }
    return before + y - x;
}

// Rows [from, to) of the table become zeros, by a block.
template <class O, int THREADS> __device__ __forceinline__ void clear_rows(const GradArgs &a, long long from, long long to) {
    constexpr int V = 16 / sizeof(O);
    const long long chunks = (a.dim + V - 1) / V;
    if (a.row == a.dim && a.dim % V == 0) {  // one run of whole chunks
        typename Loose<O>::type *p = (typename Loose<O>::type *)((O *)a.dtable + from * a.row);
        for (long long i = threadIdx.x; i < (to - from) * chunks; i += THREADS) p[i] = Some<O>{};
        return;
    }
    const int LG = chunks <= 4 ? 4 : chunks <= 16 ? 16 : 64, lane = threadIdx.x % LG;
    for (long long e = from + threadIdx.x / LG; e < to; e += THREADS / LG)
        for (long long first = (long long)lane * V; first < a.dim; first += LG * V) {
            const long long c = ends_at(first, a.dim, V);
            store_some<O>((O *)a.dtable + e * a.row + c, Some<O>{}, a.dim - c < V ? (int)(a.dim - c) : V);
        }
}

// The table is cleared before the sums, by blocks beside those of the sort, which is a chain of short waits: a part of it in each of
// the sort's launches.  Rows that ids name are written twice then; where these can be more than kTwice bytes, the others are cleared
// between the sums instead, where the sorted ids leave gaps.  (65,536 ids to 300,000 rows of 64 in 32 bits: 50 us a call with the table
// cleared before, 78 between; to 300,000 rows of 512 in 16 bits 110 and 124; to 30,000 of 2,000 in 32 bits (240 MB) 247 and 220.  550,000 ids to
// 407,000 rows of 1,024 in 16 bits (833 MB): 563 and 507.)
constexpr long long kTwice = 192ll << 20;
struct Rows {
    long long from, to;
    int blocks;
};
template <class O, int THREADS> __device__ __forceinline__ void clear_share(const GradArgs &a, const Rows &r, long long block) {
    const long long n = r.to - r.from;
    clear_rows<O, THREADS>(a, r.from + n * block / r.blocks, r.from + n * (block + 1) / r.blocks);
}

// Lists of up to kFewIds ids: an id's place is the number of ids before it in the order, counted over all of them, two instructions
// each.  A block has 16 PER ids and splits the list among 64 lanes of each; the other blocks clear the table.
// (1,984 ids, 10,000 rows of 512 in 32 bits to clear: 5.5 us; a radix sort by one block beside the clears 9.1.  12,288 ids to 30,000
// rows of 64: 20 us, by the passes below 25 and two launches more.)
template <class O, int PER, int MOST> __global__ __launch_bounds__(1024) void k_sort_few(GradArgs a, Rows rows) {
    constexpr int L = 16, IDS = L * PER;
    __shared__ __attribute__((aligned(16))) unsigned key[MOST];
    __shared__ unsigned box[16][IDS];
    const int n = (int)a.num_ids, ranks = (n + IDS - 1) / IDS;
    if ((int)blockIdx.x >= ranks) return clear_share<O, 1024>(a, rows, blockIdx.x - ranks);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, quads = (n + 3) / 4;
    for (int i = tid; i < quads * 4; i += 1024) key[i] = i < n ? key_of(a, i) : ~0u;
    __syncthreads();
    const int begin = blockIdx.x * IDS + tid % L;
    unsigned mine[PER], rank[PER];
#pragma unroll
    for (int p = 0; p < PER; p++) mine[p] = begin + p * L < n ? key[begin + p * L] : 0, rank[p] = 0;
#pragma unroll 4
    for (int j = tid / L * 4; j < quads * 4; j += 256) {  // of four ids those that are smaller, or as large and before
        const u32x4 x = *(const u32x4 *)(key + j);
#pragma unroll
        for (int p = 0; p < PER; p++) {
            const unsigned most = mine[p] + (j < ((begin + p * L) & ~3));
#pragma unroll
            for (int e = 0; e < 4; e++) rank[p] += x[e] < most;
        }
    }
#pragma unroll
    for (int p = 0; p < PER; p++) {
        const int i = begin + p * L, first = i & ~3;
        if (tid < L && i < n)  // (of the id's own four)
#pragma unroll
            for (int e = 0; e < 3; e++) rank[p] += first + e < i && key[first + e] == mine[p];
        rank[p] += __shfl_xor(rank[p], 16);
        rank[p] += __shfl_xor(rank[p], 32);
        if (lane < L) box[wave][p * L + lane] = rank[p];
    }
    __syncthreads();
    const int i = blockIdx.x * IDS + tid;
    if (tid >= IDS || i >= n) return;
    unsigned to = 0;
#pragma unroll
    for (int w = 0; w < 16; w++) to += box[w][tid];
    a.key[0][to] = key[i], a.place[0][to] = i;
}

// A pass of the sort over tiles, of 512 ids, or 2,048 where those are enough for the card: how often a digit occurs in each tile ..  (A chain of
// waits: 65,536 ids 4.8 us here, 4.6 and 8.1 in the two behind, with tiles of 2,048 11 in the last; 550,000 ids 6.6, 4.9 and 18; counts by
// digit, tile after tile, 8.7, 4.8 and 18; 6 million ids 16, 20 and 155.)
template <class O> __global__ __launch_bounds__(256) void k_sort_count(GradArgs a, int pass, int shift, int bits, Rows rows) {
    extern __shared__ unsigned found[];
    if ((int)blockIdx.x >= a.tiles) return clear_share<O, 256>(a, rows, blockIdx.x - a.tiles);
    const int tid = threadIdx.x, digits = 1 << bits;
    if (blockIdx.x == 0 && tid == 0) *a.gap_pieces = 0;
    for (int i = tid; i < digits; i += 256) found[i] = 0;
    __syncthreads();
    const long long from = (long long)blockIdx.x * a.tile;
    for (int i = tid; i < a.tile; i += 256) {
        if (from + i >= a.num_ids) break;
        const unsigned key = pass == 0 ? key_of(a, from + i) : a.key[pass & 1][from + i];
        atomicAdd(&found[key >> shift & (digits - 1)], 1u);
    }
    __syncthreads();
    for (int i = tid; i < digits; i += 256) a.count[(long long)blockIdx.x * digits + i] = found[i];
}

// .. how often before each tile, and in all (a block per 16 digits, a 32nd of the tiles to 16 threads) ..
template <class O> __global__ __launch_bounds__(512) void k_sort_before(GradArgs a, int digits, Rows rows) {
    constexpr int kDigits = 16, kSlices = 32, kAhead = 8;
    __shared__ unsigned box[kSlices][kDigits];
    const int blocks = (digits + kDigits - 1) / kDigits;
    if ((int)blockIdx.x >= blocks) return clear_share<O, 512>(a, rows, blockIdx.x - blocks);
    const int d = blockIdx.x * kDigits + threadIdx.x % kDigits, slice = threadIdx.x / kDigits, each = (a.tiles + kSlices - 1) / kSlices;
    const int from = slice * each, to = from + each < a.tiles ? from + each : a.tiles;
    unsigned *count = a.count + d;
    unsigned sum = 0;
    for (int t = from; t < to; t += kAhead) {
        unsigned x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++) x[u] = t + u < to && d < digits ? count[(long long)(t + u) * digits] : 0;
#pragma unroll
        for (int u = 0; u < kAhead; u++) sum += x[u];
    }
    box[slice][threadIdx.x % kDigits] = sum;
    __syncthreads();
    unsigned before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kSlices; w++) {
        if (w == slice) before = all;
        all += box[w][threadIdx.x % kDigits];
    }
    if (d >= digits) return;
    if (slice == 0) a.total[d] = all;
    for (int t = from; t < to; t += kAhead) {
        unsigned x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++) x[u] = t + u < to ? count[(long long)(t + u) * digits] : 0;
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            if (t + u < to) count[(long long)(t + u) * digits] = before;
            before += x[u];
        }
    }
}

// .. and every id to its place: behind the smaller digits, those of the tiles before, the wavefronts before and the lanes before.
template <class O, int TILE> __global__ __launch_bounds__(256) void k_sort_move(GradArgs a, int pass, int shift, int bits, Rows rows) {
    constexpr int kRounds = TILE / 256;
    extern __shared__ unsigned count[];  // [4][digits]
    __shared__ unsigned box[4];
    if ((int)blockIdx.x >= a.tiles) return clear_share<O, 256>(a, rows, blockIdx.x - a.tiles);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, digits = 1 << bits;
    unsigned *mine = count + wave * digits;
    // how often this thread's digits occur, in all and in the tiles before
    constexpr int kPer = (1 << kMostDigitBits) / 256;
    const int per = digits < 256 ? 1 : digits / 256, first = tid * per;
    unsigned total[kPer], tile[kPer];
#pragma unroll
    for (int j = 0; j < kPer; j++) {
        const bool in = j < per && first + j < digits;
        total[j] = in ? a.total[first + j] : 0;
        tile[j] = in ? a.count[(long long)blockIdx.x * digits + first + j] : 0;
    }
    for (int i = tid; i < 4 * digits; i += 256) count[i] = 0;
    __syncthreads();
    const long long from = (long long)blockIdx.x * TILE + wave * (TILE / 4);
    unsigned key[kRounds], rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; r++) {
        const long long i = from + r * 64 + lane;
        key[r] = i < a.num_ids ? pass == 0 ? key_of(a, i) : a.key[pass & 1][i] : 0;
    }
#pragma unroll
    for (int r = 0; r < kRounds; r++) {
        const bool in = from + r * 64 + lane < a.num_ids;
        const unsigned digit = key[r] >> shift & (digits - 1);
        const unsigned long long m = alike(digit, bits, in), below = m & ((1ull << lane) - 1);
        rank[r] = mine[digit] + __popcll(below);
        wave_sync();
        if (in && below == 0) mine[digit] += __popcll(m);
        wave_sync();
    }
    __syncthreads();
    // (up to eight digits a thread)
    unsigned all, sum = 0;
#pragma unroll
    for (int j = 0; j < kPer; j++) sum += total[j];
    unsigned before = block_before<256>(sum, box, all);
#pragma unroll
    for (int j = 0; j < kPer; j++) {
        const int d = first + j;
        if (j < per && d < digits) {
            unsigned at = before + tile[j];
            for (int w = 0; w < 4; w++) {
                const unsigned c = count[w * digits + d];
                count[w * digits + d] = at;
                at += c;
            }
        }
        before += total[j];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; r++) {
        const long long i = from + r * 64 + lane;
        if (i >= a.num_ids) continue;
        const unsigned to = mine[key[r] >> shift & (digits - 1)] + rank[r];
        a.key[~pass & 1][to] = key[r];
        a.place[~pass & 1][to] = pass == 0 ? (unsigned)i : a.place[pass & 1][i];
    }
}

// `count` of a lane's V sums, whole chunks of O at a time where all of them count
template <class O, int V> __device__ __forceinline__ void store_sums(O *to, const O (&y)[V], int count) {
    constexpr int N = 16 / sizeof(O) < V ? 16 / sizeof(O) : V;
    typedef O chunk __attribute__((ext_vector_type(N), aligned(sizeof(O))));
    if (count >= V) {
#pragma unroll
        for (int i = 0; i < V; i += N) {
            chunk x;
#pragma unroll
            for (int e = 0; e < N; e++) x[e] = y[i + e];
            *(chunk *)(to + i) = x;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < V - 1; e++)
        if (e < count) to[e] = y[e];
}

// (own: the first of the V that are this lane's alone, see ends_at)
template <class O, int V> __device__ __forceinline__ void write_sum(const GradArgs &a, unsigned id, long long c, int own, int count, const float (&x)[V]) {
    O *to = (O *)a.dtable + (long long)id * a.row + c;
    O y[V];
#pragma unroll
    for (int e = 0; e < V; e++) y[e] = (O)(x[e] * a.scale);
    if (a.accumulate) {
        if (own > 0) {
#pragma unroll
            for (int e = 1; e < V; e++)
                if (e >= own) to[e] = (O)((float)to[e] + x[e] * a.scale);
            return;
        }
#pragma unroll
        for (int e = 0; e < V; e++)
            if (e < count) y[e] = (O)((float)to[e] + x[e] * a.scale);
    }
    store_sums<O, V>(to, y, count);
}

// A group of LG lanes adds up a chunk of the sorted list, each lane 16 bytes of a row; blockIdx.y: further columns.  The list of a
// block's groups goes through LDS first, so that rows are asked for without a wait in between.  Memory bounds it where there are many: 550,000
// rows of 1,024 in bfloat16 to 407,000 (1.96 GB) 416 us, 4.7 TB/s; 65,536 of 64 in 32 bits 14 us, of which memory would take 4.
template <class T, class O, int LG> __global__ __launch_bounds__(256) void k_embed_sum(GradArgs a) {
    constexpr int V = 16 / sizeof(T), kAhead = 8, kGroups = 256 / LG;
    __shared__ unsigned keys[kGroups * kMostChunk + 2], places[kGroups * kMostChunk];
    const int tid = threadIdx.x, group = tid / LG;
    const unsigned none = (unsigned)a.num_entities;
    const long long first = (long long)blockIdx.x * kGroups * a.chunk;
    for (int i = tid; i < kGroups * a.chunk + 2; i += 256) {  // the one before and the one behind, too
        const long long at = first + i - 1;
        keys[i] = at < 0 ? ~0u : at < a.num_ids ? a.key[0][at] : none;
        if (i > 0 && i <= kGroups * a.chunk) places[i - 1] = at < a.num_ids ? a.place[0][at] : 0;
    }
    __syncthreads();
    const long long g = (long long)blockIdx.x * kGroups + group, first_c = ((long long)blockIdx.y * LG + tid % LG) * V, c = ends_at(first_c, a.dim, V);
    if (g >= a.chunks || first_c >= a.dim) return;
    const int count = a.dim - c < V ? (int)(a.dim - c) : V, own = (int)(first_c - c);
    const unsigned *key = keys + 1 + group * a.chunk, *place = places + group * a.chunk;
    unsigned id = key[-1];  // (before the list: -1, behind which the first row comes)
    bool came = id < none;  // the run began before this chunk
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; e++) sum[e] = 0.f;
    float *part = a.part + g * 2 * a.dim + c;
    const T *dout = (const T *)a.dout + c;
    // rows between two ids, which no id names: zeros, here or, where there are many, by the next kernel
    auto gap = [&](unsigned from, unsigned to) __attribute__((always_inline)) {
        if (!a.gaps || from >= to) return;
        if (to - from <= kGapRows) {
            const O zeros[V] = {};
            for (unsigned e = from; e < to; e++) store_sums<O, V>((O *)a.dtable + (long long)e * a.row + c, zeros, count);
        } else if (blockIdx.y == 0) {
            const int lanes = a.dim >= LG * V ? LG : (int)((a.dim + V - 1) / V);  // (of the group, those that are here)
            const unsigned pieces = (to - from + kGapPiece - 1) / kGapPiece;
            for (unsigned i = tid % LG; i < pieces; i += lanes) {
                const unsigned begin = from + i * kGapPiece;
                a.gap[atomicAdd(a.gap_pieces, 1u)] = uint2{begin, to - begin < kGapPiece ? to : begin + kGapPiece};
            }
        }
    };
    bool any = false;  // whether sum holds something: rows of this chunk's
#pragma unroll 1
    for (int i = 0; i < a.chunk; i += kAhead) {
        Some<T> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; u++)
            if (key[i + u] < none) x[u] = load_some<T>(dout + place[i + u] * a.dim, count);
#pragma unroll
        for (int u = 0; u < kAhead; u++) {
            const unsigned k = key[i + u];
            if (k != id) {
                if (any) {
                    if (came) {
                        store_sums<float, V>(part, sum, count);
                    } else {
                        write_sum<O, V>(a, id, c, own, count, sum);
                    }
#pragma unroll
                    for (int e = 0; e < V; e++) sum[e] = 0.f;
                    any = false;
                }
                gap(id + 1, k);
                came = false;
                id = k;
            }
            if (k >= none) continue;
            any = true;
#pragma unroll
            for (int e = 0; e < V; e++) sum[e] += (float)x[u][e];
        }
    }
    if (any) {
        const bool goes_on = key[a.chunk] == id;
        if (came || goes_on) {
            if (!came) part += a.dim;
            store_sums<float, V>(part, sum, count);
        } else {
            write_sum<O, V>(a, id, c, own, count, sum);
        }
    }
    if (g == a.chunks - 1 && id < none) gap(id + 1, none);
}

// Runs that cross chunks, by the chunks that they begin in: 16 lanes have such a chunk and 64 columns (blockIdx.y: further ones).  Runs of
// up to kFewParts parts they add up alone; of the others the block's 16 groups take a share of the parts each.  Further blocks clear the
// long gaps.  (Of the 550,000 rows, a few of which are in most lists: 32 us; of 65,536 4.)
template <class O> __global__ __launch_bounds__(256) void k_embed_join(GradArgs a) {
    constexpr int V = 4, LG = 16, kGroups = 16, kAhead = 4;
    __shared__ float box[kGroups][LG * V];
    __shared__ unsigned many[kGroups];
    const unsigned *key = a.key[0];
    const int lane = threadIdx.x % LG, group = threadIdx.x / LG;
    const long long first = (long long)blockIdx.x * kGroups;
    if (first >= a.chunks) {
        const unsigned block = blockIdx.x - (unsigned)((a.chunks + kGroups - 1) / kGroups), pieces = blockIdx.y == 0 ? *a.gap_pieces : 0;
        for (unsigned i = block; i < pieces; i += kGapBlocks) clear_rows<O, 256>(a, a.gap[i].x, a.gap[i].y);
        return;
    }
    const long long first_c = ((long long)blockIdx.y * LG + lane) * V, c = ends_at(first_c, a.dim, V);
    const int count = first_c >= a.dim ? 0 : a.dim - c < V ? (int)(a.dim - c) : V, own = (int)(first_c - c);
    // parts p .. end - 1 of the run of chunk g, whose first is that chunk's second
    auto add = [&](float (&sum)[V], long long g, long long p, long long end) {
        for (; p < end; p += kAhead) {
            Some<float> x[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; u++)
                x[u] = p + u < end ? load_some<float>(a.part + ((g + p + u) * 2 + (p + u == 0)) * a.dim + c, count) : Some<float>{};
#pragma unroll
            for (int u = 0; u < kAhead; u++)
#pragma unroll
                for (int e = 0; e < V; e++) sum[e] += x[u][e];
        }
    };
    const long long g = first + group;
    long long parts = 0;
    if (g + 1 < a.chunks) {
        const unsigned id = key[(g + 1) * a.chunk - 1], before = g == 0 ? ~0u : key[g * a.chunk - 1];
        if (id < a.num_entities && before != id && key[(g + 1) * a.chunk] == id) {
            long long lo = g + 1, hi = g + 2;  // the last chunk that begins with the run: lo .. hi - 1
            while (hi < a.chunks && key[hi * a.chunk] == id) {
                lo = hi;
                hi = g + 2 * (hi - g);
            }
            if (hi > a.chunks) hi = a.chunks;
            while (hi - lo > 1) {
                const long long mid = (lo + hi) / 2;
                if (key[mid * a.chunk] == id) lo = mid;
                else hi = mid;
            }
            parts = lo - g + 1;
            if (parts <= kFewParts && count > 0) {
                float sum[V] = {0.f, 0.f, 0.f, 0.f};
                add(sum, g, 0, parts);
                write_sum<O, V>(a, id, c, own, count, sum);
            }
        }
    }
    if (lane == 0) many[group] = parts > kFewParts ? (unsigned)parts : 0;
    __syncthreads();
    for (int i = 0; i < kGroups; i++) {
        if (many[i] == 0) continue;
        const long long share = (many[i] + kGroups - 1) / kGroups, end = (group + 1) * share;
        float sum[V] = {0.f, 0.f, 0.f, 0.f};
        if (count > 0) add(sum, first + i, group * share, end < many[i] ? end : many[i]);
#pragma unroll
        for (int e = 0; e < V; e++) box[group][lane * V + e] = sum[e];
        __syncthreads();
        if (group == 0 && count > 0) {
            for (int w = 1; w < kGroups; w++)
#pragma unroll
                for (int e = 0; e < V; e++) sum[e] += box[w][lane * V + e];
            write_sum<O, V>(a, key[(first + i + 1) * a.chunk - 1], c, own, count, sum);
        }
        __syncthreads();
    }
}

static const char *bad_type(int dtype) { return dtype < LOGOSKG_F32 || dtype > LOGOSKG_F16 ? "unknown type" : nullptr; }

template <class T> static logoskg_status launch_embed(const EmbedArgs &all, hipStream_t st) {
    constexpr long long kBlock = 256 * kEmbedPieces;  // pieces
    const long long pieces = (all.dim * (long long)sizeof(T) + 15) / 16;
    launch_ranges(all.num_ids, 1, [&](long long first, long long n) {
        EmbedArgs a = all;
        a.num_ids = n, a.ids += first, a.out = (T *)all.out + first * all.dim;
        k_embed<T><<<dim3((unsigned)((n * pieces + kBlock - 1) / kBlock)), 256, 0, st>>>(a, (unsigned)pieces, (unsigned)(0xffffffffll / pieces));
    }, kMaxBlocks * kBlock / pieces);
    LKG_HIP(hipGetLastError());
    return LOGOSKG_OK;
}

static long long up(long long x) { return (x + 255) / 256 * 256; }

// Sizes of the sort and places in the workspace; its size.  (size: of an element of the table)
static long long plan_grad(GradArgs &a, int size, char *w) {
    a.bits = 1;
    while (a.num_entities >> a.bits) a.bits++;  // (num_entities itself is a key)
    a.tile = a.num_ids < 262144 ? 512 : 2048;
    a.tiles = (int)((a.num_ids + a.tile - 1) / a.tile);
    a.chunk = a.num_ids < 65536 ? 8 : a.num_ids < 262144 ? 32 : 64;
    a.chunks = (a.num_ids + a.chunk - 1) / a.chunk;
    long long at = 0;
    auto take = [&](long long bytes) {
        char *p = w + at;
        at += up(bytes);
        return p;
    };
    const bool few = a.num_ids <= kFewIds;
    for (int i = 0; i < 2; i++) {
        a.key[i] = (unsigned *)take(few && i ? 0 : a.num_ids * 4);
        a.place[i] = (unsigned *)take(few && i ? 0 : a.num_ids * 4);
    }
    const int passes = (a.bits + kMostDigitBits - 1) / kMostDigitBits;
    a.count = (unsigned *)take(few ? 0 : ((long long)a.tiles << (a.bits + passes - 1) / passes) * 4);
    a.total = (unsigned *)take(few ? 0 : 4 << kMostDigitBits);
    a.part = (float *)take(a.chunks * 2 * a.dim * 4);
    a.gaps = !few && !a.accumulate && (a.num_ids < a.num_entities ? a.num_ids : a.num_entities) * a.dim * size > kTwice;
    a.gap_pieces = (unsigned *)take(few ? 0 : 4);
    a.gap = (uint2 *)take(!a.gaps ? 0 : (a.num_ids + 1 + a.num_entities / kGapPiece + 1) * 8);
    return at;
}

static const char *grad_args(const logoskg_embedding_grad *e, GradArgs *a) {
    if (!e || e->struct_size != sizeof(logoskg_embedding_grad)) return "struct_size";
    if (bad_type(e->dtype)) return "unknown type";
    if (e->table_dtype != e->dtype && e->table_dtype != LOGOSKG_F32) return "dtable is neither of dout's type nor float32";
    if (!(e->scale - e->scale == 0.f)) return "scale is not finite";
    if (e->num_ids < 0 || e->num_ids >= (1ll << 31) || e->num_entities < 0 || e->num_entities >= (1ll << 31) - 1 || e->dim < 0 || e->dim > 65535 * 64) return "a count is out of range";
    if (e->row < e->dim && e->num_entities > 1) return "rows overlap";
    if (e->num_ids && e->dim && (!e->ids || !e->dout)) return "ids or dout is NULL";
    if (e->num_entities && e->dim && !e->dtable) return "dtable is NULL";
    if (!aligned_to(e->dout, e->dtype) || !aligned_to(e->dtable, e->table_dtype) || !aligned_to(e->ids, LOGOSKG_F32)) return kUnaligned;
    if ((uintptr_t)e->workspace & 15) return "the workspace is not 16-byte aligned";
    memset(a, 0, sizeof *a);
    a->num_ids = e->num_ids; a->num_entities = e->num_entities; a->dim = e->dim; a->row = e->row;
    a->accumulate = e->accumulate != 0; a->scale = e->scale;
    a->ids = e->ids; a->dout = e->dout; a->dtable = e->dtable;
    return nullptr;
}

template <class O> __global__ __launch_bounds__(256) void k_clear_table(GradArgs a, Rows rows) { clear_share<O, 256>(a, rows, blockIdx.x); }

template <class T, class O> static logoskg_status launch_grad(GradArgs &a, hipStream_t st) {
    // the table from `part` to `next` of `parts`, by blocks that clear some 64 KB each
    auto share = [&](int part, int next, int parts) {
        Rows r = {a.num_entities * part / parts, a.num_entities * next / parts, 0};
        const long long some = (r.to - r.from) * a.dim * (long long)sizeof(O) / (64 << 10) + 1;
        r.blocks = a.accumulate || a.gaps ? 0 : (int)(some < 1024 ? some : 1024);
        return r;
    };
    const Rows all = share(0, 1, 1);
    if (a.num_ids == 0) {
        if (!a.accumulate) k_clear_table<O><<<dim3(all.blocks), 256, 0, st>>>(a, all);
        LKG_HIP(hipGetLastError());
        return LOGOSKG_OK;
    }
    if (a.num_ids <= 4096) {
        k_sort_few<O, 1, 4096><<<dim3((unsigned)(a.num_ids + 15) / 16 + all.blocks), 1024, 0, st>>>(a, all);
        LKG_HIP(hipGetLastError());
    } else if (a.num_ids <= kFewIds) {
        k_sort_few<O, 2, kFewIds><<<dim3((unsigned)(a.num_ids + 31) / 32 + all.blocks), 1024, 0, st>>>(a, all);
        LKG_HIP(hipGetLastError());
    } else {
        const int passes = (a.bits + kMostDigitBits - 1) / kMostDigitBits;
        for (int pass = 0, shift = 0; pass < passes; pass++) {
            const int bits = (a.bits - shift + passes - pass - 1) / (passes - pass);
            const Rows one = share(4 * pass, 4 * pass + 1, 4 * passes), two = share(4 * pass + 1, 4 * pass + 2, 4 * passes), rest = share(4 * pass + 2, 4 * pass + 4, 4 * passes);
            k_sort_count<O><<<dim3(a.tiles + one.blocks), 256, 4 << bits, st>>>(a, pass, shift, bits, one);
            LKG_HIP(hipGetLastError());
            k_sort_before<O><<<dim3(((1 << bits) + 15) / 16 + two.blocks), 512, 0, st>>>(a, 1 << bits, two);
            LKG_HIP(hipGetLastError());
            if (a.tile == 512) k_sort_move<O, 512><<<dim3(a.tiles + rest.blocks), 256, 16 << bits, st>>>(a, pass, shift, bits, rest);
            else k_sort_move<O, 2048><<<dim3(a.tiles + rest.blocks), 256, 16 << bits, st>>>(a, pass, shift, bits, rest);
            LKG_HIP(hipGetLastError());
            shift += bits;
        }
        if (passes & 1) a.key[0] = a.key[1], a.place[0] = a.place[1];
    }
    const long long lanes = (a.dim * (long long)sizeof(T) + 15) / 16;
    const int LG = lanes <= 4 ? 4 : lanes <= 16 ? 16 : 64;
    const dim3 grid((unsigned)((a.chunks + 256 / LG - 1) / (256 / LG)), (unsigned)((lanes + LG - 1) / LG));
    if (LG == 4) k_embed_sum<T, O, 4><<<grid, 256, 0, st>>>(a);
    else if (LG == 16) k_embed_sum<T, O, 16><<<grid, 256, 0, st>>>(a);
    else k_embed_sum<T, O, 64><<<grid, 256, 0, st>>>(a);
    LKG_HIP(hipGetLastError());
    if (a.chunks > 1) {
        k_embed_join<O><<<dim3((unsigned)((a.chunks + 15) / 16) + (a.gaps ? kGapBlocks : 0), (unsigned)((a.dim + 63) / 64)), 256, 0, st>>>(a);
        LKG_HIP(hipGetLastError());
    }
    return LOGOSKG_OK;
}

}  // namespace lkg

using namespace lkg;

extern "C" logoskg_status logoskg_embed_entities(const logoskg_embedding *e) {
    const char *why = nullptr;
    if (!e || e->struct_size != sizeof(logoskg_embedding)) why = "struct_size";
    else if (bad_type(e->dtype)) why = "unknown type";
    else if (!(e->scale - e->scale == 0.f)) why = "scale is not finite";
    else if (e->num_ids < 0 || e->num_ids >= (1ll << 40) || e->num_entities < 0 || e->dim < 0 || e->dim > (1ll << 24) || e->row < 0 || e->row > (1ll << 40)) why = "a count is out of range";
    else if (e->num_ids && e->dim && (!e->ids || !e->out)) why = "ids or out is NULL";
    else if (e->num_ids && e->dim && e->num_entities && !e->table) why = "table is NULL";
    else if (!aligned_to(e->table, e->dtype) || !aligned_to(e->out, e->dtype) || !aligned_to(e->ids, LOGOSKG_F32)) why = kUnaligned;
    if (why) { set_error("logoskg_embed_entities: %s", why); return LOGOSKG_EINVAL; }
    if (e->num_ids == 0 || e->dim == 0) return LOGOSKG_OK;
    const EmbedArgs a = {e->num_ids, e->num_entities, e->dim, e->row, e->scale, e->ids, e->table, e->out};
    OnDevice on;
    LKG_TRY(on.go(e->device));
    hipStream_t st = (hipStream_t)e->stream;
    if (e->dtype == LOGOSKG_F32) return launch_embed<float>(a, st);
    return e->dtype == LOGOSKG_BF16 ? launch_embed<bf16>(a, st) : launch_embed<fp16>(a, st);
}

extern "C" int64_t logoskg_embed_entities_backward_bytes(const logoskg_embedding_grad *e) {
    GradArgs a;
    if (const char *why = grad_args(e, &a)) { set_error("logoskg_embed_entities_backward_bytes: %s", why); return -1; }
    return a.num_ids && a.dim && a.num_entities ? plan_grad(a, size_of(e->table_dtype), nullptr) : 0;
}

extern "C" logoskg_status logoskg_embed_entities_backward(const logoskg_embedding_grad *e) {
    GradArgs a;
    if (const char *why = grad_args(e, &a)) { set_error("logoskg_embed_entities_backward: %s", why); return LOGOSKG_EINVAL; }
    if (a.dim == 0 || a.num_entities == 0) return LOGOSKG_OK;
    if (a.num_ids) {
        const long long need = plan_grad(a, size_of(e->table_dtype), (char *)e->workspace);
        if (e->workspace_bytes < need || !e->workspace) {
            set_error("logoskg_embed_entities_backward: the workspace has %lld of %lld bytes", (long long)e->workspace_bytes, need);
            return LOGOSKG_ERANGE;
        }
    }
    OnDevice on;
    LKG_TRY(on.go(e->device));
    hipStream_t st = (hipStream_t)e->stream;
    const bool wide = e->table_dtype == LOGOSKG_F32;
    if (e->dtype == LOGOSKG_F32) return launch_grad<float, float>(a, st);
    if (e->dtype == LOGOSKG_BF16) return wide ? launch_grad<bf16, float>(a, st) : launch_grad<bf16, bf16>(a, st);
    return wide ? launch_grad<fp16, float>(a, st) : launch_grad<fp16, fp16>(a, st);
}
