// Token embeddings: rows of a table looked up by token and scaled, and the table's gradient from sorted tokens.
//
//   out[i, :] = scale * table[ids[i], :]
//   dTable[t, :] = scale * sum of dOut[i, :] over the positions i with ids[i] = t
//
// The gradient adds rows that lie apart; a stable sort of the tokens puts the positions of a token side by side, so that every row
// of the gradient is formed by one owner in one fixed order: no floating-point atomics, bitwise reproducible.
//
// The lookup is bound by the bytes it stores (2.4 M rows of 100 fp32 columns from a bf16 table 262 us, 4.3 TB/s of what has to be moved; the rows lie 128
// apart, so that their last lines are written in part), the gradient by the bytes of dOut and dTable where those are many (65 536 rows of
// 2048 bf16 columns into 128 000: 61 us for the sums, 84 for their join and 105 000 rows of zeros) and by the launches of the sort
// where they are few (169 343 rows of 128 fp32 columns into 50 000: 37 of 70 us).
#include "common.h"
#include "values.h"

#include <cmath>

namespace slicegcn {

namespace {

constexpr int THREADS = 256;
constexpr int32_t MAX_WIDTH = INT32_MAX - 1023; // lanes count columns in 32 bits, up to 64 accesses of 8 past the end of a row

// ---- lookup ---------------------------------------------------------------------------------------------------------------

// A group of 2^log_lanes lanes moves ROWS rows at a time, V elements per lane and access; rows whose width is no multiple of V end with an access
// that is moved left and overlaps the one before it (the same values twice).
constexpr int LOOKUP_ROWS = 2; // 2.4 M rows of 100 columns, bf16 to fp32: 8 rows 296 us, 4 rows 291, 2 rows 263

template <class ID, class TT, class TR, int V, bool PAST>
__global__ __launch_bounds__(THREADS) void lookup_kernel(const ID *__restrict__ ids, int64_t n, int64_t vocab, int64_t pad, bool has_pad,
                                                         const TT *__restrict__ table, int64_t ldt, int32_t width, float scale,
                                                         TR *__restrict__ out, int64_t ldo, int log_lanes, int32_t tile)
{
    const int lane = threadIdx.x & ((1 << log_lanes) - 1), group = threadIdx.x >> log_lanes, groups = THREADS >> log_lanes;
    const int32_t last = width - V, c0 = blockIdx.y * tile, c1 = min(c0 + tile, width);
    for (int64_t r0 = (int64_t)blockIdx.x * groups * LOOKUP_ROWS + group; r0 < n; r0 += (int64_t)gridDim.x * groups * LOOKUP_ROWS) {
        int64_t id[LOOKUP_ROWS];
#pragma unroll
        for (int i = 0; i < LOOKUP_ROWS; ++i) {
            const int64_t r = r0 + i * groups;
            id[i] = r < n ? (int64_t)ids[r] : -1;
        }
        for (int32_t c = c0 + lane * V; c < c1; c += V << log_lanes) {
            const int32_t col = min(c, last);
            typename VecOf<TT, V>::type x[LOOKUP_ROWS];
#pragma unroll
            for (int i = 0; i < LOOKUP_ROWS; ++i) {
                const bool in = id[i] >= 0 && id[i] < vocab;
                x[i] = load_vec<TT, V>(table + (in ? id[i] : 0) * ldt + col);
            }
#pragma unroll
            for (int i = 0; i < LOOKUP_ROWS; ++i) {
                const int64_t r = r0 + i * groups;
                if (r >= n) break;
                const bool in = id[i] >= 0 && id[i] < vocab, zero = has_pad && id[i] == pad;
                float o[V];
#pragma unroll
                for (int j = 0; j < V; ++j) o[j] = zero ? 0.f : in ? scale * (float)x[i][j] : NAN;
                store_result<PAST, TR, V>(out + r * ldo + col, o);
            }
        }
    }
}

// ---- sort -----------------------------------------------------------------------------------------------------------------

// Stable sort by digits of at most DIGIT_BITS bits, lowest first.  Keys are tokens; padding and tokens outside the table get the key
// `vocab` and end up behind all others.
constexpr int DIGIT_BITS = 10, DIGITS = 1 << DIGIT_BITS;
constexpr int SORT_THREADS = 1024, SORT_WAVES = SORT_THREADS / 64, SORT_ITEMS = 4; // items of a thread, at most: fewer where that keeps more CUs busy
constexpr int SMALL_SORT = SORT_THREADS * SORT_ITEMS;

struct Tokens {
    const void *ids;
    int64_t n, vocab, pad;
    bool wide, has_pad;
};

__device__ inline uint32_t token_key(const Tokens &t, int64_t i)
{
    const int64_t id = t.wide ? static_cast<const int64_t *>(t.ids)[i] : (int64_t)static_cast<const int32_t *>(t.ids)[i];
    return id < 0 || id >= t.vocab || (t.has_pad && id == t.pad) ? (uint32_t)t.vocab : (uint32_t)id;
}

// Lanes of the wavefront that hold the same digit as this one, among the lanes in `active`
__device__ inline uint64_t same_digit(uint32_t digit, int bits, uint64_t active)
{
    uint64_t same = active;
#pragma unroll
    for (int b = 0; b < DIGIT_BITS; ++b) {
        if (b < bits) {
            const bool one = (digit >> b) & 1;
            const uint64_t ones = __ballot(one);
            same &= one ? ones : ~ones;
        }
    }
    return same;
}

// Orders this wavefront's accesses to LDS among its lanes
__device__ inline void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Exclusive prefix sum over the workgroup's threads
__device__ inline uint32_t block_scan(uint32_t v, uint32_t *wave_sums)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t sum = v;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const uint32_t up = (uint32_t)__shfl_up((int)sum, s, 64);
        if (lane >= s) sum += up;
    }
    if (lane == 63) wave_sums[wave] = sum;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave; ++w) before += wave_sums[w];
    __syncthreads(); // wave_sums may be written again
    return before + sum - v;
}

// Ranks the workgroup's items (a wavefront's items are ITEMS runs of 64 in a row) by digit, stable: rank[i] is the item's place among the
// wavefront's items of its digit.  counts[wave][digit] receives the wavefront's number of each digit.
template <int ITEMS>
__device__ inline void rank_items(const uint32_t (&key)[ITEMS], const bool (&there)[ITEMS], int shift, int bits,
                                  uint16_t (*counts)[DIGITS], uint32_t (&rank)[ITEMS])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t mask = (1u << bits) - 1;
    for (int d = threadIdx.x; d < SORT_WAVES << bits; d += SORT_THREADS) counts[d >> bits][d & mask] = 0;
    __syncthreads();
    uint16_t *mine = counts[wave]; // other lanes change it between two reads of this one: hence the fences
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t digit = (key[i] >> shift) & mask;
        const uint64_t same = same_digit(digit, bits, __ballot(there[i]));
        const uint32_t before = mine[digit];
        const int lower = __popcll(same & (((uint64_t)1 << lane) - 1));
        rank[i] = before + lower;
        wave_fence(); // every lane has read before one of them writes
        if (there[i] && lower == 0) mine[digit] = (uint16_t)(before + __popcll(same));
        wave_fence();
    }
    __syncthreads();
}

// counts[wave][digit] -> number of the digit in the wavefronts before; returns the total of the thread's digit
__device__ inline void counts_before(uint16_t (*counts)[DIGITS], int bits, uint32_t (&total)[DIGITS / SORT_THREADS])
{
#pragma unroll
    for (int q = 0; q < DIGITS / SORT_THREADS; ++q) {
        const int d = threadIdx.x * (DIGITS / SORT_THREADS) + q;
        uint32_t sum = 0;
        if (d < 1 << bits) {
            uint32_t c[SORT_WAVES];
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) c[w] = counts[w][d];
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) {
                counts[w][d] = (uint16_t)sum;
                sum += c[w];
            }
        }
        total[q] = sum;
    }
}

// first place in sorted keys that holds a key of at least t
__device__ inline uint32_t lower_bound(const uint32_t *keys, uint32_t count, uint32_t t)
{
    uint32_t lo = 0, len = count;
    while (len > 0) {
        const uint32_t half = len / 2;
        const bool right = keys[lo + half] < t;
        lo = right ? lo + half + 1 : lo;
        len = right ? len - half - 1 : half;
    }
    return lo;
}

// Up to SMALL_SORT tokens: every workgroup sorts all of them in LDS and writes its part of starts, the first one also the order: one launch
constexpr int STARTS_PER_BLOCK = 4 * SORT_THREADS;
template <int ITEMS>
__global__ __launch_bounds__(SORT_THREADS) void sort_small_kernel(const Tokens t, int bits, int passes, int32_t *__restrict__ order, int32_t *__restrict__ starts)
{
    __shared__ uint16_t counts[SORT_WAVES][DIGITS];
    __shared__ uint32_t base[DIGITS], wave_sums[SORT_WAVES];
    __shared__ uint32_t keys[SORT_THREADS * ITEMS];
    __shared__ uint16_t from[SORT_THREADS * ITEMS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = (int)t.n;
    const int first = wave * 64 * ITEMS + lane;
    uint32_t key[ITEMS], rank[ITEMS], index[ITEMS];
    bool there[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        index[i] = first + i * 64;
        there[i] = (int)index[i] < n;
        key[i] = there[i] ? token_key(t, index[i]) : 0;
    }
    for (int p = 0; p < passes; ++p) {
        rank_items(key, there, p * bits, bits, counts, rank);
        uint32_t total[DIGITS / SORT_THREADS];
        counts_before(counts, bits, total);
        uint32_t sum = 0;
#pragma unroll
        for (int q = 0; q < DIGITS / SORT_THREADS; ++q) sum += total[q];
        uint32_t at = block_scan(sum, wave_sums);
#pragma unroll
        for (int q = 0; q < DIGITS / SORT_THREADS; ++q) {
            base[threadIdx.x * (DIGITS / SORT_THREADS) + q] = at;
            at += total[q];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (there[i]) {
                const uint32_t digit = (key[i] >> (p * bits)) & ((1u << bits) - 1);
                const uint32_t place = base[digit] + counts[wave][digit] + rank[i];
                keys[place] = key[i];
                from[place] = (uint16_t)index[i];
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (there[i]) {
                key[i] = keys[first + i * 64];
                index[i] = from[first + i * 64];
            }
    }
    if (blockIdx.x == 0) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (there[i]) order[first + i * 64] = (int32_t)index[i];
    }
    const int64_t t0 = (int64_t)blockIdx.x * STARTS_PER_BLOCK;
    for (int64_t v = t0 + threadIdx.x; v < t0 + STARTS_PER_BLOCK && v <= t.vocab; v += SORT_THREADS)
        starts[v] = (int32_t)lower_bound(keys, (uint32_t)n, (uint32_t)v);
}

// More tokens: per digit, the tiles' histograms, their prefix sums, and the items to their places.
template <int ITEMS>
__global__ __launch_bounds__(SORT_THREADS) void digit_count_kernel(const Tokens t, const uint32_t *__restrict__ keys, int shift, int bits, uint32_t *__restrict__ hist)
{
    __shared__ uint32_t counts[DIGITS];
    const uint32_t mask = (1u << bits) - 1;
    for (int d = threadIdx.x; d < 1 << bits; d += SORT_THREADS) counts[d] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * (SORT_THREADS * ITEMS) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t at = first + i * SORT_THREADS;
        if (at < t.n) atomicAdd(&counts[((keys ? keys[at] : token_key(t, at)) >> shift) & mask], 1u);
    }
    __syncthreads();
    for (int d = threadIdx.x; d < 1 << bits; d += SORT_THREADS) hist[((int64_t)blockIdx.x << bits) + d] = counts[d];
}

// hist[tile][digit] -> number of the digit in the tiles before; total[digit].  A workgroup takes 64 digits, its wavefronts ranges of tiles.
__global__ __launch_bounds__(1024) void digit_scan_kernel(uint32_t *__restrict__ hist, int64_t tiles, int bits, uint32_t *__restrict__ total)
{
    __shared__ uint32_t sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, d = blockIdx.x * 64 + lane, digits = 1 << bits;
    const int64_t share = (tiles + 15) / 16, b = wave * share, e = min(b + share, tiles);
    uint32_t sum = 0;
    if (d < digits) {
#pragma unroll 8
        for (int64_t i = b; i < e; ++i) sum += hist[i * digits + d];
    }
    sums[wave][lane] = sum;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (int w = 0; w < 16; ++w) {
        if (w == wave) before = all;
        all += sums[w][lane];
    }
    if (d >= digits) return;
    if (wave == 0) total[d] = all;
#pragma unroll 8
    for (int64_t i = b; i < e; ++i) {
        const uint32_t c = hist[i * digits + d];
        hist[i * digits + d] = before;
        before += c;
    }
}

// Up to FEW_TILES tiles a workgroup adds up the tiles' histograms by itself: the scan's launch costs more (with the gradient, 83 tiles 62.8 us, scanned
// 65.3; 123 tiles 61.7 and 56.7).
constexpr int FEW_TILES = 96;
template <bool FEW, int ITEMS>
__global__ __launch_bounds__(SORT_THREADS) void digit_scatter_kernel(const Tokens t, const uint32_t *__restrict__ keys, const uint32_t *__restrict__ from,
                                                                     int shift, int bits, const uint32_t *__restrict__ hist,
                                                                     const uint32_t *__restrict__ total, int tiles, uint32_t *__restrict__ out_keys,
                                                                     uint32_t *__restrict__ out_from)
{
    __shared__ uint4 shared[SORT_WAVES * DIGITS / 8]; // the wavefronts' counts, then the items
    __shared__ uint32_t local[DIGITS], delta[DIGITS], wave_sums[SORT_WAVES];
    static_assert(sizeof(shared) >= sizeof(uint16_t[SORT_WAVES][DIGITS]) && sizeof(shared) >= sizeof(uint2[(SORT_THREADS * ITEMS)]), "room for either");
    auto *counts = reinterpret_cast<uint16_t(*)[DIGITS]>(shared);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.x * (SORT_THREADS * ITEMS) + wave * 64 * ITEMS + lane;
    uint32_t key[ITEMS], index[ITEMS], rank[ITEMS];
    bool there[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const int64_t at = first + i * 64;
        there[i] = at < t.n;
        key[i] = there[i] ? keys ? keys[at] : token_key(t, at) : 0;
        index[i] = there[i] && from ? from[at] : (uint32_t)at;
    }
    // a digit's items in the tiles before this one, and in all tiles: a thread per digit
    static_assert(DIGITS == SORT_THREADS, "a thread per digit");
    const int digits = 1 << bits, d = threadIdx.x;
    uint32_t before = 0, all = 0;
    if (d < digits) {
        if (FEW) {
#pragma unroll 16
            for (int i = 0; i < tiles; ++i) {
                const uint32_t c = hist[i * digits + d];
                before += i < (int)blockIdx.x ? c : 0;
                all += c;
            }
        } else {
            before = hist[(int64_t)blockIdx.x * digits + d];
            all = total[d];
        }
    }
    rank_items(key, there, shift, bits, counts, rank);
    uint32_t inside[1];
    counts_before(counts, bits, inside);
    const uint32_t here = block_scan(inside[0], wave_sums), everywhere = block_scan(all, wave_sums);
    local[d] = here;
    delta[d] = everywhere + before - here;
    __syncthreads();
    // The items in the order of their digits first: neighbouring lanes then store to neighbouring places.  Stored as they come, every item costs an
    // access of its own (2.4 M tokens, 10 bits: 42 us; so 23).
    const uint32_t mask = digits - 1;
    uint32_t place[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t digit = (key[i] >> shift) & mask;
        place[i] = local[digit] + counts[wave][digit] + rank[i];
    }
    __syncthreads(); // the items take the place of the counts
    uint2 *items = reinterpret_cast<uint2 *>(shared);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        if (there[i]) items[place[i]] = make_uint2(key[i], index[i]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t p = threadIdx.x + i * SORT_THREADS;
        if ((int64_t)blockIdx.x * (SORT_THREADS * ITEMS) + p >= t.n) break;
        const uint2 e = items[p];
        const uint32_t to = delta[(e.x >> shift) & mask] + p;
        out_keys[to] = e.x;
        out_from[to] = e.y;
    }
}

__global__ __launch_bounds__(THREADS) void starts_kernel(const uint32_t *__restrict__ keys, uint32_t n, int64_t vocab, int32_t *__restrict__ starts)
{
    for (int64_t t = (int64_t)blockIdx.x * THREADS + threadIdx.x; t <= vocab; t += (int64_t)gridDim.x * THREADS)
        starts[t] = (int32_t)lower_bound(keys, n, (uint32_t)t);
}

// ---- gradient -------------------------------------------------------------------------------------------------------------

// The order is cut into chunks of positions, whatever tokens they hold, so that work is even however tokens repeat.  A lane group adds up its
// chunk's rows token by token.  Tokens that lie within the chunk are finished there; the sums of a token that it shares with a neighbour go
// to the workspace as pieces, and a second launch adds those: row 2 * chunk holds the piece of a token that started before the chunk,
// row 2 * chunk + 1 that of one that starts in it and goes on behind it.  That launch also zeroes the rows of
// tokens without positions.
constexpr int CHUNK = 64; // positions, at most
constexpr int AHEAD = 4;  // rows that are requested at a time, a batch ahead

struct GradArgs {
    const int32_t *order, *starts;
    int64_t n, vocab, ldo, ldt;
    int32_t width;
    float scale;
    bool accumulate;
    int log_lanes;    // lanes of a group; a group's lanes hold V columns each
    int log_chunk;
    uint32_t tiles;   // tiles of a row: workgroups beside each other hold the same rows
    int64_t chunks;
    float *pieces;    // [2 * chunks][width]
    int32_t *tails;   // [chunks] the token that starts in the chunk and goes on behind it, or -1
};

// The V columns of a lane.  The last ones of a row that is no multiple of V wide are moved left; the first `skip` of them belong to the lane before.
struct Columns {
    int32_t at, skip;
    bool on; // false: past the end (`at` is valid all the same)
};

template <int V> __device__ inline Columns lane_columns(const GradArgs &a, int32_t tile)
{
    const int lane = threadIdx.x & ((1 << a.log_lanes) - 1);
    const int32_t c = (tile << a.log_lanes) * V + lane * V, at = min(c, a.width - V);
    return Columns{at, c - at, c < a.width};
}

// Each element has one owner (with ACCUMULATE a second one would add twice)
template <bool PAST, class TT, int V> __device__ inline void store_sum(const GradArgs &a, TT *__restrict__ dTable, int64_t t, const Columns &c, float (&sum)[V])
{
    if (!c.on) return;
    TT *p = dTable + t * a.ldt + c.at;
    if (a.accumulate) {
        const auto old = load_vec<TT, V>(p);
#pragma unroll
        for (int j = 0; j < V; ++j) sum[j] += (float)old[j];
    }
    if (c.skip == 0) {
        store_result<PAST, TT, V>(p, sum);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j >= c.skip) p[j] = (TT)sum[j];
    }
}

__device__ inline int32_t place(const GradArgs &a, int64_t t) // starts[t] within the order
{
    const int32_t s = a.starts[t];
    return s < 0 ? 0 : s > a.n ? (int32_t)a.n : s;
}

// The tokens that hold places p and q (below starts[vocab]): the last t with starts[t] <= p.  The lanes of a group look for them together.
__device__ inline void tokens_at(const GradArgs &a, int32_t p, int32_t q, uint32_t *tp, uint32_t *tq)
{
    const int lanes = 1 << a.log_lanes, lane = threadIdx.x & (lanes - 1), shift = (threadIdx.x & 63) - lane;
    const uint64_t mask = lanes == 64 ? ~(uint64_t)0 : ((uint64_t)1 << lanes) - 1;
    uint32_t lo[2] = {0, 0}, hi[2] = {(uint32_t)a.vocab, (uint32_t)a.vocab}; // starts[lo] <= place < starts[hi]
    while (hi[0] - lo[0] > 1 || hi[1] - lo[1] > 1) {
        uint32_t step[2];
        bool below[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            step[i] = (hi[i] - lo[i] + lanes - 1) >> a.log_lanes;
            const uint32_t at = lo[i] + (lane + 1) * step[i];
            below[i] = at < hi[i] && a.starts[at < hi[i] ? at : lo[i]] <= (i ? q : p);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            lo[i] += (uint32_t)__popcll(__ballot(below[i]) >> shift & mask) * step[i];
            hi[i] = min(hi[i], lo[i] + step[i]);
        }
    }
    *tp = lo[0];
    *tq = lo[1];
}

// Rows of tokens without positions.  A wavefront looks at so many of them (wide rows are long work).
__host__ __device__ inline int zero_tokens(int log_lanes) { return log_lanes == 6 ? 16 : 64; }
template <bool PAST, class TT, int V> __device__ inline void zero_rows(const GradArgs &a, TT *__restrict__ dTable, int64_t block)
{
    const int tokens = zero_tokens(a.log_lanes), lane = threadIdx.x & 63, sub = lane >> a.log_lanes, subs = 64 >> a.log_lanes;
    const int64_t t0 = (block * (THREADS / 64) + threadIdx.x / 64) * tokens, t = t0 + lane;
    const uint64_t empty = __ballot(lane < tokens && t < a.vocab && a.starts[t < a.vocab ? t + 1 : 0] <= a.starts[t < a.vocab ? t : 0]);
    const float zero[V] = {};
    for (int i = sub; i < tokens; i += subs) {
        if (!(empty >> i & 1)) continue;
        TT *row = dTable + (t0 + i) * a.ldt;
        for (int32_t c = (lane & ((1 << a.log_lanes) - 1)) * V; c < a.width; c += V << a.log_lanes)
            store_result<PAST, TT, V>(row + min(c, a.width - V), zero);
    }
}

template <class TR, class TT, int V, bool PAST>
__global__ __launch_bounds__(THREADS) void embed_grad_kernel(const GradArgs a, const TR *__restrict__ dOut, TT *__restrict__ dTable, uint32_t first_block)
{
    __shared__ int2 list[THREADS / 8][CHUNK + 2 * AHEAD]; // token and row of every position of a group's chunk
    const int lanes = 1 << a.log_lanes, lane = threadIdx.x & (lanes - 1), group = threadIdx.x >> a.log_lanes, len = 1 << a.log_chunk;
    const uint32_t block = first_block + blockIdx.x, tile = block % a.tiles;
    const Columns col = lane_columns<V>(a, tile);
    const int64_t chunk = ((int64_t)(block / a.tiles) * THREADS >> a.log_lanes) + group;
    const int32_t valid = place(a, a.vocab);
    if (chunk >= a.chunks) return;
    const int64_t p0l = chunk << a.log_chunk;
    if (p0l >= valid) {
        if (lane == 0 && tile == 0 && a.chunks > 1) a.tails[chunk] = -1;
        return;
    }
    const int32_t p0 = (int32_t)p0l, count = min(valid - p0, len);
    uint32_t head, tail;
    tokens_at(a, p0, p0 + count - 1, &head, &tail);
    for (int i = lane; i < len + 2 * AHEAD; i += lanes) {
        int2 e = make_int2(-1, -1);
        if (i < count) {
            e.y = a.order[p0 + i];
            if (e.y >= a.n) e.y = -1;
            uint32_t lo = head, hi = max(head, tail) + 1;
            while (hi - lo > 1) {
                const uint32_t mid = lo + (hi - lo) / 2;
                const bool right = a.starts[mid] <= p0 + i;
                lo = right ? mid : lo;
                hi = right ? hi : mid;
            }
            e.x = (int32_t)lo;
        }
        list[group][i] = e;
    }
    // one chunk holds whatever there is, and has no workspace for pieces: only starts that do not ascend could say that its last token goes on
    const bool starts_before = place(a, head) < p0, goes_on = a.chunks > 1 && (int64_t)place(a, (int64_t)tail + 1) > (int64_t)p0 + count;
    wave_fence();
    int32_t now = (int32_t)head;
    bool first = starts_before; // the token `now` started before the chunk
    float acc[V] = {};
    typename VecOf<TR, V>::type x[AHEAD];
    int2 e[AHEAD];
    auto request = [&](int b) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) e[i] = list[group][b + i];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (e[i].y >= 0) {
                x[i] = load_vec<TR, V>(dOut + e[i].y * a.ldo + col.at);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) x[i][j] = (TR)0.f;
            }
        }
    };
    request(0);
    for (int b = 0; b < count; b += AHEAD) {
        // Sums of tokens that end in this batch are set aside and stored once all of its rows are used and the next ones are requested: a store
        // between uses of loads would have every later use wait for the store (loads and stores are counted together).
        float done[AHEAD][V];
        int32_t token[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const bool same = e[i].x == now || e[i].x < 0;
            token[i] = same ? -1 : now;
            now = same ? now : e[i].x;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                done[i][j] = acc[j];
                acc[j] = (same ? acc[j] : 0.f) + (float)x[i][j];
            }
        }
        if (b + AHEAD < count) request(b + AHEAD);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (token[i] < 0) continue;
            if (first) {
                if (col.on) store_vec<float, V>(a.pieces + 2 * chunk * a.width + col.at, done[i]);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) done[i][j] *= a.scale;
                store_sum<PAST, TT, V>(a, dTable, token[i], col, done[i]);
            }
            first = false;
        }
    }
    if (first || goes_on) {
        if (col.on) store_vec<float, V>(a.pieces + (2 * chunk + (first ? 0 : 1)) * a.width + col.at, acc);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] *= a.scale;
        store_sum<PAST, TT, V>(a, dTable, now, col, acc);
    }
    if (lane == 0 && tile == 0 && a.chunks > 1) a.tails[chunk] = goes_on && !first ? now : -1;
}

// Tokens that several chunks share: the pieces are added where the token starts.  A wavefront takes a chunk; what has many pieces is
// added by the whole workgroup.  One workgroup adds all pieces of a token, for its tile of columns: 2 M rows of 64 fp32 columns into 30 tokens, the
// most frequent of which holds a fifth, 104 us for the sums and 32 for their join.
constexpr int JOIN_CHUNKS = THREADS / 64, JOIN_MANY = 64;
template <class TT, int V, bool PAST>
__global__ __launch_bounds__(THREADS) void embed_join_kernel(const GradArgs a, TT *__restrict__ dTable, uint32_t first_block, uint32_t join_blocks)
{
    __shared__ double sums[THREADS / 64][64][V];
    const int wave = threadIdx.x / 64, sub = (threadIdx.x & 63) >> a.log_lanes, subs = 64 >> a.log_lanes, lanes = 1 << a.log_lanes;
    const uint32_t block = first_block + blockIdx.x;
    if (block >= join_blocks) {
        zero_rows<PAST, TT, V>(a, dTable, block - join_blocks);
        return;
    }
    const int64_t chunk0 = (int64_t)(block / a.tiles) * JOIN_CHUNKS;
    const Columns col = lane_columns<V>(a, block % a.tiles);
    // the sum over every step-th piece of the token that starts in chunk c, from the first-th on; then over the lanes of a wavefront
    auto add = [&](int64_t c, int64_t last, int64_t first, int64_t step, double (&acc)[V]) {
#pragma unroll
        for (int j = 0; j < V; ++j) acc[j] = 0.0;
#pragma unroll 8
        for (int64_t k = c + first; k <= last; k += step) {
            const auto x = load_vec<float, V>(a.pieces + (2 * k + (k == c)) * a.width + col.at);
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += (double)x[j];
        }
        for (int s = lanes; s < 64; s <<= 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] += __shfl_xor(acc[j], s, 64);
        }
    };
    auto store = [&](int64_t t, const double (&acc)[V]) {
        float out[V];
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = (float)((double)a.scale * acc[j]);
        store_sum<PAST, TT, V>(a, dTable, t, col, out);
    };
    auto token = [&](int64_t c) { return c < a.chunks ? a.tails[c] : -1; };
    auto last_chunk = [&](int32_t t) { return (int64_t)(place(a, (int64_t)t + 1) - 1) >> a.log_chunk; };
    int32_t t[JOIN_CHUNKS];
    int64_t last[JOIN_CHUNKS];
#pragma unroll
    for (int w = 0; w < JOIN_CHUNKS; ++w) t[w] = token(chunk0 + w);
#pragma unroll
    for (int w = 0; w < JOIN_CHUNKS; ++w) last[w] = t[w] >= 0 ? last_chunk(t[w]) : -1;
#pragma unroll
    for (int w = 0; w < JOIN_CHUNKS; ++w) {
        const int64_t c = chunk0 + w, pieces = last[w] - c + 1;
        if (t[w] < 0) continue;
        double acc[V];
        if (pieces <= JOIN_MANY) {
            if (wave != w) continue;
            add(c, last[w], sub, subs, acc);
            if (sub == 0) store(t[w], acc);
        } else { // the same for the whole workgroup
            add(c, last[w], wave * subs + sub, JOIN_CHUNKS * subs, acc);
            __syncthreads();
#pragma unroll
            for (int j = 0; j < V; ++j) sums[wave][threadIdx.x & 63][j] = acc[j];
            __syncthreads();
            if (wave == 0 && sub == 0) {
#pragma unroll
                for (int j = 0; j < V; ++j) acc[j] = ((sums[0][threadIdx.x][j] + sums[1][threadIdx.x][j]) + sums[2][threadIdx.x][j]) + sums[3][threadIdx.x][j];
                store(t[w], acc);
            }
        }
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------------

// A pair of types that differ has fp32 on one side
template <class F> auto with_types(int32_t table, int32_t rows, F f)
{
    return with_type(table, [&](auto t) {
        return with_type(rows, [&](auto r) {
            using TT = decltype(t);
            using TR = decltype(r);
            if constexpr (std::is_same_v<TT, TR> || std::is_same_v<TT, float> || std::is_same_v<TR, float>) return f(t, r);
            else return (int)SLICEGCN_EINVAL; // refused before
        });
    });
}

int check_desc(const char *what, const slicegcn_embed_desc *d, bool rows)
{
    SG_REQUIRE(d != nullptr, SLICEGCN_EINVAL, "%s: NULL descriptor", what);
    SG_REQUIRE(d->n >= 0 && d->vocab >= 1, SLICEGCN_EINVAL, "%s: need n >= 0 and vocab >= 1", what);
    SG_REQUIRE(d->n <= INT32_MAX && d->vocab < INT32_MAX, SLICEGCN_ERANGE, "%s: n = %lld or vocab = %lld too large", what, (long long)d->n, (long long)d->vocab);
    SG_REQUIRE((d->flags & ~(SLICEGCN_EMBED_IDS64 | SLICEGCN_EMBED_PAD | SLICEGCN_EMBED_ACCUMULATE)) == 0, SLICEGCN_EINVAL, "%s: unknown flag", what);
    if (!rows) return SLICEGCN_OK;
    SG_REQUIRE(d->width >= 1, SLICEGCN_EINVAL, "%s: width < 1", what);
    SG_REQUIRE(d->width <= MAX_WIDTH, SLICEGCN_ERANGE, "%s: width = %d too large", what, d->width);
    SG_REQUIRE(known_type(d->table_type) && known_type(d->row_type), SLICEGCN_EINVAL, "%s: unknown type", what);
    SG_REQUIRE(d->table_type == d->row_type || d->table_type == SLICEGCN_F32 || d->row_type == SLICEGCN_F32, SLICEGCN_EINVAL,
               "%s: a table and rows in two different 16-bit types", what);
    SG_REQUIRE(std::isfinite((float)d->scale), SLICEGCN_EINVAL, "%s: scale is not finite", what);
    return SLICEGCN_OK;
}

int check_ids(const char *what, const slicegcn_embed_desc *d, const void *ids)
{
    SG_REQUIRE(ids || d->n == 0, SLICEGCN_EINVAL, "%s: NULL ids", what);
    SG_REQUIRE((reinterpret_cast<uintptr_t>(ids) & (d->flags & SLICEGCN_EMBED_IDS64 ? 7u : 3u)) == 0, SLICEGCN_EINVAL, "%s: misaligned ids", what);
    return SLICEGCN_OK;
}

// log2 of the lanes that hold a row's accesses, 8 to 64
int log_lanes_for(int32_t accesses)
{
    int l = 3;
    while (l < 6 && (1 << l) < accesses) ++l;
    return l;
}

// How the gradient is cut: accesses of a row over lanes (and tiles of lanes), positions over chunks.
struct GradPlan {
    int log_lanes, log_chunk;
    int64_t chunks;
    int32_t tiles;
    GradPlan(int64_t n, int32_t width, int v)
    {
        const int32_t accesses = (width + v - 1) / v;
        log_lanes = log_lanes_for(accesses);
        tiles = (accesses + (1 << log_lanes) - 1) >> log_lanes;
        // as many wavefronts as keep the chip busy before chunks get longer: a longer chunk leaves fewer pieces
        log_chunk = 3;
        while ((1 << log_chunk) < CHUNK && (n * tiles << log_lanes >> (log_chunk + 1)) >= 64 * 2048) ++log_chunk;
        chunks = (n + (1 << log_chunk) - 1) >> log_chunk;
    }
    size_t piece_bytes(int32_t width) const { return (size_t)round_up(2 * chunks * (int64_t)width * 4, 256); }
    size_t bytes(int32_t width) const { return chunks <= 1 ? 0 : piece_bytes(width) + (size_t)round_up(4 * chunks, 256); }
};

int grad_access(int32_t width, int32_t row_type)
{
    const int v = 16 / type_bytes(row_type);
    return width < v ? 1 : v;
}

// Calls f with the number of items of a thread
template <class F> auto with_items(int items, F f)
{
    return items == 1 ? f(std::integral_constant<int, 1>()) : items == 2 ? f(std::integral_constant<int, 2>()) : f(std::integral_constant<int, SORT_ITEMS>());
}

// Tokens up to which a thread of the sort takes one, two of them (else SORT_ITEMS): sort and gradient of 16 columns, 16 000 tokens with one, two, four
// 32.9, 38.0, 39.5 us, 120 000 with two, four 48.6, 53.7, 500 000 65.8, 69.0, 1 M 126.6, 118.4.
constexpr int64_t FEW_ITEMS[2] = {65536, 524288};
struct SortPlan {
    int bits, passes; // per digit
    int items;        // per thread
    int64_t tiles;
    SortPlan(int64_t n, int64_t vocab)
    {
        int all = 1;
        while ((vocab >> all) != 0) ++all; // keys 0 to vocab
        passes = (all + DIGIT_BITS - 1) / DIGIT_BITS;
        bits = (all + passes - 1) / passes;
        items = n <= FEW_ITEMS[0] ? 1 : n <= FEW_ITEMS[1] ? 2 : SORT_ITEMS;
        tiles = (n + SORT_THREADS * items - 1) / (SORT_THREADS * items);
    }
    int64_t hist_words() const { return round_up(tiles << bits, 64); }
};

} // namespace
} // namespace slicegcn

using namespace slicegcn;

extern "C" int slicegcn_embed_fwd(const slicegcn_embed_desc *d, const void *ids, const void *table, int64_t ldt, void *out, int64_t ldo,
                                  void *stream)
{
    if (int rc = check_desc("embed_fwd", d, true)) return rc;
    if (int rc = check_ids("embed_fwd", d, ids)) return rc;
    SG_REQUIRE(table && (out || d->n == 0), SLICEGCN_EINVAL, "embed_fwd: NULL pointer");
    SG_REQUIRE(ldt >= d->width && ldo >= d->width, SLICEGCN_EINVAL, "embed_fwd: leading dimension smaller than the width");
    SG_REQUIRE(aligned_for(table, d->table_type) && aligned_for(out, d->row_type), SLICEGCN_EINVAL, "embed_fwd: misaligned base");
    if (d->n == 0) return SLICEGCN_OK;
    ProfScope prof(SLICEGCN_PROF_EMBED, d->width, as_stream(stream));
    const bool has_pad = d->flags & SLICEGCN_EMBED_PAD;
    return with_types(d->table_type, d->row_type, [&](auto t, auto r) {
        using TT = decltype(t);
        using TR = decltype(r);
        auto launch = [&](auto access) {
            constexpr int V = decltype(access)::value;
            const int32_t accesses = (d->width + V - 1) / V;
            const int log_lanes = log_lanes_for(accesses), groups = THREADS >> log_lanes;
            const int64_t blocks = (d->n + groups * LOOKUP_ROWS - 1) / (groups * LOOKUP_ROWS);
            const int32_t tile = (V << log_lanes) * 4;
            const int64_t tiles = ((int64_t)d->width + tile - 1) / tile;
            SG_REQUIRE(tiles < 65536, SLICEGCN_ERANGE, "embed_fwd: width = %d too large", d->width);
            const dim3 grid((unsigned)(blocks < 65536 ? blocks : 65536), (unsigned)tiles);
            with_flag(past_cache(d->n, ldo, d->row_type), [&](auto past) {
                with_flag(d->flags & SLICEGCN_EMBED_IDS64, [&](auto wide) {
                    using ID = std::conditional_t<decltype(wide)::value, int64_t, int32_t>;
                    lookup_kernel<ID, TT, TR, V, decltype(past)::value><<<grid, THREADS, 0, as_stream(stream)>>>(
                        static_cast<const ID *>(ids), d->n, d->vocab, d->pad, has_pad, static_cast<const TT *>(table), ldt, d->width,
                        (float)d->scale, static_cast<TR *>(out), ldo, log_lanes, tile);
                });
            });
            SG_LAUNCH_CHECK();
            return (int)SLICEGCN_OK;
        };
        constexpr int V = 16 / (int)sizeof(TR);
        if (d->width >= V) return launch(std::integral_constant<int, V>());
        return launch(std::integral_constant<int, 1>());
    });
}

extern "C" size_t slicegcn_embed_sort_workspace_bytes(int64_t n, int64_t vocab)
{
    if (n < 0 || vocab < 1 || n > INT32_MAX || vocab >= INT32_MAX || n <= SMALL_SORT) return 0;
    const SortPlan plan(n, vocab);
    return (size_t)round_up(4 * (plan.hist_words() + DIGITS + 4 * round_up(n, 64)), 256);
}

extern "C" int slicegcn_embed_sort(const slicegcn_embed_desc *d, const void *ids, int32_t *order, int32_t *starts, void *ws, size_t ws_bytes,
                                   void *stream)
{
    if (int rc = check_desc("embed_sort", d, false)) return rc;
    if (int rc = check_ids("embed_sort", d, ids)) return rc;
    SG_REQUIRE((order || d->n == 0) && starts, SLICEGCN_EINVAL, "embed_sort: NULL pointer");
    SG_REQUIRE((reinterpret_cast<uintptr_t>(order) & 3u) == 0 && (reinterpret_cast<uintptr_t>(starts) & 3u) == 0 &&
                   (reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SLICEGCN_EINVAL, "embed_sort: misaligned array or workspace");
    const size_t need = slicegcn_embed_sort_workspace_bytes(d->n, d->vocab);
    SG_REQUIRE(need == 0 || (ws && ws_bytes >= need), SLICEGCN_EWORKSPACE, "embed_sort: workspace of %zu bytes, %zu needed", ws_bytes, need);
    ProfScope prof(SLICEGCN_PROF_EMBED, 0, as_stream(stream));
    const Tokens t{ids, d->n, d->vocab, d->pad, (d->flags & SLICEGCN_EMBED_IDS64) != 0, (d->flags & SLICEGCN_EMBED_PAD) != 0};
    const SortPlan plan(d->n, d->vocab);
    hipStream_t s = as_stream(stream);
    if (d->n <= SMALL_SORT)
        return launch_parts((d->vocab + STARTS_PER_BLOCK) / STARTS_PER_BLOCK, [&](unsigned, unsigned count) { // below 2^19 workgroups: one part
            with_items(d->n <= SORT_THREADS ? 1 : d->n <= 2 * SORT_THREADS ? 2 : SORT_ITEMS, [&](auto items) {
                sort_small_kernel<decltype(items)::value><<<count, SORT_THREADS, 0, s>>>(t, plan.bits, plan.passes, order, starts);
            });
        });
    uint32_t *hist = static_cast<uint32_t *>(ws), *total = hist + plan.hist_words(), *buf = total + DIGITS;
    const int64_t stride = round_up(d->n, 64);
    uint32_t *keys[2] = {buf, buf + stride}, *from[2] = {buf + 2 * stride, buf + 3 * stride};
    const uint32_t *in_keys = nullptr, *in_from = nullptr;
    for (int p = 0; p < plan.passes; ++p) {
        uint32_t *out_keys = keys[p & 1], *out_from = p == plan.passes - 1 ? reinterpret_cast<uint32_t *>(order) : from[p & 1];
        const int shift = p * plan.bits;
        if (int rc = with_items(plan.items, [&](auto items) {
                constexpr int ITEMS = decltype(items)::value;
                digit_count_kernel<ITEMS><<<(unsigned)plan.tiles, SORT_THREADS, 0, s>>>(t, in_keys, shift, plan.bits, hist);
                SG_LAUNCH_CHECK();
                // one item a thread only ever means few tiles, SORT_ITEMS never
                static_assert(FEW_ITEMS[0] <= (int64_t)FEW_TILES * SORT_THREADS && FEW_ITEMS[1] >= (int64_t)FEW_TILES * SORT_THREADS * SORT_ITEMS, "tiles");
                if constexpr (ITEMS < SORT_ITEMS) {
                    if (plan.tiles <= FEW_TILES) {
                        digit_scatter_kernel<true, ITEMS><<<(unsigned)plan.tiles, SORT_THREADS, 0, s>>>(t, in_keys, in_from, shift, plan.bits, hist, nullptr,
                                                                                                       (int)plan.tiles, out_keys, out_from);
                        SG_LAUNCH_CHECK();
                        return (int)SLICEGCN_OK;
                    }
                }
                if constexpr (ITEMS > 1) {
                    digit_scan_kernel<<<(unsigned)(((1 << plan.bits) + 63) / 64), 1024, 0, s>>>(hist, plan.tiles, plan.bits, total);
                    SG_LAUNCH_CHECK();
                    digit_scatter_kernel<false, ITEMS><<<(unsigned)plan.tiles, SORT_THREADS, 0, s>>>(t, in_keys, in_from, shift, plan.bits, hist, total, 0,
                                                                                                    out_keys, out_from);
                    SG_LAUNCH_CHECK();
                }
                return (int)SLICEGCN_OK;
            }))
            return rc;
        in_keys = out_keys;
        in_from = out_from;
    }
    const int64_t blocks = (d->vocab + 1 + THREADS - 1) / THREADS;
    starts_kernel<<<(unsigned)(blocks < 65536 ? blocks : 65536), THREADS, 0, s>>>(in_keys, (uint32_t)d->n, d->vocab, starts);
    SG_LAUNCH_CHECK();
    return SLICEGCN_OK;
}

extern "C" size_t slicegcn_embed_bwd_workspace_bytes(int64_t n, int32_t width)
{
    if (n < 1 || n > INT32_MAX || width < 1 || width > MAX_WIDTH) return 0;
    const size_t a = GradPlan(n, width, grad_access(width, SLICEGCN_F32)).bytes(width), b = GradPlan(n, width, grad_access(width, SLICEGCN_BF16)).bytes(width);
    return a > b ? a : b;
}

extern "C" int slicegcn_embed_bwd(const slicegcn_embed_desc *d, const int32_t *order, const int32_t *starts, const void *dOut, int64_t ldo,
                                  void *dTable, int64_t ldt, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = check_desc("embed_bwd", d, true)) return rc;
    SG_REQUIRE(starts && dTable && ((order && dOut) || d->n == 0), SLICEGCN_EINVAL, "embed_bwd: NULL pointer");
    SG_REQUIRE(ldt >= d->width && ldo >= d->width, SLICEGCN_EINVAL, "embed_bwd: leading dimension smaller than the width");
    SG_REQUIRE(aligned_for(dTable, d->table_type) && aligned_for(dOut, d->row_type) && (reinterpret_cast<uintptr_t>(order) & 3u) == 0 &&
                   (reinterpret_cast<uintptr_t>(starts) & 3u) == 0 && (reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SLICEGCN_EINVAL,
               "embed_bwd: misaligned array or workspace");
    const size_t need = slicegcn_embed_bwd_workspace_bytes(d->n, d->width);
    SG_REQUIRE(need == 0 || (ws && ws_bytes >= need), SLICEGCN_EWORKSPACE, "embed_bwd: workspace of %zu bytes, %zu needed", ws_bytes, need);
    ProfScope prof(SLICEGCN_PROF_EMBED, d->width, as_stream(stream));
    return with_types(d->table_type, d->row_type, [&](auto t, auto r) {
        using TT = decltype(t);
        using TR = decltype(r);
        auto launch = [&](auto access) {
            constexpr int V = decltype(access)::value;
            const GradPlan plan(d->n, d->width, V);
            GradArgs a{order, starts, d->n, d->vocab, ldo, ldt, d->width, (float)d->scale, (d->flags & SLICEGCN_EMBED_ACCUMULATE) != 0,
                       plan.log_lanes, plan.log_chunk, (uint32_t)plan.tiles, plan.chunks, static_cast<float *>(ws),
                       reinterpret_cast<int32_t *>(static_cast<char *>(ws) + plan.piece_bytes(d->width))};
            const int64_t groups = THREADS >> a.log_lanes;
            const int64_t chunk_blocks = (a.chunks + groups - 1) / groups * plan.tiles, per_block = (int64_t)zero_tokens(a.log_lanes) * (THREADS / 64);
            const int64_t join_blocks = a.chunks > 1 ? (a.chunks + JOIN_CHUNKS - 1) / JOIN_CHUNKS * plan.tiles : 0;
            const int64_t zero_blocks = a.accumulate ? 0 : (d->vocab + per_block - 1) / per_block;
            SG_REQUIRE(chunk_blocks < ((int64_t)1 << 31) && join_blocks + zero_blocks < ((int64_t)1 << 31), SLICEGCN_ERANGE,
                       "embed_bwd: %lld rows of %d columns are too many for a call", (long long)d->n, d->width);
            // Past the caches only whole lines, or parts of a line reach the memory one by one: a gradient of 500 000 rows of 300 fp32 columns 213 us,
            // through the caches 180; 128 000 rows of 2048 bf16 columns 183 and 219
            const int64_t row_bytes = (int64_t)d->width * type_bytes(d->table_type);
            const bool whole_lines = row_bytes % 128 == 0 && ldt * type_bytes(d->table_type) % 128 == 0 && (reinterpret_cast<uintptr_t>(dTable) & 127u) == 0;
            auto go = [&](auto past) {
                constexpr bool PAST = decltype(past)::value;
                if (int rc = launch_parts(chunk_blocks, [&](unsigned first, unsigned count) {
                        embed_grad_kernel<TR, TT, V, PAST><<<count, THREADS, 0, as_stream(stream)>>>(a, static_cast<const TR *>(dOut), static_cast<TT *>(dTable), first);
                    }))
                    return rc;
                return launch_parts(join_blocks + zero_blocks, [&](unsigned first, unsigned count) {
                    embed_join_kernel<TT, V, PAST><<<count, THREADS, 0, as_stream(stream)>>>(a, static_cast<TT *>(dTable), first, (uint32_t)join_blocks);
                });
            };
            if constexpr (V > 1)
                if (whole_lines && past_cache(d->vocab, ldt, d->table_type)) return go(std::true_type());
            return go(std::false_type());
        };
        constexpr int V = 16 / (int)sizeof(TR);
        if (d->width >= V) return launch(std::integral_constant<int, V>());
        return launch(std::integral_constant<int, 1>());
    });
}
