// Products of 16-bit operands that lie on 16-byte boundaries, in tiles of 256 x 256.
//
// A workgroup of eight wavefronts, two of them a SIMD, each with 128 x 64 of the results.  Steps of 32 k go from memory straight into LDS (buffer loads with
// the lds bit: no registers, and what lies outside of the operand arrives as zeros), DEPTH - 1 steps ahead in DEPTH buffers.  A load writes 64 units of 16 bytes
// in the order of its lanes, so the order in LDS that lds_unit wants is made by the addresses that the lanes read from.  At the top of a
// step a wavefront waits for its own loads of the step after this one and meets the others at a barrier: then that step is whole in LDS, and nobody reads the
// buffer any more that the next loads are for.  During a step the operand registers for the next one are read: those of the N side into a second set, those of the M
// side into the registers that the step is done with.
// 8192 rows 4096 -> 10240 gated bf16: 1.05 ms, 1.31 PFLOP/s (a library's plain products of these sizes: 0.90 to 1.35); bound by the matrix instructions, which run 60 to 70 % of
// the time at the clock that their power leaves.  With four wavefronts of 128 x 128 each, with five buffers or with 32 x 32 x 16
// instructions (1.81 PFLOP/s by themselves, these 2.05) slower.
// The waits are counted by hand, since the compiler does not know which reads of LDS a load in flight has to do with; the loads are therefore inline assembly,
// which has no register results.
#pragma once

#include "product_kernels.h"

namespace slicegcn {
namespace {

typedef int int4v __attribute__((ext_vector_type(4)));

constexpr int DIRECT_THREADS = 512, DIRECT_DEPTH = 4;

// 64 x 16 bytes from the buffer at rsrc, each lane's at its offset and the scalar one, to LDS at `lds` and behind it.  (m0, which holds that address, cannot be named as overwritten; the
// compiler sets it itself right before instructions that use it, of which these kernels have no others.  Nor does it look into the block for hazards: m0 is to be written one
// wait state ahead of the load, and a scalar register that a vector instruction wrote five.)
__device__ inline void load_to_lds(int4v rsrc, uint32_t offset, uint32_t scalar, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(rsrc), "s"(scalar) : "memory");
}

template <int COUNT> __device__ inline void wait_loads_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(COUNT) : "memory");
}

// How a lane's loads of a step reach an operand's piece of R outer indexes.  KC: a buffer from the tile's first row on, of which a step reads 32 k from its
// scalar offset on.  OC: a buffer of the step's own lines.  All of a step's arithmetic is scalar, in 32 bits and without branches, so that the compiler can
// put it between the matrix instructions of the step before.
// THREADS: those that share the loads out: the workgroup's, or a wavefront's
template <int LAYOUT, int R, int THREADS> struct DirectPiece {
    static constexpr int UNITS = R * DIRECT_K / 8, LOADS = UNITS / THREADS;
    static_assert(UNITS % THREADS == 0, "units are dealt evenly");
    static constexpr uint32_t NOWHERE = 0xffffff00u; // beyond any buffer, with all words of an access
    uint32_t offset[LOADS];
    uint64_t base;
    uint32_t line, size, scalar; // bytes: of a line; KC: of the buffer, OC: of a line's part; KC: the step's offset
    int4v rsrc;

    __device__ static int unit(int i) { return (int)threadIdx.x % THREADS + i * THREADS; }
    // k of a load's unit within the step (KC)
    __device__ static int unit_k(int i) { return ((unit(i) % 4) ^ ((unit(i) / 4 >> 1) & 3)) * 8; }

    // The piece from outer index o0 and k0 on, of `outer` and K
    __device__ void aim(const Operand &op, int64_t o0, int64_t outer, int32_t k0, int32_t K)
    {
        line = (uint32_t)op.ld * 2;
        const int64_t here = outer - o0 < R ? outer - o0 : R;
        if (LAYOUT == LAYOUT_KC) {
            base = (uint64_t)op.p + (uint64_t)o0 * line;
            size = (uint32_t)(here - 1) * line + (uint32_t)(K + 7) / 8 * 16; // whole units: what is behind the last k are zeros
            scalar = (uint32_t)k0 * 2;
        } else {
            base = (uint64_t)op.p + (uint64_t)k0 * line + (uint64_t)o0 * 2;
            size = (uint32_t)(here + 7) / 8 * 16;
            scalar = 0;
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int u = unit(i);
            if (LAYOUT == LAYOUT_KC) {
                offset[i] = (uint32_t)(u / 4) * line + unit_k(i) * 2;
            } else {
                const int k = u / (R / 8), turn = line_turn<R>(k);
                offset[i] = (uint32_t)k * line + ((u % (R / 8)) ^ (turn << 1)) * 16;
            }
        }
    }

    // The step whose operand has `left` more k (none: nothing is read, and zeros arrive)
    __device__ void prepare(int32_t left)
    {
        uint32_t bytes;
        if (LAYOUT == LAYOUT_KC) {
            bytes = left > 0 ? size : 0;
        } else {
            const int32_t lines = left < DIRECT_K ? left : DIRECT_K;
            bytes = left > 0 ? (uint32_t)(lines - 1) * line + size : 0;
        }
        rsrc = int4v{__builtin_amdgcn_readfirstlane((int)(uint32_t)base), __builtin_amdgcn_readfirstlane((int)(uint32_t)(base >> 32) & 0xffff),
                     __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000};
    }

    // Load i of that step, to LDS
    __device__ void load(int i, uint32_t lds, int32_t left, int wave) const
    {
        const uint32_t off = LAYOUT == LAYOUT_KC && unit_k(i) >= left ? NOWHERE : offset[i]; // the row's end
        load_to_lds(rsrc, off, scalar, lds + (uint32_t)(wave * 64 + i * THREADS) * 16);
    }

    __device__ void advance()
    {
        if (LAYOUT == LAYOUT_KC) scalar += DIRECT_K * 2;
        else base += (uint64_t)DIRECT_K * line;
    }

    // On to the same lines' continuation in another operand of the same ld
    __device__ void turn_to(const char *p, int64_t o0, bool now)
    {
        const uint64_t there = (uint64_t)p + (LAYOUT == LAYOUT_KC ? (uint64_t)o0 * line : (uint64_t)o0 * 2);
        base = now ? there : base;
        if (LAYOUT == LAYOUT_KC) scalar = now ? 0 : scalar;
    }
};

// What a launch forms: all tiles but the tail, parts of all tiles, or parts of the tail's tiles
constexpr int WHOLE = 0, PARTS = 1, TAIL_PARTS = 2;

// GATED: the N side is a piece of 128 columns of each of the two products
template <class T, int LM, int LN, int EPI, int FORM>
__global__ __launch_bounds__(DIRECT_THREADS, 2) void product_direct_kernel(const ProductArgs a)
{
    constexpr bool TURNS = EPI == EPI_GATED, SEGMENTS = LM == LAYOUT_KC && LN == LAYOUT_KC;
    constexpr int BM = DIRECT_TILE, BN = DIRECT_TILE, BK = DIRECT_K, COLS = TURNS ? BN / 2 : BN, PIECES = BN / COLS;
    constexpr int WN = 4, FM = 8, FN = 4, UNITS_M = BM * BK / 8, UNITS_N = COLS * BK / 8, STEP_UNITS = UNITS_M + PIECES * UNITS_N;
    constexpr int LOADS_M = UNITS_M / DIRECT_THREADS, LOADS_N = UNITS_N / DIRECT_THREADS, LOADS = LOADS_M + PIECES * LOADS_N; // of a wavefront and step
    __shared__ short8 lds[DIRECT_DEPTH * STEP_UNITS];

    const int64_t tile_rows = (a.M + BM - 1) / BM, tile_cols = (a.N + COLS - 1) / COLS, tiles = tile_rows * tile_cols;
    const int64_t whole = tiles * a.sets - a.tail;
    int64_t id = tile_of(a.first + blockIdx.x, FORM == WHOLE ? whole : FORM == PARTS ? tiles * a.splits * a.sets : (int64_t)a.tail * a.splits), row_tile, col_tile;
    const int64_t part_of_tail = id; // TAIL_PARTS
    if (FORM == TAIL_PARTS) id = whole + id % a.tail;
    const int64_t each = FORM == PARTS ? tiles * a.splits : tiles;
    const int set = a.sets > 1 ? (int)(id / each) : 0;
    id -= set * each;
    const int split = FORM == PARTS ? (int)(id / tiles) : FORM == TAIL_PARTS ? (int)(part_of_tail / a.tail) : 0;
    tile_place(FORM == PARTS ? id - split * tiles : id, tile_rows, tile_cols, row_tile, col_tile);
    const int64_t m0 = row_tile * BM, n0 = col_tile * COLS;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), lane = threadIdx.x % 64, wm = wave / WN * 128, wn = wave % WN * 64;

    float4v acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};

    const int32_t K = (int32_t)a.K, steps_each = (K + BK - 1) / BK, all = SEGMENTS ? steps_each * a.segments : steps_each;
    const int32_t begin = FORM != WHOLE ? split * a.steps_per_split : 0;
    const int32_t end = FORM != WHOLE && begin + a.steps_per_split < all ? begin + a.steps_per_split : all;

    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) short8 *)lds;
    DirectPiece<LM, BM, DIRECT_THREADS> pm;
    DirectPiece<LN, COLS, DIRECT_THREADS> pn[PIECES];
    int32_t next = begin, left, segment = SEGMENTS && begin >= steps_each ? 1 : 0; // step of the next loads, k that are left from there on, its segment
    uint32_t to;
    {
        const int which = set + segment; // one of them is 0
        const int32_t k0 = (begin - segment * steps_each) * BK;
        pm.aim(a.a[which], m0, a.M, k0, K);
#pragma unroll
        for (int q = 0; q < PIECES; ++q) pn[q].aim(a.b[TURNS ? q : which], n0, a.N, k0, K);
    }
    const char *second_m = a.a[1].p, *second_n = a.b[1].p;
    auto prepare = [&]() { // the loads of step `next`
        if (SEGMENTS) {
            const bool now = next == steps_each && segment == 0 && a.segments > 1;
            pm.turn_to(second_m, m0, now);
            pn[0].turn_to(second_n, n0, now);
            segment = now ? 1 : segment;
        }
        left = K - (next - segment * steps_each) * BK;
        left = next < end ? left : 0;
        to = lds0 + (uint32_t)((next - begin) % DIRECT_DEPTH) * (STEP_UNITS * 16);
        pm.prepare(left);
#pragma unroll
        for (int q = 0; q < PIECES; ++q) pn[q].prepare(left);
    };
    auto load = [&](int i) { // one of LOADS
        if (i < LOADS_M) pm.load(i, to, left, wave);
        else pn[(i - LOADS_M) / LOADS_N].load((i - LOADS_M) % LOADS_N, to + (UNITS_M + (i - LOADS_M) / LOADS_N * UNITS_N) * 16, left, wave);
    };
    auto advance = [&]() {
        pm.advance();
#pragma unroll
        for (int q = 0; q < PIECES; ++q) pn[q].advance();
        ++next;
    };
    short8 fm[FM], fn[2][FN];
    auto read_m = [&](int t, int i) { return fragment<LM, BM, BK>(lds + t % DIRECT_DEPTH * STEP_UNITS, wm + 16 * i, 0, lane); };
    auto read_n = [&](int t, int j) {
        const short8 *at = lds + t % DIRECT_DEPTH * STEP_UNITS + UNITS_M;
        return TURNS ? fragment<LN, COLS, BK>(at + j % 2 * UNITS_N, wn / 2 + 8 * (j - j % 2), 0, lane) : fragment<LN, COLS, BK>(at, wn + 16 * j, 0, lane);
    };

#pragma unroll
    for (int d = 0; d < DIRECT_DEPTH - 1; ++d) {
        prepare();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load(i);
        advance();
    }
    prepare();
    wait_loads_and_meet<(DIRECT_DEPTH - 2) * LOADS>();
#pragma unroll
    for (int i = 0; i < FM; ++i) fm[i] = read_m(0, i);
#pragma unroll
    for (int j = 0; j < FN; ++j) fn[0][j] = read_n(0, j);
    // Matrix instructions in groups of one fragment of the M side, with a load and a fragment of the N side beside each of the first four and the scalar
    // arithmetic of the next loads in the last four; the barriers keep the compiler from moving reads that the next step begins with to its end.
    static_assert(LOADS == 4 && FN == 4 && FM == 8, "the groups of a step");
    auto step = [&](int t, auto parity) {
        constexpr int Q = decltype(parity)::value;
        wait_loads_and_meet<(DIRECT_DEPTH - 3) * LOADS>();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            if (i < LOADS) load(i);
            if (i < FN) fn[1 - Q][i] = read_n(t + 1, i);
            if (i == LOADS) {
                advance();
                prepare();
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = mfma<T>(fn[Q][j], fm[i], acc[i][j]);
            fm[i] = read_m(t + 1, i);
            if (i < LOADS) __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    for (int32_t t = 0; t < end - begin; t += 2) { // an odd number of steps ends with one of zeros
        step(t, std::integral_constant<int, 0>());
        step(t + 1, std::integral_constant<int, 1>());
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); // no load into LDS outlives the workgroup

    if constexpr (FORM == TAIL_PARTS) {
        float *to = a.partial + (part_of_tail * BM + wm + lane % 16) * BN + wn + 4 * (lane / 16);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) *reinterpret_cast<float4v *>(to + 16 * i * BN + 16 * j) = acc[i][j];
    } else {
        finish_tile<T, EPI, FORM == PARTS, BM>(a, set, split, m0, n0, wm, wn, COLS, acc);
    }
}

// The parts of the tail's tiles added in fp64, in order, 16 rows of a tile a workgroup.  GATED: 16 columns of a tile are of the first product, 16 of the second, and so on.
template <class T, int EPI> __global__ __launch_bounds__(256) void product_tail_kernel(const ProductArgs a)
{
    constexpr int Q = EPI == EPI_GATED ? 2 : 1, BM = DIRECT_TILE, BN = DIRECT_TILE, COLS = BN / Q, FOURS = COLS / 4, ROWS = 256 / FOURS;
    const int64_t tile_rows = (a.M + BM - 1) / BM, tile_cols = (a.N + COLS - 1) / COLS, tiles = tile_rows * tile_cols;
    const int tile = (int)((a.first + blockIdx.x) / (BM / 16)), rows16 = (int)((a.first + blockIdx.x) % (BM / 16));
    const int64_t id = tiles * a.sets - a.tail + tile;
    const int set = (int)(id / tiles);
    int64_t row_tile, col_tile;
    tile_place(id - set * tiles, tile_rows, tile_cols, row_tile, col_tile);
    const int in_row = threadIdx.x % FOURS * 4, at = Q == 2 ? in_row / 16 * 32 + in_row % 16 : in_row;
    const int64_t col = col_tile * COLS + in_row;
    const int left = a.N - col < 4 ? (int)(a.N - col) : 4;
    if (left <= 0) return;
#pragma unroll
    for (int r = 0; r < 16; r += ROWS) {
        const int in = 16 * rows16 + r + threadIdx.x / FOURS;
        const int64_t row = row_tile * BM + in;
        if (row >= a.M) return;
        double sum[Q][4] = {};
        for (int s = 0; s < a.splits; ++s)
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const float4v v = *reinterpret_cast<const float4v *>(a.partial + (((int64_t)s * a.tail + tile) * BM + in) * BN + at + 16 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[q][i] += (double)v[i];
            }
        float s[Q][4];
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[q][i] = (float)sum[q][i];
        finish4<T, EPI>(a, set, row, col, left, s[0], s[Q - 1]);
    }
}

template <class T, int LM, int LN, int EPI, int FORM> int launch_direct(ProductArgs &a, hipStream_t stream)
{
    constexpr int COLS = EPI == EPI_GATED ? DIRECT_TILE / 2 : DIRECT_TILE;
    const int64_t tiles = (a.M + DIRECT_TILE - 1) / DIRECT_TILE * ((a.N + COLS - 1) / COLS) * a.sets;
    return launch_parts(FORM == WHOLE ? tiles - a.tail : FORM == PARTS ? tiles * a.splits : (int64_t)a.tail * a.splits, [&](unsigned first, unsigned count) {
        a.first = first;
        product_direct_kernel<T, LM, LN, EPI, FORM><<<count, DIRECT_THREADS, 0, stream>>>(a);
    });
}

// All tiles of a product that is not cut, and those of a last round that would leave most CUs idle in parts
template <class T, int LM, int LN, int EPI> int launch_whole(const ProductPlan &plan, ProductArgs &a, hipStream_t stream)
{
    a.tail = plan.tail;
    if (int rc = launch_direct<T, LM, LN, EPI, WHOLE>(a, stream)) return rc;
    if (!a.tail) return SLICEGCN_OK;
    a.splits = plan.tail_splits;
    if (int rc = launch_direct<T, LM, LN, EPI, TAIL_PARTS>(a, stream)) return rc;
    return launch_parts((int64_t)a.tail * (DIRECT_TILE / 16), [&](unsigned first, unsigned count) {
        a.first = first;
        product_tail_kernel<T, EPI><<<count, 256, 0, stream>>>(a);
    });
}

} // namespace
} // namespace slicegcn
