// Products of few rows (up to 32) of 16-bit operands that lie on 16-byte boundaries, sums of up to 2048: a request or some requests at a time, where the weights are all there is
// to read, and a second launch would take as long as reading them.
//
// A workgroup forms all rows of a strip of 64 columns (GATED: 32 of each product).  Its wavefronts share out the strip's k, each with a ring of its own in LDS
// that its loads go to straight from memory, ROWS_DEPTH - 1 steps of 32 k ahead: no barrier in the loop, and some 80 KB on their way per CU.  The
// wavefronts' sums are added in order through LDS at the end.  One row 1024 -> 2816 gated bf16: 6.4 us, 1.8 TB/s; bound by the latency of the launch and of a wavefront's four
// steps.
#pragma once

#include "product_direct.h"

namespace slicegcn {
namespace {

constexpr int ROWS_DEPTH = 3, ROWS_WAVES = 8;

// F: 16 rows each
template <class T, int LN, int EPI, int F> __global__ __launch_bounds__(64 * ROWS_WAVES) void product_rows_kernel(const ProductArgs a)
{
    constexpr bool TURNS = EPI == EPI_GATED, SEGMENTS = LN == LAYOUT_KC;
    constexpr int WAVES = ROWS_WAVES, BK = DIRECT_K, COLS = TURNS ? 32 : 64, PIECES = 64 / COLS, FN = 4;
    constexpr int UNITS_M = 16 * F * BK / 8, UNITS_N = COLS * BK / 8, STEP_UNITS = UNITS_M + PIECES * UNITS_N;
    constexpr int LOADS_M = UNITS_M / 64, LOADS_N = UNITS_N / 64, LOADS = LOADS_M + PIECES * LOADS_N;
    constexpr int RING = ROWS_DEPTH * STEP_UNITS, SUMS = 16 * F * 64; // floats of a wavefront's sums
    static_assert(SUMS * 4 <= RING * 16, "the sums take the place of the rings");
    __shared__ short8 lds[WAVES * RING];

    const int64_t n0 = (a.first + blockIdx.x) * COLS;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), lane = threadIdx.x % 64;

    float4v acc[F][FN];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};

    const int32_t K = (int32_t)a.K, steps_each = (K + BK - 1) / BK, all = SEGMENTS ? steps_each * a.segments : steps_each;
    const int32_t share = (all + WAVES - 1) / WAVES, begin = wave * share, end = begin + share < all ? begin + share : all;

    const short8 *ring = lds + wave * RING;
    const uint32_t ring0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) short8 *)lds + (uint32_t)wave * (RING * 16);
    DirectPiece<LAYOUT_KC, 16 * F, 64> pm;
    DirectPiece<LN, COLS, 64> pn[PIECES];
    int32_t next = begin, segment = SEGMENTS && begin >= steps_each ? 1 : 0, slot = 0;
    {
        const int32_t k0 = (begin - segment * steps_each) * BK;
        pm.aim(a.a[segment], 0, a.M, k0, K);
#pragma unroll
        for (int q = 0; q < PIECES; ++q) pn[q].aim(a.b[TURNS ? q : segment], n0, a.N, k0, K);
    }
    const char *second_m = a.a[1].p, *second_n = a.b[1].p;
    auto issue = [&]() { // the loads of step `next`; of one that is not there, zeros
        if (SEGMENTS) {
            const bool now = next == steps_each && segment == 0 && a.segments > 1;
            pm.turn_to(second_m, 0, now);
            pn[0].turn_to(second_n, n0, now);
            segment = now ? 1 : segment;
        }
        int32_t left = K - (next - segment * steps_each) * BK;
        left = next < end ? left : 0;
        const uint32_t to = ring0 + (uint32_t)slot * (STEP_UNITS * 16);
        pm.prepare(left);
#pragma unroll
        for (int i = 0; i < LOADS_M; ++i) pm.load(i, to, left, 0);
        pm.advance();
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            pn[q].prepare(left);
#pragma unroll
            for (int i = 0; i < LOADS_N; ++i) pn[q].load(i, to + (UNITS_M + q * UNITS_N) * 16, left, 0);
            pn[q].advance();
        }
        ++next;
        slot = slot == ROWS_DEPTH - 1 ? 0 : slot + 1;
    };
#pragma unroll
    for (int d = 0; d < ROWS_DEPTH - 1; ++d) issue();
    int at = 0;
    for (int32_t t = begin; t < end; ++t) {
        // the reads of the step before have arrived, so its place is free for the loads that go there now
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        issue();
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((ROWS_DEPTH - 1) * LOADS) : "memory");
        __builtin_amdgcn_sched_barrier(0);
        const short8 *here = ring + at * STEP_UNITS;
        at = at == ROWS_DEPTH - 1 ? 0 : at + 1;
        short8 fn[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j)
            fn[j] = TURNS ? fragment<LN, COLS, BK>(here + UNITS_M + j % 2 * UNITS_N, 8 * (j - j % 2), 0, lane) : fragment<LN, COLS, BK>(here + UNITS_M, 16 * j, 0, lane);
#pragma unroll
        for (int i = 0; i < F; ++i) {
            const short8 fm = fragment<LAYOUT_KC, 16 * F, BK>(here, 16 * i, 0, lane);
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = mfma<T>(fn[j], fm, acc[i][j]);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();

    // [wavefront][row][column]: GATED 32 columns of the first product, then 32 of the second
    float *sums = reinterpret_cast<float *>(lds);
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int col = (TURNS ? j % 2 * 32 + 8 * (j - j % 2) : 16 * j) + 4 * (lane / 16);
            *reinterpret_cast<float4v *>(sums + wave * SUMS + (16 * i + lane % 16) * 64 + col) = acc[i][j];
        }
    __syncthreads();
    for (int q = threadIdx.x; q < 16 * F * (COLS / 4); q += 64 * WAVES) {
        const int64_t row = q / (COLS / 4), col = n0 + q % (COLS / 4) * 4;
        const int left = a.N - col < 4 ? (int)(a.N - col) : 4;
        if (row >= a.M || left <= 0) continue;
        float s[PIECES][4] = {};
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float4v v = *reinterpret_cast<const float4v *>(sums + w * SUMS + row * 64 + p * 32 + q % (COLS / 4) * 4);
#pragma unroll
                for (int r = 0; r < 4; ++r) s[p][r] += v[r];
            }
        finish4<T, EPI>(a, 0, row, col, left, s[0], s[PIECES - 1]);
    }
}

template <class T, int LN, int EPI> int launch_rows(ProductArgs &a, hipStream_t stream)
{
    constexpr int COLS = EPI == EPI_GATED ? 32 : 64;
    return launch_parts((a.N + COLS - 1) / COLS, [&](unsigned first, unsigned count) {
        a.first = first;
        if (a.M <= 16) product_rows_kernel<T, LN, EPI, 1><<<count, 64 * ROWS_WAVES, 0, stream>>>(a);
        else product_rows_kernel<T, LN, EPI, 2><<<count, 64 * ROWS_WAVES, 0, stream>>>(a);
    });
}

} // namespace
} // namespace slicegcn
