// The backward pass of a narrow product or gated projection of 16-bit rows on many rows, in one sweep over them: up to 128 columns of X and 256 of the gradients before
// the activation (GATED: 128 of each product).
//
//   dP = dY act'(P)   or   dG = dH U act'(G), dU = dH act(G);   dX = dP W^T;   dW += X^T dP;   db += column sums of dP
//
// Such layers are bound by their rows, which the passes of the general form read several times and between which the gradients before the activation go to memory and
// back.  Here a workgroup of eight wavefronts stays for the whole launch and takes 32 rows at a time: two such blocks are on their way into registers while one is
// worked on; the gradients before the activation are formed on the way to LDS, whose rows then are both the M side of dX (k along the rows: 16-byte reads) and the
// N side of dW (k across the rows: transposing reads).  The weights for dX stay in registers, a wavefront's for 16 columns of dX, and so do the sums of dW, a
// wavefront's 64 x 64.  Nothing in the loop branches on a lane: rows and columns that are not there are read as zeros and not written by the buffers' range checks, so
// that the compiler can count the loads in flight.
// 2.4 M rows 100 -> 256 bf16 gelu: 0.96 ms, 3.6 TB/s; bound by the arithmetic of the gelu's slope (some 35 instructions an element).
// Order of the sums: a workgroup's blocks in turn (1024 at most), the workgroups' sums in fp64 in order.
#pragma once

#include "product_kernels.h"

namespace slicegcn {
namespace {

constexpr int NARROW_THREADS = 512, NARROW_X = NARROW_WIDTH_IN / 8, NARROW_G = NARROW_WIDTH_OUT / 8; // units of 8 columns

// A block's rows of a matrix as a buffer
__device__ inline __amdgpu_buffer_rsrc_t rows_buffer(const char *p, int64_t ld, int64_t row0, int64_t n, int32_t w)
{
    const int64_t rows = n - row0 < NARROW_ROWS ? n - row0 : NARROW_ROWS;
    const int32_t bytes = rows > 0 ? (int32_t)((rows - 1) * ld + w) * 2 : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p + row0 * ld * 2), 0, bytes, 0x00020000);
}

// Units of a row in LDS are permuted in pairs by its index: eight lanes that read a unit of eight rows, and sixteen that read a pair of units of four rows and of the
// four rows eight further, meet in different banks.
__device__ inline int row_turn(int row) { return ((row & 7) ^ ((row >> 3 & 1) << 2)) << 1; }

template <int UNITS> __device__ inline short8 narrow_rows(const short8 *tile, int row0, int unit0, int lane)
{
    const int row = row0 + lane % 16;
    return tile[row * UNITS + ((unit0 + lane / 16) ^ row_turn(row))];
}

template <int UNITS> __device__ inline short8 narrow_columns(const short8 *tile, int col0, int lane)
{
    short8 f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int k = 8 * (lane / 16) + 4 * h + lane % 16 / 4, col = col0 + 4 * (lane % 4);
        short *at = reinterpret_cast<short *>(const_cast<short8 *>(tile) + k * UNITS + ((col / 8) ^ row_turn(k))) + col % 8;
        const short4v t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v *)at);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[4 * h + i] = t[i];
    }
    return f;
}

template <class T, bool GATED, int ACT>
__global__ __launch_bounds__(NARROW_THREADS, 2) void product_narrow_kernel(const NarrowArgs a)
{
    constexpr int Q = GATED ? 2 : 1, EACH = GATED ? 1 : 2; // pieces of the gradients; units of a piece and block that a thread forms
    constexpr int PIECE = NARROW_G / Q;                    // units
    constexpr bool SLOPES = GATED || ACT != SLICEGCN_ACT_NONE;
    constexpr uint32_t NOWHERE = 0xffffff00u; // beyond any buffer
    __shared__ short8 tile_g[2][NARROW_ROWS * NARROW_G], tile_x[2][NARROW_ROWS * NARROW_X];
    const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);

    // the weights of dX's columns 16 wave .. + 15, k in the order of a row of tile_g
    short8 fw[8];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
        const int k = kk * 32 + 8 * (lane / 16), q = k / (8 * PIECE), col = k % (8 * PIECE), row = 16 * wave + lane % 16;
        T v[8];
        const bool there = a.dx != nullptr && row < a.w_in && col < a.w_out;
        const T *p = reinterpret_cast<const T *>(a.w[q].p) + (there ? (int64_t)row * a.w[q].ld + col : 0);
        load8(p, there ? a.w_out - col : 0, v);
        __builtin_memcpy(&fw[kk], v, 16);
    }

    // the thread's units: of a piece, unit tid % PIECE of rows tid / PIECE and on; of X, unit tid % NARROW_X of row tid / NARROW_X
    const int unit = tid % PIECE, row = tid / PIECE, left = a.w_out - unit * 8; // columns of the unit that exist
    uint32_t at_d[EACH], at_g[EACH], at_u[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int r = row + i * (NARROW_THREADS / PIECE);
        at_d[i] = left > 0 ? (uint32_t)(r * a.d.ld + unit * 8) * 2 : NOWHERE;
        at_g[i] = left > 0 ? (uint32_t)(r * a.g.ld + unit * 8) * 2 : NOWHERE;
        at_u[i] = left > 0 ? (uint32_t)(r * a.u.ld + unit * 8) * 2 : NOWHERE;
    }
    const int x_unit = tid % NARROW_X, x_row = tid / NARROW_X;
    const uint32_t at_x = x_unit * 8 < a.w_in ? (uint32_t)(x_row * a.x.ld + x_unit * 8) * 2 : NOWHERE;

    struct Loaded {
        uint4v d[EACH], g[EACH], u[EACH], x;
    };
    auto load = [&](int64_t block, Loaded &l) {
        const int64_t row0 = block * NARROW_ROWS;
        const auto bd = rows_buffer(a.d.p, a.d.ld, row0, a.n, a.w_out);
#pragma unroll
        for (int i = 0; i < EACH; ++i) l.d[i] = __builtin_amdgcn_raw_buffer_load_b128(bd, at_d[i], 0, 0);
        if (SLOPES) {
            const auto bg = rows_buffer(a.g.p, a.g.ld, row0, a.n, a.w_out);
#pragma unroll
            for (int i = 0; i < EACH; ++i) l.g[i] = __builtin_amdgcn_raw_buffer_load_b128(bg, at_g[i], 0, 0);
        }
        if (GATED) {
            const auto bu = rows_buffer(a.u.p, a.u.ld, row0, a.n, a.w_out);
#pragma unroll
            for (int i = 0; i < EACH; ++i) l.u[i] = __builtin_amdgcn_raw_buffer_load_b128(bu, at_u[i], 0, 0);
        }
        if (a.want_w) l.x = __builtin_amdgcn_raw_buffer_load_b128(rows_buffer(a.x.p, a.x.ld, row0, a.n, a.w_in), at_x, 0, 0);
    };

    float run[Q][8] = {};
    double total[Q][8] = {};
    typedef T T8 __attribute__((ext_vector_type(8)));
    auto form = [&](const Loaded &l, short8 *to_g, short8 *to_x) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const T8 d = __builtin_bit_cast(T8, l.d[i]);
            T8 g, u, o[Q];
            if (SLOPES) g = __builtin_bit_cast(T8, l.g[i]);
            if (GATED) u = __builtin_bit_cast(T8, l.u[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float y = 0.f, slope = 1.f, v[Q];
                if (SLOPES) activated_slope<ACT>((float)g[j], y, slope);
                v[0] = through_slope<ACT>(GATED ? (float)d[j] * (float)u[j] : (float)d[j], SLOPES ? (float)g[j] : 0.f, slope);
                if (GATED) v[Q - 1] = (float)d[j] * y;
#pragma unroll
                for (int q = 0; q < Q; ++q) {
                    v[q] = j < left ? v[q] : 0.f; // columns behind the last one are not the row's
                    run[q][j] += v[q];
                    o[q][j] = (T)v[q];
                }
            }
            const int r = row + i * (NARROW_THREADS / PIECE);
#pragma unroll
            for (int q = 0; q < Q; ++q) to_g[r * NARROW_G + ((q * PIECE + unit) ^ row_turn(r))] = __builtin_bit_cast(short8, o[q]);
        }
        if (a.want_w) to_x[x_row * NARROW_X + (x_unit ^ row_turn(x_row))] = __builtin_bit_cast(short8, l.x);
    };

    const int wa = wave / 4 * 64, wb = wave % 4 * 64; // the wavefront's sums of dW: rows, columns
    float4v sum[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
    // whether there is anything in 64 columns of a row of tile_g
    auto filled = [&](int col) { return col % (8 * PIECE) < a.w_out; };
    const bool has_w = a.want_w && wa < a.w_in && filled(wb), has_x = a.dx != nullptr && 16 * wave < a.w_in;
    const int x_cols = a.w_in - (16 * wave + 4 * (lane / 16)); // columns of dX from the lane's on
    auto multiply = [&](int64_t block, const short8 *g, const short8 *x) {
        if (has_x) {
            const auto to = rows_buffer(a.dx, a.lddx, block * NARROW_ROWS, a.n, a.w_in);
#pragma unroll
            for (int i = 0; i < NARROW_ROWS / 16; ++i) {
                float4v s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                    if (filled(kk * 32)) s = mfma<T>(fw[kk], narrow_rows<NARROW_G>(g, 16 * i, kk * 4, lane), s);
                typedef T T4 __attribute__((ext_vector_type(4)));
                T4 o;
#pragma unroll
                for (int r = 0; r < 4; ++r) o[r] = (T)s[r];
                const uint2v v = __builtin_bit_cast(uint2v, o);
                const uint32_t at = (uint32_t)((16 * i + lane % 16) * a.lddx + 16 * wave + 4 * (lane / 16)) * 2;
                if (a.w_in % 4 == 0) {
                    __builtin_amdgcn_raw_buffer_store_b64(v, to, x_cols >= 4 ? at : NOWHERE, 0, 0);
                } else { // even
                    __builtin_amdgcn_raw_buffer_store_b32(v[0], to, x_cols >= 2 ? at : NOWHERE, 0, 0);
                    __builtin_amdgcn_raw_buffer_store_b32(v[1], to, x_cols >= 4 ? at + 4 : NOWHERE, 0, 0);
                }
            }
        }
        if (has_w) {
            short8 fx[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) fx[i] = narrow_columns<NARROW_X>(x, wa + 16 * i, lane);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const short8 fg = narrow_columns<NARROW_G>(g, wb + 16 * j, lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i][j] = mfma<T>(fg, fx[i], sum[i][j]);
            }
        }
    };

    // Block b of this workgroup goes to buffer b % 2 of LDS.  Who writes it has met the others behind block b - 1, and so behind their reads of block b - 2.
    const int64_t blocks = (a.n + NARROW_ROWS - 1) / NARROW_ROWS, stride = gridDim.x;
    Loaded l[2];
    load(blockIdx.x, l[0]);
    load(blockIdx.x + stride, l[1]);
    int in_run = 0;
    auto turn = [&](int64_t block, auto parity) {
        constexpr int B = decltype(parity)::value;
        form(l[B], tile_g[B], tile_x[B]);
        load(block + 2 * stride, l[B]); // zeros behind the last block
        if ((in_run += 1) == NARROW_RUN) {
            in_run = 0;
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    total[q][j] += (double)run[q][j];
                    run[q][j] = 0.f;
                }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        multiply(block, tile_g[B], tile_x[B]);
    };
    for (int64_t block = blockIdx.x; block < blocks; block += 2 * stride) { // a second block that is not there is of zeros
        turn(block, std::integral_constant<int, 0>());
        turn(block + stride, std::integral_constant<int, 1>());
    }

    if (has_w) {
        // [set][workgroup][w_in][w_out], as product_join_kernel takes it
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int m = wa + 16 * i + lane % 16;
            if (m >= a.w_in) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = wb + 16 * j + 4 * (lane / 16), q = c / (8 * PIECE), col = c % (8 * PIECE), n_left = a.w_out - col < 4 ? a.w_out - col : 4;
                if (n_left <= 0) continue;
                float s[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) s[r] = sum[i][j][r];
                store4<float>(reinterpret_cast<char *>(a.partial), (((int64_t)q * gridDim.x + blockIdx.x) * a.w_in + m) * a.w_out + col, n_left, s);
            }
        }
    }
    if (a.columns) {
        __syncthreads();
        // the threads of a unit of columns, rows ascending
        double *sums = reinterpret_cast<double *>(tile_g); // 32 KB
        static_assert(sizeof(tile_g) >= NARROW_THREADS * 8 * sizeof(double), "column sums");
#pragma unroll
        for (int q = 0; q < Q; ++q) {
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[tid * 8 + j] = total[q][j] + (double)run[q][j];
            __syncthreads();
            if (row == 0 && left > 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j >= left) continue;
                    double t = 0.0;
                    for (int r = 0; r < NARROW_THREADS / PIECE; ++r) t += sums[(r * PIECE + unit) * 8 + j];
                    a.columns[((int64_t)blockIdx.x * Q + q) * a.w_out + unit * 8 + j] = t;
                }
            }
            __syncthreads();
        }
    }
}

template <class T> int launch_narrow(const NarrowArgs &a, int act, bool gated, unsigned blocks, hipStream_t stream)
{
    with_act(act, [&](auto c) {
        if (gated) product_narrow_kernel<T, true, decltype(c)::value><<<blocks, NARROW_THREADS, 0, stream>>>(a);
        else product_narrow_kernel<T, false, decltype(c)::value><<<blocks, NARROW_THREADS, 0, stream>>>(a);
    });
    SG_LAUNCH_CHECK();
    return SLICEGCN_OK;
}

} // namespace
} // namespace slicegcn
