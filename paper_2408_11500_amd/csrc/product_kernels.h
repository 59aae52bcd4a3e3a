// The kernels of product.h for one element type (each type is compiled by a file of its own).
//
// A workgroup forms a tile of BM x BN results.  Per step of k both operands' pieces go through registers into LDS as 16-bit values, and from there into the
// operand registers of v_mfma_f32_16x16x32: the N side is the instruction's first operand, so that a lane ends up with four consecutive columns of
// a row.  Pieces stay in the order of memory: those with k first are read 16 bytes (8 k of a row) at a time, the others with the
// transposing read ds_read_b64_tr_b16, of which 16 lanes together take 4 k of 16 columns and get 4 k of a column each.
// fp32 operands are split into three bf16 terms each, x = x0 + x1 + x2, every term the rest rounded to 8 bits: |x1| <= 2^-8 |x|, |x2| <= 2^-16 |x|, and what
// is left is at most 2^-24 |x|.  Six products are added, smallest first; the three that are left out are below 2^-23 of the product together.  Six bf16
// instructions take 96 cycles for what the fp32 instruction takes 256 for.
#pragma once

#include "product.h"

namespace slicegcn {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short short8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));

template <class T> struct Planes { static constexpr int count = 1; };
template <> struct Planes<float> { static constexpr int count = 3; };

template <class T> __device__ inline float4v mfma(short8 a, short8 b, float4v c)
{
    if constexpr (std::is_same_v<T, f16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Eight elements of a line of which `left` exist; zeros beyond
template <class T> __device__ inline void load8(const T *p, int64_t left, T (&v)[8])
{
    constexpr int V = 16 / sizeof(T);
    if (left >= 8) {
#pragma unroll
        for (int i = 0; i < 8; i += V) {
            const auto x = load_vec<T, V>(p + i);
#pragma unroll
            for (int j = 0; j < V; ++j) v[i + j] = x[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : (T)0.f;
    }
}

// The 16-bit terms of eight elements
template <class T> __device__ inline void split8(const T (&v)[8], short8 (&out)[Planes<T>::count])
{
    if constexpr (std::is_same_v<T, float>) {
        typedef float float2v __attribute__((ext_vector_type(2)));
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        uint32_t w[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float2v rest = {v[2 * i], v[2 * i + 1]};
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                w[p][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, bf16x2)); // to nearest
                rest[0] -= __uint_as_float(w[p][i] << 16);
                rest[1] -= __uint_as_float(w[p][i] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int p = 0; p < 3; ++p) __builtin_memcpy(&out[p], w[p], 16);
    } else {
        __builtin_memcpy(&out[0], v, 16);
    }
}

// Where a tile's piece of an operand lies in LDS (in 16-byte units; R outer indexes by BK of k), so that the lanes of a read meet in different banks:
// KC: a row's units are permuted by its index; OC: 32-byte pairs of units of a line of k are permuted by its index, as the transposing read takes pairs.
template <int R> __device__ inline int line_turn(int k) { return ((k & 3) | ((k >> 3) & 1) << 2) & (R / 16 - 1); }
template <int LAYOUT, int R, int BK> __device__ inline int lds_unit(int outer_or_unit, int k_or_unit)
{
    if constexpr (LAYOUT == LAYOUT_KC) {
        const int row = outer_or_unit, unit = k_or_unit;
        return row * (BK / 8) + (unit ^ (BK == 64 ? row & 7 : (row >> 1) & 3));
    } else {
        const int unit = outer_or_unit, k = k_or_unit;
        return k * (R / 8) + (unit ^ (line_turn<R>(k) << 1));
    }
}

// A piece of an operand on its way from memory to LDS, 8 elements a unit
template <class T, int LAYOUT, int R, int BK, int THREADS, bool TURNS> struct Piece {
    static constexpr int UNITS = R * BK / 8, EACH = (UNITS + THREADS - 1) / THREADS;
    T v[EACH][8];

    // outer indexes from o0 on (of `outer` in all), k from k0 on (of K).  TURNS: 16 columns of the first operand, 16 of the second, and so on.
    __device__ void load(const Operand *op, int64_t o0, int64_t outer, int64_t k0, int64_t K)
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int q = threadIdx.x + i * THREADS;
            if (UNITS % THREADS != 0 && q >= UNITS) break;
            int64_t o, k;
            int which = 0;
            if constexpr (LAYOUT == LAYOUT_KC) {
                static_assert(!TURNS, "only columns take turns");
                o = o0 + q / (BK / 8);
                k = k0 + q % (BK / 8) * 8;
            } else {
                k = k0 + q / (R / 8);
                const int c = q % (R / 8) * 8;
                if (TURNS) {
                    which = c / 16 % 2;
                    o = o0 + c / 32 * 16 + c % 16;
                } else {
                    o = o0 + c;
                }
            }
            const Operand m = op[which];
            const T *p = reinterpret_cast<const T *>(m.p);
            if constexpr (LAYOUT == LAYOUT_KC) load8(p + o * m.ld + k, o < outer ? K - k : 0, v[i]);
            else load8(p + k * m.ld + o, k < K ? outer - o : 0, v[i]);
        }
    }

    __device__ void store(short8 *lds) const
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int q = threadIdx.x + i * THREADS;
            if (UNITS % THREADS != 0 && q >= UNITS) break;
            const int at = LAYOUT == LAYOUT_KC ? lds_unit<LAYOUT, R, BK>(q / (BK / 8), q % (BK / 8)) : lds_unit<LAYOUT, R, BK>(q % (R / 8), q / (R / 8));
            short8 t[Planes<T>::count];
            split8(v[i], t);
#pragma unroll
            for (int p = 0; p < Planes<T>::count; ++p) lds[p * UNITS + at] = t[p];
        }
    }
};

// The operand registers of 16 outer indexes from `base` on and 32 k from 32 * kk on: lane l holds 8 k of the index l % 16
template <int LAYOUT, int R, int BK> __device__ inline short8 fragment(const short8 *lds, int base, int kk, int lane)
{
    if constexpr (LAYOUT == LAYOUT_KC) {
        return lds[lds_unit<LAYOUT, R, BK>(base + lane % 16, kk * 4 + lane / 16)];
    } else {
        short8 f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = kk * 32 + 8 * (lane / 16) + 4 * h + lane % 16 / 4;
            const int column = base + 4 * (lane % 4);
            short *at = reinterpret_cast<short *>(const_cast<short8 *>(lds) + lds_unit<LAYOUT, R, BK>(column / 8, k)) + column % 8;
            const short4v t = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v *)at);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[4 * h + i] = t[i];
        }
        return f;
    }
}

// Workgroup b of a launch runs on XCD b mod 8: consecutive tiles go to one XCD, in strips of 8 rows of tiles, so that its L2 holds what they share
__device__ inline int64_t tile_of(int64_t b, int64_t total)
{
    const int64_t each = total / 8, more = total % 8, xcd = b % 8;
    return xcd * each + (xcd < more ? xcd : more) + b / 8;
}
__device__ inline void tile_place(int64_t t, int64_t rows, int64_t cols, int64_t &row, int64_t &col)
{
    constexpr int64_t STRIP = 8;
    const int64_t strip = t / (STRIP * cols), first = strip * STRIP, high = rows - first < STRIP ? rows - first : STRIP, in = t - first * cols;
    row = first + in % high;
    col = in / high;
}

template <class T> __device__ inline void store4(char *base, int64_t at, int left, const float (&v)[4])
{
    T *p = reinterpret_cast<T *>(base) + at;
    if (left >= 4) {
        store_vec<T, 4>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = (T)v[i];
    }
}

template <class T> __device__ inline void load4(const char *base, int64_t at, int left, float (&v)[4])
{
    const T *p = reinterpret_cast<const T *>(base) + at;
    if (left >= 4) {
        const auto x = load_vec<T, 4>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (float)x[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < left ? (float)p[i] : 0.f;
    }
}

__device__ inline void load_bias(const float *b, int64_t col, int left, float (&v)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = b && i < left ? b[col + i] : 0.f;
}

// Four consecutive results of a row, `left` of which exist.  s: their sums (and of the second product of a gated pair)
template <class T, int EPI>
__device__ inline void finish4(const ProductArgs &a, int set, int64_t row, int64_t col, int left, const float (&s)[4], const float (&s2)[4])
{
    if constexpr (EPI == EPI_STORE) {
        store4<T>(a.out[set], row * a.ldo[set] + col, left, s);
    } else if constexpr (EPI == EPI_FORWARD) {
        float b[4], y[4];
        load_bias(a.bias[0], col, left, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] += s[i];
        if (a.keep[0]) store4<T>(a.keep[0], row * a.ldk[0] + col, left, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = activated(a.act, b[i]);
        if (a.r.p) {
            float r[4];
            load4<T>(a.r.p, row * a.r.ld + col, left, r);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = fmaf(a.residual, r[i], y[i]);
        }
        store4<T>(a.out[0], row * a.ldo[0] + col, left, y);
    } else {
        float g[4], u[4], h[4];
        load_bias(a.bias[0], col, left, g);
        load_bias(a.bias[1], col, left, u);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            g[i] += s[i];
            u[i] += s2[i];
            h[i] = activated(a.act, g[i]) * u[i];
        }
        if (a.keep[0]) {
            store4<T>(a.keep[0], row * a.ldk[0] + col, left, g);
            store4<T>(a.keep[1], row * a.ldk[1] + col, left, u);
        }
        store4<T>(a.out[0], row * a.ldo[0] + col, left, h);
    }
}

// WM x WN wavefronts.  SPLIT: sums of a part of k go to a.partial.
template <class T, int LM, int LN, int EPI, int BM, int BN, int WM, int WN, bool SPLIT>
__global__ __launch_bounds__(64 * WM * WN) void product_kernel(const ProductArgs a)
{
    constexpr int P = Planes<T>::count, BK = P == 3 ? STEP_K_F32 : STEP_K_16, THREADS = 64 * WM * WN;
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr bool TURNS = EPI == EPI_GATED;
    constexpr int COLS = TURNS ? BN / 2 : BN; // columns of results
    static_assert(!TURNS || FN % 2 == 0, "a wavefront holds both products of its columns");
    __shared__ short8 lds[P * (BM + BN) * BK / 8];
    short8 *lds_m = lds, *lds_n = lds + P * BM * BK / 8;

    const int64_t tile_rows = (a.M + BM - 1) / BM, tile_cols = (a.N + COLS - 1) / COLS, tiles = tile_rows * tile_cols;
    int64_t id = tile_of(a.first + blockIdx.x, tiles * a.splits * a.sets), row_tile, col_tile;
    const int set = a.sets > 1 ? (int)(id / (tiles * a.splits)) : 0;
    id -= set * (tiles * a.splits);
    const int split = SPLIT ? (int)(id / tiles) : 0;
    tile_place(id - split * tiles, tile_rows, tile_cols, row_tile, col_tile);
    const int64_t m0 = row_tile * BM, n0 = col_tile * COLS;
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);

    float4v acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};

    const int64_t steps_each = (a.K + BK - 1) / BK, steps = steps_each * a.segments;
    int64_t step = SPLIT ? (int64_t)split * a.steps_per_split : 0;
    const int64_t end = SPLIT && step + a.steps_per_split < steps ? step + a.steps_per_split : steps;
    Piece<T, LM, BM, BK, THREADS, false> pm;
    Piece<T, LN, BN, BK, THREADS, TURNS> pn;
    auto load = [&](int64_t t) {
        const int seg = t >= steps_each ? 1 : 0, which = seg + set; // one of them is 0
        const int64_t k0 = (t - seg * steps_each) * BK;
        pm.load(a.a + which, m0, a.M, k0, a.K);
        pn.load(a.b + (TURNS ? 0 : which), n0, a.N, k0, a.K);
    };
    if (step < end) load(step);
    for (; step < end; ++step) {
        __syncthreads();
        pm.store(lds_m);
        pn.store(lds_n);
        __syncthreads();
        if (step + 1 < end) load(step + 1);
#pragma unroll
        for (int kk = 0; kk < BK / 32; ++kk) {
            short8 fm[FM][P];
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int p = 0; p < P; ++p) fm[i][p] = fragment<LM, BM, BK>(lds_m + p * BM * BK / 8, wm + 16 * i, kk, lane);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                short8 fn[P];
#pragma unroll
                for (int p = 0; p < P; ++p) fn[p] = fragment<LN, BN, BK>(lds_n + p * BN * BK / 8, wn + 16 * j, kk, lane);
                if constexpr (P == 3) {
#pragma unroll
                    for (int order = 2; order >= 0; --order) // terms of order 2, 1, 0: the sum of the two planes' numbers
#pragma unroll
                        for (int p = 0; p <= order; ++p)
#pragma unroll
                            for (int i = 0; i < FM; ++i) acc[i][j] = mfma<T>(fn[p], fm[i][order - p], acc[i][j]);
                } else {
#pragma unroll
                    for (int i = 0; i < FM; ++i) acc[i][j] = mfma<T>(fn[0], fm[i][0], acc[i][j]);
                }
            }
        }
    }

    // lane l holds columns 4 (l / 16) .. + 3 of row l % 16 of every 16 x 16 results
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int64_t row = m0 + wm + 16 * i + lane % 16;
        if (row >= a.M) continue;
#pragma unroll
        for (int j = 0; j < FN; j += TURNS ? 2 : 1) {
            const int64_t col = n0 + (TURNS ? wn / 2 + 8 * j : wn + 16 * j) + 4 * (lane / 16);
            const int left = a.N - col < 4 ? (int)(a.N - col) : 4;
            if (left <= 0) continue;
            float s[4], s2[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                s[r] = acc[i][j][r];
                s2[r] = acc[i][TURNS ? j + 1 : j][r];
            }
            if constexpr (SPLIT) {
                char *to = reinterpret_cast<char *>(a.partial + ((int64_t)set * a.splits + split) * a.M * a.N);
                store4<float>(to, row * a.N + col, left, s);
            } else {
                finish4<T, EPI>(a, set, row, col, left, s, s2);
            }
        }
    }
}

// The sums of all parts of k, added in order in fp64; four columns a thread.  GATED: the parts of the second product are those of set 1.
template <class T, int EPI> __global__ __launch_bounds__(256) void product_join_kernel(const ProductArgs a)
{
    const int64_t per_row = (a.N + 3) / 4, at = (a.first + blockIdx.x) * 256 + threadIdx.x;
    const int64_t each = per_row * a.M;
    const int sets = EPI == EPI_STORE ? a.sets : 1;
    if (at >= each * sets) return;
    const int set = (int)(at / each);
    const int64_t row = (at - set * each) / per_row, col = (at - set * each) % per_row * 4;
    const int left = a.N - col < 4 ? (int)(a.N - col) : 4;
    double sum[2][4] = {};
    for (int q = 0; q < (EPI == EPI_GATED ? 2 : 1); ++q) {
        const char *part = reinterpret_cast<const char *>(a.partial + (int64_t)(set + q) * a.splits * a.M * a.N);
        for (int i = 0; i < a.splits; ++i) {
            float v[4];
            load4<float>(part, ((int64_t)i * a.M + row) * a.N + col, left, v);
#pragma unroll
            for (int r = 0; r < 4; ++r) sum[q][r] += (double)v[r];
        }
    }
    float s[2][4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        s[0][r] = (float)sum[0][r];
        s[1][r] = (float)sum[1][r];
    }
    finish4<T, EPI>(a, set, row, col, left, s[0], s[1]);
}

template <class T, int LM, int LN, int EPI, int TILE, bool SPLIT> int launch_tile(ProductArgs &a, hipStream_t stream)
{
    constexpr int BM = TILE_M[TILE], BN = TILE_N[TILE], WM = TILE == 2 ? 1 : 2, WN = TILE == 2 ? 4 : 2;
    constexpr int COLS = EPI == EPI_GATED ? BN / 2 : BN;
    const int64_t blocks = (a.M + BM - 1) / BM * ((a.N + COLS - 1) / COLS) * a.splits * a.sets;
    return launch_parts(blocks, [&](unsigned first, unsigned count) {
        a.first = first;
        product_kernel<T, LM, LN, EPI, BM, BN, WM, WN, SPLIT><<<count, 64 * WM * WN, 0, stream>>>(a);
    });
}

} // namespace
} // namespace slicegcn
