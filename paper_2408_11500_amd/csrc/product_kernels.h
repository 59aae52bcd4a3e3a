// The kernels of product.h for one element type (each type is compiled by a file of its own).
//
// A workgroup forms a tile of BM x BN results.  Per step of k both operands' pieces go through registers into LDS as 16-bit values, and from there into the
// operand registers of v_mfma_f32_16x16x32: the N side is the instruction's first operand, so that a lane ends up with four consecutive columns of
// a row.  Pieces stay in the order of memory: those with k first are read 16 bytes (8 k of a row) at a time, the others with the
// transposing read ds_read_b64_tr_b16, of which 16 lanes together take 4 k of 16 columns and get 4 k of a column each.
// fp32 operands are split into three bf16 terms each, x = x0 + x1 + x2, every term the rest rounded to 8 bits: |x1| <= 2^-8 |x|, |x2| <= 2^-16 |x|, and what
// is left is at most 2^-24 |x|.  Six products are added, smallest first; the three that are left out are below 2^-23 of the product together.  Six bf16
// instructions take 96 cycles for what the fp32 instruction takes 256 for.  fp32, 233 k rows 602 -> 256 with gelu: 447 us, 161 TFLOP/s (a library's product of 8192^3 reaches 154);
// bound by the matrix instructions (53 % of the time), the reads of LDS and the splitting, which three workgroups a CU overlap in part, and by the stores of results.
#pragma once

#include "product.h"

namespace slicegcn {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short short8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));

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
template <int R> __device__ inline int line_turn(int k)
{
    if constexpr (R >= 128) return (k & 3) | ((k >> 3) & 1) << 2;
    return ((k & 3) ^ ((k >> 3) & 1)) & (R / 16 - 1); // lines shorter than the banks: two or four of them side by side
}
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

// A tile's rows of a matrix as a buffer: what a lane reads or writes of them is four columns at its own offset plus a scalar one per 16 x 16 results, and rows behind the
// last one are neither read nor written.
constexpr uint32_t NOT_THERE = 0xffffff00u; // beyond any buffer
template <class T> struct TileRows {
    __amdgpu_buffer_rsrc_t rsrc;
    uint32_t offset, line; // bytes

    __device__ TileRows(const char *p, int64_t ld, int64_t m0, int64_t n0, int64_t rows, int32_t cols, int row, int col)
    {
        line = (uint32_t)ld * sizeof(T);
        const uint32_t bytes = (uint32_t)(rows - 1) * line + (uint32_t)cols * sizeof(T);
        rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p + (m0 * ld + n0) * (int64_t)sizeof(T)), 0, (int)bytes, 0x00020000);
        offset = (uint32_t)row * line + (uint32_t)col * sizeof(T);
    }
    // `there`: columns that the lane has there, of four.  TAIL: it may be one to three of them
    template <bool TAIL> __device__ void load(int i, int col, int there, float (&v)[4]) const
    {
        const int at = (int)(there >= 4 ? offset : NOT_THERE), scalar = (int)(16 * i * line + col * sizeof(T));
        if constexpr (sizeof(T) == 4) {
            const uint4v x = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at, scalar, 0);
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = __uint_as_float(x[r]);
        } else {
            typedef T T4 __attribute__((ext_vector_type(4)));
            const T4 x = __builtin_bit_cast(T4, __builtin_amdgcn_raw_buffer_load_b64(rsrc, at, scalar, 0));
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = (float)x[r];
        }
        if constexpr (TAIL) {
#pragma unroll
            for (int r = 0; r < 3; ++r) {
                const int one = (int)(there < 4 && r < there ? offset + r * sizeof(T) : NOT_THERE);
                float x;
                if constexpr (sizeof(T) == 4) x = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rsrc, one, scalar, 0));
                else x = (float)__builtin_bit_cast(T, (short)__builtin_amdgcn_raw_buffer_load_b16(rsrc, one, scalar, 0));
                v[r] = there < 4 ? x : v[r];
            }
        }
    }
    template <bool TAIL> __device__ void store(int i, int col, int there, const float (&v)[4]) const
    {
        const int at = (int)(there >= 4 ? offset : NOT_THERE), scalar = (int)(16 * i * line + col * sizeof(T));
        typedef T T4 __attribute__((ext_vector_type(4)));
        T4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = (T)v[r];
        // 16 bytes without a scalar offset: with one in a register the compiler lets the next instruction overwrite the stored registers, and the fourth of them has then
        // been read too late in the last lanes of each row of 16 now and then
        if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4v, x), rsrc, there >= 4 ? at + scalar : at, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(uint2v, x), rsrc, at, scalar, 0);
        if constexpr (TAIL) {
#pragma unroll
            for (int r = 0; r < 3; ++r) {
                const int one = (int)(there < 4 && r < there ? offset + r * sizeof(T) : NOT_THERE);
                if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v[r]), rsrc, one, scalar, 0);
                else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (T)v[r]), rsrc, one, scalar, 0);
            }
        }
    }
};

// A wavefront's sums into results, as finish4 forms them.  Lane l holds columns 4 (l / 16) .. + 3 of row l % 16 of every 16 x 16 results, which begin at row wm and column wn of
// the tile; GATED: acc[.][j] and acc[.][j + 1] are both products of the same columns.  Stores have a scalar address each, and the parts of a row follow one another, so that
// lines are whole when they leave the L2.  TAIL: the last tile of columns where N is no multiple of 4.
template <class T, int EPI, bool SPLIT, bool TAIL, int ACT, int BM, int FM, int FN>
__device__ inline void finish_with(const ProductArgs &a, int set, int split, int64_t m0, int64_t n0, int wm, int wn, const float4v (&acc)[FM][FN])
{
    constexpr bool TURNS = EPI == EPI_GATED;
    constexpr int J = TURNS ? 2 : 1, W = TURNS ? 8 : 16;
    const int lane = threadIdx.x % 64, row = wm + lane % 16, col = (TURNS ? wn / 2 : wn) + 4 * (lane / 16);
    const int64_t rows = a.M - m0 < BM ? a.M - m0 : BM;
    const int32_t cols = a.N - (int32_t)n0;
    auto sums = [&](int i, int j, float (&s)[4]) {
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = acc[i][j][r];
    };
    if constexpr (SPLIT) {
        const TileRows<float> to(reinterpret_cast<const char *>(a.partial + ((int64_t)set * a.splits + split) * a.M * a.N), a.N, m0, n0, rows, cols, row, col);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                float s[4];
                sums(i, j, s);
                to.template store<TAIL>(i, W * j, cols - (col + W * j), s);
            }
    } else if constexpr (EPI == EPI_STORE) {
        const TileRows<T> to(a.out[set], a.ldo[set], m0, n0, rows, cols, row, col);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                float s[4];
                sums(i, j, s);
                to.template store<TAIL>(i, W * j, cols - (col + W * j), s);
            }
    } else {
        const TileRows<T> to(a.out[0], a.ldo[0], m0, n0, rows, cols, row, col), k0(a.keep[0], a.ldk[0], m0, n0, rows, cols, row, col);
        const TileRows<T> other(TURNS ? a.keep[1] : a.r.p, TURNS ? a.ldk[1] : a.r.ld, m0, n0, rows, cols, row, col);
        float bias[FN][4];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const int at = col + W * (TURNS ? j - j % 2 : j);
            load_bias(a.bias[TURNS ? j % 2 : 0], n0 + at, cols - at, bias[j]);
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) {
#pragma unroll
            for (int j = 0; j < FN; j += J) {
                const int there = cols - (col + W * j);
                float s[4], y[4];
                sums(i, j, s);
#pragma unroll
                for (int r = 0; r < 4; ++r) s[r] += bias[j][r];
                if (a.keep[0]) k0.template store<TAIL>(i, W * j, there, s);
                if constexpr (TURNS) {
                    float u[4];
                    sums(i, j + 1, u);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        u[r] += bias[j + 1][r];
                        y[r] = activated<ACT>(s[r]) * u[r];
                    }
                    if (a.keep[0]) other.template store<TAIL>(i, W * j, there, u);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) y[r] = activated<ACT>(s[r]);
                    if (a.r.p) {
                        float v[4];
                        other.template load<TAIL>(i, W * j, there, v);
#pragma unroll
                        for (int r = 0; r < 4; ++r) y[r] = fmaf(a.residual, v[r], y[r]);
                    }
                }
                to.template store<TAIL>(i, W * j, there, y);
            }
        }
    }
}

template <class T, int EPI, bool SPLIT, int BM, int FM, int FN>
__device__ inline void finish_tile(const ProductArgs &a, int set, int split, int64_t m0, int64_t n0, int wm, int wn, int tile_cols, const float4v (&acc)[FM][FN])
{
    const bool tail = a.N % 4 != 0 && n0 + tile_cols > a.N;
    auto with = [&](auto act) {
        constexpr int ACT = decltype(act)::value;
        if (tail) finish_with<T, EPI, SPLIT, true, ACT, BM>(a, set, split, m0, n0, wm, wn, acc);
        else finish_with<T, EPI, SPLIT, false, ACT, BM>(a, set, split, m0, n0, wm, wn, acc);
    };
    if (SPLIT || EPI == EPI_STORE) {
        with(std::integral_constant<int, SLICEGCN_ACT_NONE>());
        return;
    }
    switch (a.act) {
    case SLICEGCN_ACT_RELU: with(std::integral_constant<int, SLICEGCN_ACT_RELU>()); break;
    case SLICEGCN_ACT_SILU: with(std::integral_constant<int, SLICEGCN_ACT_SILU>()); break;
    case SLICEGCN_ACT_GELU: with(std::integral_constant<int, SLICEGCN_ACT_GELU>()); break;
    default: with(std::integral_constant<int, SLICEGCN_ACT_NONE>());
    }
}

// The sums of all parts of k, in fp64: four columns a thread, and a.shares threads of a workgroup share the parts out (part s, s + shares, ... each), whose sums
// are added in order.  GATED: the parts of the second product are those of set 1.  256 parts of 100 x 256 with one share 84 us.
template <int EPI> constexpr int JOIN_SUMS = (EPI == EPI_GATED ? 2 : 1) * 4 + 1;
template <class T, int EPI> __device__ inline void join_parts(const ProductArgs &a, int64_t block, double *sums)
{
    constexpr int Q = EPI == EPI_GATED ? 2 : 1, EACH = JOIN_SUMS<EPI>;
    const int here = 256 / a.shares, share = threadIdx.x / here;
    const int64_t per_row = (a.N + 3) / 4, each = per_row * a.M, at = block * here + threadIdx.x % here;
    const bool there = at < each * (EPI == EPI_STORE ? a.sets : 1);
    const int set = there ? (int)(at / each) : 0;
    const int64_t row = there ? (at - set * each) / per_row : 0, col = there ? (at - set * each) % per_row * 4 : 0;
    const int left = a.N - col < 4 ? (int)(a.N - col) : 4;
    double sum[Q][4] = {};
    if (there)
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const char *part = reinterpret_cast<const char *>(a.partial + (int64_t)(set + q) * a.splits * a.M * a.N);
#pragma unroll 4
            for (int i = share; i < a.splits; i += a.shares) {
                float v[4];
                load4<float>(part, ((int64_t)i * a.M + row) * a.N + col, left, v);
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[q][r] += (double)v[r];
            }
        }
    if (a.shares > 1) {
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int r = 0; r < 4; ++r) sums[threadIdx.x * EACH + q * 4 + r] = sum[q][r];
        __syncthreads();
        if (share > 0) return;
        for (int i = 1; i < a.shares; ++i)
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int r = 0; r < 4; ++r) sum[q][r] += sums[(i * here + threadIdx.x) * EACH + q * 4 + r];
    }
    if (!there) return;
    float s[2][4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        s[0][r] = (float)sum[0][r];
        s[1][r] = (float)sum[Q - 1][r];
    }
    finish4<T, EPI>(a, set, row, col, left, s[0], s[1]);
}

template <class T, int EPI> __global__ __launch_bounds__(256) void product_join_kernel(const ProductArgs a)
{
    __shared__ double sums[256 * JOIN_SUMS<EPI>];
    join_parts<T, EPI>(a, a.first + blockIdx.x, sums);
}

// How many threads share the parts out: about four parts each
inline int join_shares(ProductArgs &a)
{
    a.shares = 1;
    while (a.shares < 32 && a.shares * 4 <= a.splits) a.shares *= 2;
    return a.shares;
}

template <class T, int EPI> int launch_join(ProductArgs &a, hipStream_t stream)
{
    const int64_t here = 256 / join_shares(a), threads = (a.N + 3) / 4 * a.M * (EPI == EPI_STORE ? a.sets : 1);
    return launch_parts((threads + here - 1) / here, [&](unsigned first, unsigned count) {
        a.first = first;
        product_join_kernel<T, EPI><<<count, 256, 0, stream>>>(a);
    });
}

// A piece of an operand (R outer indexes, BK of k) on its way from memory to LDS, 8 elements a unit.  It is read through a buffer whose range check takes care of rows, lines
// and columns behind the last one, so that the loads of a step depend on no lane's branch and two steps can be in flight.  KC: the buffer of the tile's rows, of which a step
// reads from its scalar offset on; OC: the buffer of the step's lines.
// The range check goes by words.  ODD: 16-bit elements of which a word may hold one that exists and one that does not, or whose rows begin within a word: a unit is read as
// the five words that it lies in (a word with an element of the operand can be read whole) and shifted into place on its way to LDS, where elements that are not there turn
// into zeros.  (2000 rows 4001 -> 557 bf16: 58 us, with
// loads that branch by the lane 139; 2000 rows 1001 -> 1203 forward 26 and 37, backward 63 and 121.)
template <class T, int LAYOUT, int R, int BK, int THREADS, bool ODD> struct BufferPiece {
    static constexpr int UNITS = R * BK / 8, EACH = (UNITS + THREADS - 1) / THREADS, V = sizeof(T) / 2; // accesses of 16 bytes a unit
    static_assert(!ODD || V == 1, "elements of 16 bits");
    static constexpr uint32_t NOWHERE = 0xffffff00u;
    uint32_t offset[EACH];
    uint64_t base;
    uint32_t line, size; // bytes: of a line; KC: of the buffer, OC: of a line's part
    struct Regs {
        uint4v v[EACH][V];
        uint32_t more[ODD ? EACH : 1];
    };

    __device__ static int unit(int i) { return (int)threadIdx.x + i * THREADS; }
    __device__ static int unit_k(int i) { return unit(i) % (BK / 8) * 8; } // KC

    __device__ void aim(const Operand &op, int64_t o0, int64_t outer, int32_t K)
    {
        line = (uint32_t)op.ld * sizeof(T);
        const int64_t here = outer - o0 < R ? outer - o0 : R;
        base = (uint64_t)op.p + (LAYOUT == LAYOUT_KC ? (uint64_t)o0 * line : (uint64_t)o0 * sizeof(T));
        size = LAYOUT == LAYOUT_KC ? (uint32_t)(here - 1) * line + (uint32_t)K * sizeof(T) : (uint32_t)here * sizeof(T);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int q = unit(i);
            offset[i] = LAYOUT == LAYOUT_KC ? (uint32_t)(q / (BK / 8)) * line + unit_k(i) * sizeof(T)
                                            : (uint32_t)(q / (R / 8)) * line + (uint32_t)(q % (R / 8)) * 8 * sizeof(T);
            if (UNITS % THREADS != 0 && q >= UNITS) offset[i] = NOWHERE;
            // OC: a unit that begins behind the last column would read the next line's first ones
            if (LAYOUT == LAYOUT_OC && (q % (R / 8)) * 8 >= here) offset[i] = NOWHERE;
        }
    }

    // The step from k0 on; zeros where it is not there
    __device__ void load(Regs &r, int32_t k0, int32_t K, bool there) const
    {
        uint32_t bytes = size, scalar = 0;
        uint64_t from = base;
        if (LAYOUT == LAYOUT_KC) {
            scalar = (uint32_t)k0 * sizeof(T);
        } else {
            const int32_t lines = K - k0 < BK ? K - k0 : BK;
            from += (uint64_t)(uint32_t)k0 * line;
            bytes += (uint32_t)(lines - 1) * line;
        }
        const uint32_t within = ODD ? (uint32_t)from & 2u : 0u; // steps are whole words apart
        if (ODD) bytes = (bytes + within + 3u) & ~3u;
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void *>(from - within), 0, there ? (int)bytes : 0, 0x00020000);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const uint32_t at = ODD ? (offset[i] + within) & ~3u : offset[i];
#pragma unroll
            for (int v = 0; v < V; ++v) r.v[i][v] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(at + 16 * v), (int)scalar, 0);
            if (ODD) r.more[i] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, (int)(at + 16), (int)scalar, 0);
        }
    }

    // left: k that exist from the step's first one on (KC: what follows in the buffer is the next row).  from: what base was for the step
    __device__ void store(const Regs &r, short8 *lds, int32_t left, uint64_t from) const
    {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int q = unit(i);
            if (UNITS % THREADS != 0 && q >= UNITS) break;
            T v[8];
            if constexpr (ODD) {
                const uint32_t by = (offset[i] + (uint32_t)from) & 2u; // bytes into its first word
                const uint32_t w[5] = {r.v[i][0][0], r.v[i][0][1], r.v[i][0][2], r.v[i][0][3], r.more[i]};
                uint32_t x[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_alignbyte(w[j + 1], w[j], by);
                __builtin_memcpy(v, x, sizeof(v));
            } else {
                __builtin_memcpy(v, r.v[i], sizeof(v));
            }
            if (LAYOUT == LAYOUT_KC && left < BK) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = unit_k(i) + j < left ? v[j] : (T)0.f;
            }
            if (ODD && LAYOUT == LAYOUT_OC && left < BK) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = q / (R / 8) < left ? v[j] : (T)0.f;
            }
            const int at = LAYOUT == LAYOUT_KC ? lds_unit<LAYOUT, R, BK>(q / (BK / 8), q % (BK / 8)) : lds_unit<LAYOUT, R, BK>(q % (R / 8), q / (R / 8));
            short8 t[Planes<T>::count];
            split8(v, t);
#pragma unroll
            for (int p = 0; p < Planes<T>::count; ++p) lds[p * UNITS + at] = t[p];
        }
    }
};

// LDS of product_buffer_tile, in units
template <class T, int BM, int BN> constexpr int buffer_units = Planes<T>::count * (BM + BN) * (sizeof(T) == 4 ? STEP_K_F32 : STEP_K_16) / 8;

// A tile of results of such operands, by workgroup `block` of a product: SETS steps on their way in registers, one in LDS.  (fp32: with two on their way 233 k rows 602 -> 256
// take 500 us, with one 452; with three workgroups a CU instead of two 484.)
template <class T, int LM, int LN, int EPI, int BM, int BN, int WM, int WN, bool SPLIT, bool ODD>
__device__ inline void product_buffer_tile(const ProductArgs &a, int64_t block, short8 *lds)
{
    constexpr int SETS = sizeof(T) == 4 ? 1 : 2;
    constexpr int P = Planes<T>::count, BK = P == 3 ? STEP_K_F32 : STEP_K_16, THREADS = 64 * WM * WN;
    constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr bool TURNS = EPI == EPI_GATED, SEGMENTS = LM == LAYOUT_KC && LN == LAYOUT_KC;
    constexpr int PIECES = TURNS ? 2 : 1, COLS = BN / PIECES; // columns of results; GATED: a piece of each product
    static_assert(!TURNS || FN % 2 == 0, "a wavefront holds both products of its columns");
    typedef BufferPiece<T, LM, BM, BK, THREADS, ODD> PieceM;
    typedef BufferPiece<T, LN, COLS, BK, THREADS, ODD> PieceN;
    static_assert(P * (PieceM::UNITS + PIECES * PieceN::UNITS) == buffer_units<T, BM, BN>, "LDS of a step");
    short8 *lds_m = lds, *lds_n = lds + P * PieceM::UNITS;

    const int64_t tile_rows = (a.M + BM - 1) / BM, tile_cols = (a.N + COLS - 1) / COLS, tiles = tile_rows * tile_cols;
    int64_t id = tile_of(block, tiles * a.splits * a.sets), row_tile, col_tile;
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

    const int32_t K = (int32_t)a.K, steps_each = (K + BK - 1) / BK, all = SEGMENTS ? steps_each * a.segments : steps_each;
    const bool rest = SPLIT && a.terms == 2 && split >= a.splits / 2;
    const int32_t begin = SPLIT ? (rest ? split - a.splits / 2 : split) * a.steps_per_split : 0;
    const int32_t end = SPLIT && begin + a.steps_per_split < all ? begin + a.steps_per_split : all;
    PieceM pm;
    PieceN pn[PIECES];
    pm.aim(a.a[set], m0, a.M, K);
#pragma unroll
    for (int q = 0; q < PIECES; ++q) pn[q].aim(a.b[TURNS ? q : set], n0, a.N, K);
    if (rest) {
        pm.base += a.rest_a;
        pn[0].base += a.rest_b;
    }
    // the second segment's operands have the leading dimensions of the first one's
    const uint64_t base_m = pm.base, base_n = pn[0].base, second_m = base_m + (uint64_t)(a.a[1].p - a.a[0].p), second_n = base_n + (uint64_t)(a.b[1].p - a.b[0].p);
    struct Step {
        typename PieceM::Regs m;
        typename PieceN::Regs n[PIECES];
    } regs[SETS];
    auto load = [&](Step &s, int32_t t) {
        int32_t k0 = t * BK;
        if (SEGMENTS) {
            const bool second = t >= steps_each;
            k0 -= second ? steps_each * BK : 0;
            pm.base = second ? second_m : base_m;
            pn[0].base = second ? second_n : base_n;
        }
        pm.load(s.m, k0, K, t < end);
#pragma unroll
        for (int q = 0; q < PIECES; ++q) pn[q].load(s.n[q], k0, K, t < end);
    };
    auto step = [&](Step &s, int32_t t) {
        const int32_t left = K - (SEGMENTS && t >= steps_each ? t - steps_each : t) * BK;
        __syncthreads();
        const bool second = SEGMENTS && t >= steps_each;
        pm.store(s.m, lds_m, left, second ? second_m : base_m);
#pragma unroll
        for (int q = 0; q < PIECES; ++q) pn[q].store(s.n[q], lds_n + q * P * PieceN::UNITS, left, q ? pn[q].base : second ? second_n : base_n);
        __syncthreads();
        load(s, t + SETS);
#pragma unroll
        for (int kk = 0; kk < BK / 32; ++kk) {
            short8 fm[FM][P];
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int p = 0; p < P; ++p) fm[i][p] = fragment<LM, BM, BK>(lds_m + p * PieceM::UNITS, wm + 16 * i, kk, lane);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                short8 fn[P];
                const int q = TURNS ? j % 2 : 0, base = TURNS ? wn / 2 + 8 * (j - j % 2) : wn + 16 * j;
#pragma unroll
                for (int p = 0; p < P; ++p) fn[p] = fragment<LN, COLS, BK>(lds_n + (q * P + p) * PieceN::UNITS, base, kk, lane);
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
    };
#pragma unroll
    for (int i = 0; i < SETS; ++i) load(regs[i], begin + i);
    for (int32_t t = begin; t < end; t += SETS) { // with two sets an odd number of steps ends with one of zeros
#pragma unroll
        for (int i = 0; i < SETS; ++i) step(regs[i], t + i);
    }

    finish_tile<T, EPI, SPLIT, BM>(a, set, split, m0, n0, wm, wn, COLS, acc);
}

// WM x WN wavefronts.  SPLIT: sums of a part of k go to a.partial.
template <class T, int LM, int LN, int EPI, int BM, int BN, int WM, int WN, bool SPLIT, bool ODD>
__global__ __launch_bounds__(64 * WM * WN, 2) void product_buffer_kernel(const ProductArgs a)
{
    __shared__ short8 lds[buffer_units<T, BM, BN>];
    product_buffer_tile<T, LM, LN, EPI, BM, BN, WM, WN, SPLIT, ODD>(a, a.first + blockIdx.x, lds);
}

// Both products of a backward pass in one launch, where they are short and launches would take longer than they: dX by the first workgroups, dW by the others, all as sums of
// parts of k.
template <class T, bool ODD> __global__ __launch_bounds__(256, 2) void product_pair_kernel(const ProductArgs x, const ProductArgs w, unsigned blocks_x)
{
    __shared__ short8 lds[buffer_units<T, PAIR_TILE, PAIR_TILE>];
    if (blockIdx.x < blocks_x) product_buffer_tile<T, LAYOUT_KC, LAYOUT_KC, EPI_STORE, PAIR_TILE, PAIR_TILE, 2, 2, true, ODD>(x, blockIdx.x, lds);
    else product_buffer_tile<T, LAYOUT_OC, LAYOUT_OC, EPI_STORE, PAIR_TILE, PAIR_TILE, 2, 2, true, ODD>(w, blockIdx.x - blocks_x, lds);
}

// What is left of it: the parts of dX and of dW joined, and the column sums' parts
template <class T>
__global__ __launch_bounds__(256) void product_pair_join_kernel(const ProductArgs x, const ProductArgs w, const BiasSums bias, unsigned blocks_x, unsigned blocks_w)
{
    __shared__ double sums[256 * JOIN_SUMS<EPI_STORE>];
    if (blockIdx.x < blocks_x) join_parts<T, EPI_STORE>(x, blockIdx.x, sums);
    else if (blockIdx.x < blocks_x + blocks_w) join_parts<T, EPI_STORE>(w, blockIdx.x - blocks_x, sums);
    else bias_sums<256>(bias, blockIdx.x - blocks_x - blocks_w, sums);
}

template <class T> int launch_pair(ProductArgs *x, ProductArgs *w, const BiasSums &bias, hipStream_t stream)
{
    auto tiles = [](const ProductArgs *a) {
        return a ? (a->M + PAIR_TILE - 1) / PAIR_TILE * ((a->N + PAIR_TILE - 1) / PAIR_TILE) * a->splits * a->sets : 0;
    };
    auto joins = [](ProductArgs *a) -> int64_t {
        if (!a) return 0;
        const int64_t here = 256 / join_shares(*a), threads = (a->N + 3) / 4 * a->M * a->sets;
        return (threads + here - 1) / here;
    };
    const ProductArgs none{};
    const int64_t x_tiles = tiles(x), w_tiles = tiles(w), x_joins = joins(x), w_joins = joins(w), bias_blocks = bias_workgroups(bias);
    if (x_tiles + w_tiles > 0) {
        const bool odd = (x && !x->on_words) || (w && !w->on_words);
        const dim3 grid((unsigned)(x_tiles + w_tiles));
        if constexpr (sizeof(T) == 2)
            if (odd) product_pair_kernel<T, true><<<grid, 256, 0, stream>>>(x ? *x : none, w ? *w : none, (unsigned)x_tiles);
        if (!odd) product_pair_kernel<T, false><<<grid, 256, 0, stream>>>(x ? *x : none, w ? *w : none, (unsigned)x_tiles);
        SG_LAUNCH_CHECK();
    }
    if (x_joins + w_joins + bias_blocks > 0) {
        product_pair_join_kernel<T><<<(unsigned)(x_joins + w_joins + bias_blocks), 256, 0, stream>>>(x ? *x : none, w ? *w : none, bias, (unsigned)x_joins,
                                                                                                     (unsigned)w_joins);
        SG_LAUNCH_CHECK();
    }
    return SLICEGCN_OK;
}

template <class T, int LM, int LN, int EPI, int TILE, bool SPLIT> int launch_tile(ProductArgs &a, hipStream_t stream)
{
    constexpr int BM = TILE_M[TILE], BN = TILE_N[TILE], WM = TILE == 2 ? 1 : 2, WN = TILE == 2 ? 4 : 2;
    constexpr int COLS = EPI == EPI_GATED ? BN / 2 : BN;
    const int64_t blocks = (a.M + BM - 1) / BM * ((a.N + COLS - 1) / COLS) * a.splits * a.sets;
    return launch_parts(blocks, [&](unsigned first, unsigned count) {
        a.first = first;
        if constexpr (sizeof(T) == 2)
            if (!a.on_words) {
                product_buffer_kernel<T, LM, LN, EPI, BM, BN, WM, WN, SPLIT, true><<<count, 64 * WM * WN, 0, stream>>>(a);
                return;
            }
        product_buffer_kernel<T, LM, LN, EPI, BM, BN, WM, WN, SPLIT, false><<<count, 64 * WM * WN, 0, stream>>>(a);
    });
}

} // namespace
} // namespace slicegcn
