// Products of rows and weights on the matrix cores: what the kernels take, shared by the host code and the kernels of each type.
//
// Every product is C[M, N] = sum over k of A[m, k] B[n, k], with either operand stored k first (its rows lie along k: KC) or outer index first
// (OC):           M side           N side
//   X W           X, KC            W, OC
//   dP W^T        dP, KC           W, KC
//   X^T dP        X, OC            dP, OC
#pragma once

#include "common.h"
#include "values.h"

namespace slicegcn {

constexpr int LAYOUT_KC = 0, LAYOUT_OC = 1;

struct Operand {
    const char *p;
    int64_t ld;
    int32_t padded; // host: rows end with zeros up to whole units of 8 elements, which ld has room for
};

// What becomes of the sums
//   FORWARD  Y = residual R + act(P), P = sum + b
//   GATED    H = act(G) U of two products with the same rows, which take turns of 16 columns in a tile
//   STORE    the sum itself
constexpr int EPI_FORWARD = 0, EPI_GATED = 1, EPI_STORE = 2;

struct ProductArgs {
    Operand a[2], b[2];    // operands of each set of products that the grid's depth counts, or of each segment of a sum
    int64_t M, K;          // K of one segment
    int32_t N;
    int32_t segments;      // products that add up to one result (with `sets` = 1)
    int32_t sets;          // results formed by one launch; GATED: 1
    char *out[2];          // STORE: a result per set;  FORWARD: Y;  GATED: H
    int64_t ldo[2];
    const float *bias[2];
    Operand r;             // FORWARD: the residual rows
    char *keep[2];         // FORWARD: P;  GATED: G and U
    int64_t ldk[2];
    float residual;
    int32_t act;
    float *partial;        // sums of parts of k: [set][split][M][N], where splits > 1
    int32_t splits;
    int32_t steps_per_split;
    int32_t terms;         // 2, products of a pair alone: an operand is the sum of two, of which the second lies rest_a or rest_b bytes behind; its parts come behind the others
    int64_t rest_a, rest_b;
    int32_t tail;          // BY_TILES: how many of the last tiles are formed by themselves, cut along k: [part][tile][DIRECT_TILE][DIRECT_TILE]
    int64_t first;         // first workgroup of this launch
    int32_t shares;        // threads that share the parts of a result out where they are joined
    int32_t on_words;      // whether buffers can read the operands as they lie: product_kernels.h
};

// Sizes of a product and how it is cut: everything that a launch depends on follows from these
struct ProductShape {
    int64_t M, K;
    int32_t N;
    int32_t segments, sets, type;
    bool gated;   // GATED
    bool by_rows; // rows of the M side lie along k
};
constexpr int BY_REGISTERS = 0, BY_TILES = 1, BY_ROWS = 2; // product_kernels.h, product_direct.h, product_rows.h
constexpr int ALL = 0, SUMS_ALONE = 1, JOIN_ALONE = 2;     // of a product that is cut: sums of parts and their join, either by itself
struct ProductPlan {
    int32_t kernel;
    int32_t stage;
    int32_t tile; // BY_REGISTERS: index of a tile shape
    int32_t splits, steps_per_split;
    int32_t tail, tail_splits; // BY_TILES, splits = 1: the last tiles, and in how many parts of steps_per_split they are cut
    size_t bytes; // of the sums of parts of k
};
ProductPlan plan_product(const ProductShape &s, bool aligned);

// product_f32.hip, product_bf16.hip, product_f16.hip
int launch_product_f32(int layouts, int epilogue, const ProductPlan &plan, ProductArgs &a, hipStream_t stream);
int launch_product_bf16(int layouts, int epilogue, const ProductPlan &plan, ProductArgs &a, hipStream_t stream);
int launch_product_f16(int layouts, int epilogue, const ProductPlan &plan, ProductArgs &a, hipStream_t stream);

// Column sums of parts of the rows, [part][q][w] in fp64, on their way into fp32 gradients of one or two biases
struct BiasSums {
    const double *partial; // NULL: none are wanted
    int32_t parts, q, w;
    float *db[2];
};
constexpr int BIAS_COLS = 16; // columns of a workgroup
inline int64_t bias_workgroups(const BiasSums &b) { return b.partial ? (int64_t)((b.w + BIAS_COLS - 1) / BIAS_COLS) * b.q : 0; }

// 16 columns of one bias; the threads of a column share the parts out, and their sums are added in order.  sums: THREADS + THREADS / 16 of them
template <int THREADS> __device__ inline void bias_sums(const BiasSums &b, unsigned block, double *sums)
{
    constexpr int SHARES = THREADS / BIAS_COLS;
    const int lane = threadIdx.x % BIAS_COLS, share = threadIdx.x / BIAS_COLS, q = (int)(block % b.q);
    const int64_t col = (int64_t)(block / b.q) * BIAS_COLS + lane;
    double t = 0.0;
    if (col < b.w) {
#pragma unroll 4
        for (int32_t p = share; p < b.parts; p += SHARES) t += b.partial[((int64_t)p * b.q + q) * b.w + col];
    }
    sums[share * (BIAS_COLS + 1) + lane] = t;
    __syncthreads();
    if (share != 0 || col >= b.w || !b.db[q]) return;
    for (int s = 1; s < SHARES; ++s) t += sums[s * (BIAS_COLS + 1) + lane];
    b.db[q][col] = (float)t;
}

// Backward passes of which both products take one launch: tiles of 64 x 64 through registers
constexpr int PAIR_TILE = 64;
int launch_pair_f32(ProductArgs *x, ProductArgs *w, const BiasSums &bias, hipStream_t stream);
int launch_pair_bf16(ProductArgs *x, ProductArgs *w, const BiasSums &bias, hipStream_t stream);
int launch_pair_f16(ProductArgs *x, ProductArgs *w, const BiasSums &bias, hipStream_t stream);

// product_narrow.h: a backward pass in one sweep over the rows
constexpr int NARROW_WIDTH_IN = 128, NARROW_WIDTH_OUT = 256; // at most; of all products together
constexpr int NARROW_ROWS = 32;                              // of a block
constexpr int NARROW_RUN = 32;                               // blocks of rows whose column sums a thread adds in fp32
struct NarrowArgs {
    Operand x, w[2], g, u, d; // as in a backward pass
    char *dx;                 // NULL: not wanted
    int64_t lddx, n;
    int32_t w_in, w_out, want_w;
    float *partial;  // sums of dW: [set][workgroup][w_in][w_out]
    double *columns; // NULL, or column sums [workgroup][1 or 2][w_out]
};
int launch_narrow_bf16(const NarrowArgs &a, ProductArgs &join, int act, bool gated, unsigned blocks, hipStream_t stream);
int launch_narrow_f16(const NarrowArgs &a, ProductArgs &join, int act, bool gated, unsigned blocks, hipStream_t stream);

// layouts: which operands a product has
constexpr int PRODUCT_XW = 0, PRODUCT_GWT = 1, PRODUCT_XTG = 2;

constexpr int TILES = 3;
constexpr int TILE_M[TILES] = {128, 64, 32}, TILE_N[TILES] = {128, 64, 128};
constexpr int DIRECT_TILE = 256, DIRECT_K = 32;
constexpr int ROWS_MOST = 32;
constexpr int STEP_K_F32 = 32, STEP_K_16 = 64;
inline int step_k(int32_t type) { return type == SLICEGCN_F32 ? STEP_K_F32 : STEP_K_16; }

// Activations of v and their derivatives in some 5 (silu) and 20 (gelu) instructions, within a few 2^-24 of |v| and of 1 + |v|.
__device__ inline float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.4426950408889634f)); }

// The normal distribution Phi(v), and e = exp(-v^2 / 2).  The tail Phi(-|v|) is e times half of erfcx(|v| / sqrt 2), which is a polynomial of t = 1 / (1 + 0.265 |v|)
// without constant term: degree 9, fitted for the least relative error over |v| <= 14 (1.2e-8, and with all constants in fp32, as here, 7.6e-8: 1.3 2^-24).  With erfcf and expf, some 100 instructions, the gradients before a gelu
// were bound by them: 2.4 M rows of 256 bf16 columns 1.22 ms.
__device__ inline float normal_distribution(float v, float &e)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.265f, fabsf(v), 1.f));
    e = __builtin_amdgcn_exp2f(v * v * -0.72134752044448170f);
    float q = 0.030821435153484344f;
    q = fmaf(q, t, -0.1442311853170395f);
    q = fmaf(q, t, 0.21781975030899048f);
    q = fmaf(q, t, -0.11636755615472794f);
    q = fmaf(q, t, 0.1379561871290207f);
    q = fmaf(q, t, 0.060311924666166306f);
    q = fmaf(q, t, 0.10270125418901443f);
    q = fmaf(q, t, 0.10524662584066391f);
    q = fmaf(q, t, 0.10574156790971756f);
    const float tail = q * t * e;
    return v < 0.f ? tail : 1.f - tail;
}

template <int ACT> __device__ inline float activated(float v)
{
    float e;
    if (ACT == SLICEGCN_ACT_RELU) return v < 0.f ? 0.f : v;
    if (ACT == SLICEGCN_ACT_SILU) return v * sigmoid(v);
    if (ACT == SLICEGCN_ACT_GELU) return v * normal_distribution(v, e);
    return v;
}
__device__ inline float activated(int act, float v)
{
    switch (act) {
    case SLICEGCN_ACT_RELU: return activated<SLICEGCN_ACT_RELU>(v);
    case SLICEGCN_ACT_SILU: return activated<SLICEGCN_ACT_SILU>(v);
    case SLICEGCN_ACT_GELU: return activated<SLICEGCN_ACT_GELU>(v);
    default: return v;
    }
}

// act(v) and its derivative
template <int ACT> __device__ inline void activated_slope(float v, float &y, float &slope)
{
    if (ACT == SLICEGCN_ACT_RELU) {
        y = v < 0.f ? 0.f : v;
        slope = v > 0.f ? 1.f : 0.f;
    } else if (ACT == SLICEGCN_ACT_SILU) {
        const float s = sigmoid(v);
        y = v * s;
        slope = s * fmaf(v, 1.f - s, 1.f);
    } else if (ACT == SLICEGCN_ACT_GELU) {
        float e;
        const float p = normal_distribution(v, e);
        y = v * p;
        slope = fmaf(v * 0.39894228040143268f, e, p);
    } else {
        y = v;
        slope = 1.f;
    }
}

// d act'(v).  Where a relu is flat, whatever d is
template <int ACT> __device__ inline float through_slope(float d, float v, float slope)
{
    return ACT == SLICEGCN_ACT_RELU ? (v > 0.f ? d : 0.f) : d * slope;
}

// f(std::integral_constant) with the activation as a constant
template <class F> inline auto with_act(int act, F f)
{
    switch (act) {
    case SLICEGCN_ACT_RELU: return f(std::integral_constant<int, SLICEGCN_ACT_RELU>());
    case SLICEGCN_ACT_SILU: return f(std::integral_constant<int, SLICEGCN_ACT_SILU>());
    case SLICEGCN_ACT_GELU: return f(std::integral_constant<int, SLICEGCN_ACT_GELU>());
    default: return f(std::integral_constant<int, SLICEGCN_ACT_NONE>());
    }
}

} // namespace slicegcn
