// Norms before and after a block, fused with the block's gate and the residual, forward and backward.
//
//   p = post(y) * post_w + post_b;   h = residual * x + s * p;   u = pre(h) * pre_w + pre_b
//
// With yn, hn the normalised rows, ry, rh the factors 1 / sqrt(...) they were multiplied by, and means over a row's columns:
//   dun = du * pre_w;    dH = dh + rh * (dun - [mean dun] - hn * mean(dun * hn))          [..]: layer norm only
//   dx = residual * dH;  dgate = dH * p (times s (1 - s) through a sigmoid)
//   dyn = dH * s * post_w;  dy = ry * (dyn - [mean dyn] - yn * mean(dyn * yn))
//   dpre_w = sum du * hn;  dpre_b = sum du;  dpost_w = sum dH * s * yn;  dpost_b = sum dH * s     (sums over rows)
// A gate per column has dgate = post_w * sum dH * yn + post_b * sum dH, so that two sums per norm serve all parameters.
//
// A row lies in the registers of a group of lanes from its one read to its one write, and h is formed again in the backward pass instead of
// being read: bound by bytes.
#include "common.h"
#include "values.h"

#include <cmath>

namespace slicegcn {

namespace {

constexpr int NONE = SLICEGCN_NORM_NONE, LAYER = SLICEGCN_NORM_LAYER;
constexpr int FWD_ELEMS = 16;         // elements of a row per lane, at most
constexpr int BWD_ELEMS = 8;          // ... in the backward pass, which holds six of a row's operands and four sums; 16 on the widest rows
constexpr int BWD_WIDE = 1024 * BWD_ELEMS;
constexpr int SUM_COLS = 2048;        // widest row of which a workgroup holds several
constexpr int PLANES = 4;             // sums over rows: du * hn, du, dH * s * yn, dH * s (without s where the gate is per column)

struct RowPtr {
    char *data;
    int64_t ld;
};

struct Args {
    RowPtr x, y, gate, h, u, dh, du, dx, dy, dgate;
    float *stats;
    const float *post_w, *post_b, *pre_w, *pre_b, *gate_col;
    float *partial;
    int64_t n;
    int32_t width, lanes; // lanes of a row
    int32_t post, pre;
    float residual, eps, inv_width;
    bool sigmoid;
    uint32_t planes; // bit p: the sums of plane p are wanted
};

template <int V> struct Lane { // K accesses of V columns; the last access of a row that is no multiple of V wide is moved left
    int32_t col;
    int skip; // leading columns that the access before it holds too
    bool on;
};

template <class T, int V, int K, bool MULTI, bool FULL> struct Row {
    const Args &a;
    float *shared; // MULTI: [2][16][2]
    int lane, slot; // lane within the row, row within the workgroup
    int turn = 0;
    Lane<V> at[K];

    __device__ Row(const Args &args, float *sh) : a(args), shared(sh)
    {
        lane = threadIdx.x & (a.lanes - 1);
        slot = threadIdx.x / a.lanes;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int32_t c = (lane + k * a.lanes) * V;
            at[k].on = FULL || c < a.width;
            at[k].col = FULL ? c : min(c, a.width - V);
            at[k].skip = FULL ? 0 : c - at[k].col;
        }
    }

    // sums over the row's columns, in every lane; f(k, j) is the summand
    template <class F> __device__ float sum(F f)
    {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!at[k].on) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float v = f(k, j);
                s += FULL || j >= at[k].skip ? v : 0.f;
            }
        }
        return over_lanes(s);
    }

    __device__ float over_lanes(float s)
    {
        if (!MULTI) return group_sum(s, a.lanes);
        s = group_sum(s, 64);
        float *buf = shared + turn * 16; // written again two sums later, when every wavefront has read it
        turn ^= 1;
        const int wave = threadIdx.x / 64, waves = a.lanes / 64, first = slot * waves;
        if (threadIdx.x % 64 == 0) buf[wave] = s;
        __syncthreads();
        float total = 0.f;
        for (int w = 0; w < waves; ++w) total += buf[first + w];
        return total;
    }

    __device__ void load(const RowPtr &p, int64_t row, bool there, float (&v)[K][V]) const
    {
        const T *q = reinterpret_cast<const T *>(p.data) + row * p.ld;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (there && at[k].on) {
                const auto r = load_vec<T, V>(q + at[k].col);
#pragma unroll
                for (int j = 0; j < V; ++j) v[k][j] = (float)r[j];
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) v[k][j] = 0.f;
            }
        }
    }

    __device__ void store(const RowPtr &p, int64_t row, const float (&v)[K][V]) const
    {
        T *q = reinterpret_cast<T *>(p.data) + row * p.ld;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (at[k].on) store_vec<T, V>(q + at[k].col, v[k]);
    }

    // f(k, j, parameter) for the lane's columns
    template <class F> __device__ void with_param(const float *p, F f) const
    {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const auto w = load_vec<float, V>(p + at[k].col);
#pragma unroll
            for (int j = 0; j < V; ++j) f(k, j, (float)w[j]);
        }
    }

    template <class F> __device__ void each(F f) const
    {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) f(k, j);
    }

    // mean and 1 / sqrt(...) of a row
    __device__ void moments(const float (&v)[K][V], int kind, float *mean, float *factor)
    {
        *mean = kind == LAYER ? sum([&](int k, int j) { return v[k][j]; }) * a.inv_width : 0.f;
        const float m = *mean;
        const float var = sum([&](int k, int j) { const float d = v[k][j] - m; return d * d; }) * a.inv_width;
        *factor = 1.f / sqrtf(var + a.eps);
    }

    // g -> s, the factor of p
    __device__ void gate(int64_t row, bool there, float (&g)[K][V]) const
    {
        if (a.gate.data) load(a.gate, row, there, g);
        else with_param(a.gate_col, [&](int k, int j, float w) { g[k][j] = w; });
        if (a.sigmoid) each([&](int k, int j) { g[k][j] = 1.f / (1.f + expf(-g[k][j])); });
    }

    __device__ bool gated() const { return a.gate.data || a.gate_col; }

    // yn -> p
    __device__ void affine(const float (&v)[K][V], const float *w, const float *b, float (&o)[K][V]) const
    {
        each([&](int k, int j) { o[k][j] = v[k][j]; });
        if (w) with_param(w, [&](int k, int j, float p) { o[k][j] *= p; });
        if (b) with_param(b, [&](int k, int j, float p) { o[k][j] += p; });
    }
};

template <class T, int V, int K, bool MULTI, bool FULL, int THREADS>
__global__ __launch_bounds__(THREADS) void resnorm_fwd_kernel(const Args a)
{
    __shared__ float shared[MULTI ? 32 : 1];
    Row<T, V, K, MULTI, FULL> r(a, shared);
    const int rows = THREADS / a.lanes;
    for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < a.n; r0 += (int64_t)gridDim.x * rows) {
        const int64_t row = r0 + r.slot;
        const bool there = row < a.n;
        float h[K][V], y[K][V], g[K][V], st[4] = {0.f, 1.f, 0.f, 1.f};
        if (a.x.data) r.load(a.x, row, there, h);
        else r.each([&](int k, int j) { h[k][j] = 0.f; });
        if (a.y.data) r.load(a.y, row, there, y);
        if (r.gated()) r.gate(row, there, g);
        r.each([&](int k, int j) { h[k][j] *= a.residual; });
        if (a.y.data) {
            if (a.post != NONE) {
                r.moments(y, a.post, &st[0], &st[1]);
                r.each([&](int k, int j) { y[k][j] = (y[k][j] - st[0]) * st[1]; });
                r.affine(y, a.post_w, a.post_b, y);
            }
            if (r.gated()) r.each([&](int k, int j) { h[k][j] = fmaf(g[k][j], y[k][j], h[k][j]); });
            else r.each([&](int k, int j) { h[k][j] += y[k][j]; });
        }
        // rows in place: all of a row is read before any of it is written (a sum over the row sees to that too)
        if (MULTI && !FULL && !(a.y.data && a.post != NONE)) __syncthreads();
        if (a.h.data && there) r.store(a.h, row, h);
        if (a.u.data) {
            if (a.pre != NONE) {
                r.moments(h, a.pre, &st[2], &st[3]);
                r.each([&](int k, int j) { h[k][j] = (h[k][j] - st[2]) * st[3]; });
                r.affine(h, a.pre_w, a.pre_b, h);
            }
            if (there) r.store(a.u, row, h);
        }
        if (a.stats && there && r.lane == 0) *reinterpret_cast<float4 *>(a.stats + 4 * row) = make_float4(st[0], st[1], st[2], st[3]);
    }
}

template <class T, int V, int K, bool MULTI, bool FULL, int THREADS>
__global__ __launch_bounds__(THREADS) void resnorm_bwd_kernel(const Args a)
{
    __shared__ float shared[MULTI ? 32 : 1];
    __shared__ float sums[THREADS <= 256 ? SUM_COLS : 1];
    Row<T, V, K, MULTI, FULL> r(a, shared);
    const int rows = THREADS / a.lanes;
    const bool column_gate = a.gate_col != nullptr;
    float acc[PLANES][K][V] = {};
    for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < a.n; r0 += (int64_t)gridDim.x * rows) {
        const int64_t row = r0 + r.slot;
        const bool there = row < a.n;
        float h[K][V], yn[K][V], p[K][V], g[K][V], dH[K][V], du[K][V];
        const float4 st = there ? *reinterpret_cast<const float4 *>(a.stats + 4 * row) : make_float4(0.f, 1.f, 0.f, 1.f);
        if (a.x.data) r.load(a.x, row, there, h);
        else r.each([&](int k, int j) { h[k][j] = 0.f; });
        if (a.y.data) r.load(a.y, row, there, yn);
        if (a.dh.data) r.load(a.dh, row, there, dH);
        else r.each([&](int k, int j) { dH[k][j] = 0.f; });
        if (a.du.data) r.load(a.du, row, there, du);
        if (r.gated()) r.gate(row, there, g);
        // h again, from what it was formed of
        r.each([&](int k, int j) { h[k][j] *= a.residual; });
        if (a.y.data) {
            r.each([&](int k, int j) { yn[k][j] = (yn[k][j] - st.x) * st.y; });
            r.affine(yn, a.post_w, a.post_b, p);
            if (r.gated()) r.each([&](int k, int j) { h[k][j] = fmaf(g[k][j], p[k][j], h[k][j]); });
            else r.each([&](int k, int j) { h[k][j] += p[k][j]; });
        }
        if (a.du.data) {
            if (a.pre == NONE) {
                r.each([&](int k, int j) { dH[k][j] += du[k][j]; });
            } else {
                r.each([&](int k, int j) { h[k][j] = (h[k][j] - st.z) * st.w; }); // hn
                if (there) {
                    if (a.planes & 1) r.each([&](int k, int j) { acc[0][k][j] = fmaf(du[k][j], h[k][j], acc[0][k][j]); });
                    if (a.planes & 2) r.each([&](int k, int j) { acc[1][k][j] += du[k][j]; });
                }
                r.affine(du, a.pre_w, nullptr, du);
                const float c1 = r.sum([&](int k, int j) { return du[k][j] * h[k][j]; }) * a.inv_width;
                const float c0 = a.pre == LAYER ? r.sum([&](int k, int j) { return du[k][j]; }) * a.inv_width : 0.f;
                r.each([&](int k, int j) { dH[k][j] += st.w * (du[k][j] - c0 - h[k][j] * c1); });
            }
        }
        if (MULTI && !FULL && !(a.du.data && a.pre != NONE)) __syncthreads(); // rows in place, as in the forward pass
        if (a.dx.data && there) {
            r.each([&](int k, int j) { h[k][j] = a.residual * dH[k][j]; });
            r.store(a.dx, row, h);
        }
        if (!a.y.data) continue;
        if (a.dgate.data && there) {
            r.each([&](int k, int j) { p[k][j] *= a.sigmoid ? dH[k][j] * (g[k][j] * (1.f - g[k][j])) : dH[k][j]; });
            r.store(a.dgate, row, p);
        }
        if (column_gate && there) {
            if (a.planes & 4) r.each([&](int k, int j) { acc[2][k][j] = fmaf(dH[k][j], yn[k][j], acc[2][k][j]); });
            if (a.planes & 8) r.each([&](int k, int j) { acc[3][k][j] += dH[k][j]; });
        }
        if (r.gated()) r.each([&](int k, int j) { dH[k][j] *= g[k][j]; });
        if (!column_gate && there) {
            if (a.planes & 4) r.each([&](int k, int j) { acc[2][k][j] = fmaf(dH[k][j], yn[k][j], acc[2][k][j]); });
            if (a.planes & 8) r.each([&](int k, int j) { acc[3][k][j] += dH[k][j]; });
        }
        if (!a.dy.data) continue;
        if (a.post != NONE) {
            r.affine(dH, a.post_w, nullptr, dH);
            const float d1 = r.sum([&](int k, int j) { return dH[k][j] * yn[k][j]; }) * a.inv_width;
            const float d0 = a.post == LAYER ? r.sum([&](int k, int j) { return dH[k][j]; }) * a.inv_width : 0.f;
            r.each([&](int k, int j) { dH[k][j] = st.y * (dH[k][j] - d0 - yn[k][j] * d1); });
        }
        if (there) r.store(a.dy, row, dH);
    }
    if (!a.planes) return;
    // the workgroup's sums: over the rows of a wavefront, then over wavefronts (or over the rows beside each other), in order
    const int span = a.lanes < 64 ? 64 : a.lanes, part = threadIdx.x / span, parts = THREADS / span;
    float *out = a.partial + (int64_t)blockIdx.x * PLANES * a.width;
#pragma unroll
    for (int q = 0; q < PLANES; ++q) {
        if (!(a.planes >> q & 1)) continue;
        for (int step = a.lanes; step < 64; step <<= 1) r.each([&](int k, int j) { acc[q][k][j] += __shfl_xor(acc[q][k][j], step, 64); });
        const bool mine = a.lanes >= 64 || (threadIdx.x & 63) < a.lanes;
        if (parts > 1) {
            for (int w = 0; w < parts; ++w) {
                if (part == w && mine) {
#pragma unroll
                    for (int k = 0; k < K; ++k)
#pragma unroll
                        for (int j = 0; j < V; ++j)
                            if (r.at[k].on && j >= r.at[k].skip) {
                                float *s = sums + r.at[k].col + j;
                                *s = w ? *s + acc[q][k][j] : acc[q][k][j];
                            }
                }
                __syncthreads();
            }
            for (int c = threadIdx.x; c < a.width; c += THREADS) out[q * a.width + c] = sums[c];
            __syncthreads();
        } else if (mine) {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (r.at[k].on) store_vec<float, V>(out + q * a.width + r.at[k].col, acc[q][k]);
        }
    }
}

// Sums over the workgroups in fp64, and from them the parameters' gradients.  A workgroup takes 16 columns.
constexpr int FINAL_COLS = 16, FINAL_THREADS = 1024;
__global__ __launch_bounds__(FINAL_THREADS) void resnorm_params_kernel(const Args a, int32_t blocks, const slicegcn_resnorm_grads d)
{
    __shared__ double sums[FINAL_THREADS / FINAL_COLS][FINAL_COLS];
    const int c = threadIdx.x % FINAL_COLS, part = threadIdx.x / FINAL_COLS, parts = FINAL_THREADS / FINAL_COLS;
    const int32_t col = blockIdx.x * FINAL_COLS + c;
    double total[PLANES] = {};
    for (int q = 0; q < PLANES; ++q) {
        if (!(a.planes >> q & 1)) continue;
        double s = 0.0;
        if (col < a.width) {
#pragma unroll 8
            for (int32_t b = part; b < blocks; b += parts) s += (double)a.partial[((int64_t)b * PLANES + q) * a.width + col];
        }
        sums[part][c] = s;
        __syncthreads();
        if (part == 0)
            for (int i = 0; i < parts; ++i) total[q] += sums[i][c];
        __syncthreads();
    }
    if (part != 0 || col >= a.width) return;
    if (d.pre_w) d.pre_w[col] = (float)total[0];
    if (d.pre_b) d.pre_b[col] = (float)total[1];
    double s = 1.0, slope = 1.0;
    if (a.gate_col) {
        s = a.gate_col[col];
        if (a.sigmoid) {
            s = 1.0 / (1.0 + exp(-s));
            slope = s * (1.0 - s);
        }
    }
    if (d.post_w) d.post_w[col] = (float)(s * total[2]);
    if (d.post_b) d.post_b[col] = (float)(s * total[3]);
    if (d.gate) d.gate[col] = (float)(slope * ((a.post_w ? (double)a.post_w[col] : 1.0) * total[2] + (a.post_b ? (double)a.post_b[col] * total[3] : 0.0)));
}

// ---- host -----------------------------------------------------------------------------------------------------------------

// A row's accesses over lanes: as few lanes as the registers of a row allow (8 at least: a whole line), so that a sum over the row takes few steps.
struct Shape {
    int lanes, accesses; // per row, per lane
    Shape(int32_t width, int v, bool bwd)
    {
        const int all = (width + v - 1) / v, most = v == 1 ? 1 : (bwd && width <= BWD_WIDE ? BWD_ELEMS : FWD_ELEMS) / v;
        lanes = 8;
        while (lanes * most < all) lanes *= 2;
        accesses = (all + lanes - 1) / lanes;
    }
    int threads() const { return lanes > 256 ? lanes : 256; }
    bool full(int32_t width, int v) const { return width == lanes * accesses * v; }
};

int access_elems(int32_t width, int32_t type)
{
    const int v = 16 / type_bytes(type);
    return width < v ? 1 : v;
}

// Workgroups of the backward pass: each leaves one set of sums.
int64_t bwd_blocks(int64_t n, int32_t width, int32_t type)
{
    const Shape s(width, access_elems(width, type), true);
    const int64_t rows = s.threads() / s.lanes, want = (n + rows - 1) / rows, most = s.threads() > 512 ? 256 : s.threads() > 256 ? 512 : 1024;
    return want < most ? want : most;
}

template <bool BWD, class T, int V, int K, bool MULTI, bool FULL, int THREADS> void launch_kernel(const Args &a, int64_t blocks, hipStream_t s)
{
    if constexpr (BWD) resnorm_bwd_kernel<T, V, K, MULTI, FULL, THREADS><<<(unsigned)blocks, THREADS, 0, s>>>(a);
    else resnorm_fwd_kernel<T, V, K, MULTI, FULL, THREADS><<<(unsigned)blocks, THREADS, 0, s>>>(a);
}

template <bool BWD, class T, int V, int K, bool FULL> void launch_shape(const Args &a, const Shape &s, int64_t blocks, hipStream_t stream)
{
    constexpr int ELEMS = BWD ? BWD_ELEMS : FWD_ELEMS;
    if constexpr (K * V > ELEMS) { // the widest rows
        launch_kernel<BWD, T, V, K, true, FULL, 1024>(a, blocks, stream);
    } else {
        if (s.lanes <= 64) launch_kernel<BWD, T, V, K, false, FULL, 256>(a, blocks, stream);
        else if constexpr (2 * K * V > ELEMS) { // rows of fewer elements per lane take fewer lanes
            if (s.lanes <= 256) launch_kernel<BWD, T, V, K, true, FULL, 256>(a, blocks, stream);
            else if (s.lanes == 512) launch_kernel<BWD, T, V, K, true, FULL, 512>(a, blocks, stream);
            else launch_kernel<BWD, T, V, K, true, FULL, 1024>(a, blocks, stream);
        }
    }
}

template <bool BWD> int launch(Args &a, int32_t type, hipStream_t stream)
{
    const int v = access_elems(a.width, type);
    const Shape s(a.width, v, BWD);
    const bool full = s.full(a.width, v);
    a.lanes = s.lanes;
    const int64_t rows = s.threads() / s.lanes, want = (a.n + rows - 1) / rows;
    const int64_t blocks = BWD ? bwd_blocks(a.n, a.width, type) : want < (1 << 20) ? want : 1 << 20;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr int V = 16 / (int)sizeof(T);
        if (v == 1) launch_shape<BWD, T, 1, 1, false>(a, s, blocks, stream);
        else if (s.accesses == 1) full ? launch_shape<BWD, T, V, 1, true>(a, s, blocks, stream) : launch_shape<BWD, T, V, 1, false>(a, s, blocks, stream);
        else if (s.accesses == 2) full ? launch_shape<BWD, T, V, 2, true>(a, s, blocks, stream) : launch_shape<BWD, T, V, 2, false>(a, s, blocks, stream);
        else if constexpr (V == 4) {
            if (s.accesses == 3) full ? launch_shape<BWD, T, V, 3, true>(a, s, blocks, stream) : launch_shape<BWD, T, V, 3, false>(a, s, blocks, stream);
            else full ? launch_shape<BWD, T, V, 4, true>(a, s, blocks, stream) : launch_shape<BWD, T, V, 4, false>(a, s, blocks, stream);
        }
    });
    SG_LAUNCH_CHECK();
    return SLICEGCN_OK;
}

bool norm_kind(int32_t k) { return k == SLICEGCN_NORM_NONE || k == SLICEGCN_NORM_RMS || k == SLICEGCN_NORM_LAYER; }

int check(const char *what, const slicegcn_resnorm_desc *d, const slicegcn_resnorm_params *p, const slicegcn_resnorm_io *io, bool fwd)
{
    SG_REQUIRE(d && p && io, SLICEGCN_EINVAL, "%s: NULL descriptor, parameters or rows", what);
    SG_REQUIRE(d->n >= 0 && d->width >= 1, SLICEGCN_EINVAL, "%s: need n >= 0 and width >= 1", what);
    SG_REQUIRE(d->width <= SLICEGCN_RESNORM_MAX_WIDTH, SLICEGCN_EUNSUPPORTED, "%s: width = %d exceeds %d", what, d->width, SLICEGCN_RESNORM_MAX_WIDTH);
    SG_REQUIRE(known_type(d->type) && norm_kind(d->post) && norm_kind(d->pre), SLICEGCN_EINVAL, "%s: unknown type or norm", what);
    SG_REQUIRE((d->flags & ~SLICEGCN_GATE_SIGMOID) == 0, SLICEGCN_EINVAL, "%s: unknown flag", what);
    SG_REQUIRE(std::isfinite((float)d->residual), SLICEGCN_EINVAL, "%s: residual is not finite", what);
    SG_REQUIRE(d->eps > 0.0 && (float)d->eps > 0.f && std::isfinite((float)d->eps), SLICEGCN_EINVAL, "%s: eps must be positive", what);
    SG_REQUIRE(io->x.data || io->y.data, SLICEGCN_EINVAL, "%s: neither x nor y", what);
    SG_REQUIRE(!(p->gate && io->gate.data), SLICEGCN_EINVAL, "%s: two gates", what);
    const bool gated = p->gate || io->gate.data;
    SG_REQUIRE(gated || !(d->flags & SLICEGCN_GATE_SIGMOID), SLICEGCN_EINVAL, "%s: a sigmoid without gate", what);
    SG_REQUIRE(io->y.data || (d->post == SLICEGCN_NORM_NONE && !gated), SLICEGCN_EINVAL, "%s: a norm after the block or a gate without y", what);
    SG_REQUIRE(d->post != SLICEGCN_NORM_NONE || (!p->post_w && !p->post_b), SLICEGCN_EINVAL, "%s: a weight or bias without its norm (post)", what);
    SG_REQUIRE(d->pre != SLICEGCN_NORM_NONE || (!p->pre_w && !p->pre_b), SLICEGCN_EINVAL, "%s: a weight or bias without its norm (pre)", what);
    for (const float *v : {p->post_w, p->post_b, p->pre_w, p->pre_b, p->gate})
        SG_REQUIRE((reinterpret_cast<uintptr_t>(v) & 3u) == 0, SLICEGCN_EINVAL, "%s: misaligned parameter", what);
    auto rows = [&](const slicegcn_rows &r) { return !r.data || (r.ld >= d->width && aligned_for(r.data, d->type)); };
    SG_REQUIRE(rows(io->x) && rows(io->y) && rows(io->gate), SLICEGCN_EINVAL, "%s: ld smaller than the width, or misaligned base", what);
    SG_REQUIRE((reinterpret_cast<uintptr_t>(io->stats) & 15u) == 0, SLICEGCN_EINVAL, "%s: misaligned stats", what);
    if (fwd) {
        SG_REQUIRE(io->h.data || io->u.data, SLICEGCN_EINVAL, "%s: neither h nor u", what);
        SG_REQUIRE(rows(io->h) && rows(io->u), SLICEGCN_EINVAL, "%s: ld smaller than the width, or misaligned base", what);
        SG_REQUIRE(!io->stats || io->u.data || d->pre == SLICEGCN_NORM_NONE, SLICEGCN_EINVAL, "%s: stats of a norm that is not formed (no u)", what);
    } else {
        SG_REQUIRE(io->dh.data || io->du.data, SLICEGCN_EINVAL, "%s: neither dh nor du", what);
        SG_REQUIRE(rows(io->dh) && rows(io->du) && rows(io->dx) && rows(io->dy) && rows(io->dgate), SLICEGCN_EINVAL,
                   "%s: ld smaller than the width, or misaligned base", what);
        SG_REQUIRE((!io->dx.data || io->x.data) && (!io->dy.data || io->y.data) && (!io->dgate.data || io->gate.data), SLICEGCN_EINVAL,
                   "%s: a gradient of absent rows", what);
        SG_REQUIRE(io->stats || d->n == 0, SLICEGCN_EINVAL, "%s: no stats", what);
    }
    return SLICEGCN_OK;
}

Args make_args(const slicegcn_resnorm_desc *d, const slicegcn_resnorm_params *p, const slicegcn_resnorm_io *io)
{
    auto rows = [](const slicegcn_rows &r) { return RowPtr{static_cast<char *>(r.data), r.ld}; };
    Args a{};
    a.x = rows(io->x); a.y = rows(io->y); a.gate = rows(io->gate); a.h = rows(io->h); a.u = rows(io->u);
    a.dh = rows(io->dh); a.du = rows(io->du); a.dx = rows(io->dx); a.dy = rows(io->dy); a.dgate = rows(io->dgate);
    a.stats = io->stats;
    a.post_w = p->post_w; a.post_b = p->post_b; a.pre_w = p->pre_w; a.pre_b = p->pre_b; a.gate_col = p->gate;
    a.n = d->n;
    a.width = d->width;
    a.post = d->post; a.pre = d->pre;
    a.residual = (float)d->residual; a.eps = (float)d->eps; a.inv_width = 1.f / (float)d->width;
    a.sigmoid = (d->flags & SLICEGCN_GATE_SIGMOID) != 0;
    return a;
}

} // namespace
} // namespace slicegcn

using namespace slicegcn;

extern "C" int slicegcn_resnorm_fwd(const slicegcn_resnorm_desc *d, const slicegcn_resnorm_params *p, const slicegcn_resnorm_io *io, void *stream)
{
    if (int rc = check("resnorm_fwd", d, p, io, true)) return rc;
    if (d->n == 0) return SLICEGCN_OK;
    ProfScope prof(SLICEGCN_PROF_RESNORM, d->width, as_stream(stream));
    Args a = make_args(d, p, io);
    return launch<false>(a, d->type, as_stream(stream));
}

extern "C" size_t slicegcn_resnorm_bwd_workspace_bytes(int64_t n, int32_t width)
{
    if (n < 0 || width < 1 || width > SLICEGCN_RESNORM_MAX_WIDTH) return 0;
    const int64_t a = bwd_blocks(n, width, SLICEGCN_F32), b = bwd_blocks(n, width, SLICEGCN_BF16);
    return (size_t)round_up((a > b ? a : b) * PLANES * (int64_t)width * 4, 256);
}

extern "C" int slicegcn_resnorm_bwd(const slicegcn_resnorm_desc *d, const slicegcn_resnorm_params *p, const slicegcn_resnorm_io *io,
                                    const slicegcn_resnorm_grads *grads, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = check("resnorm_bwd", d, p, io, false)) return rc;
    const slicegcn_resnorm_grads g = grads ? *grads : slicegcn_resnorm_grads{};
    SG_REQUIRE((!g.post_w || p->post_w) && (!g.post_b || p->post_b) && (!g.pre_w || p->pre_w) && (!g.pre_b || p->pre_b) && (!g.gate || p->gate),
               SLICEGCN_EINVAL, "resnorm_bwd: a gradient of an absent parameter");
    for (const float *v : {g.post_w, g.post_b, g.pre_w, g.pre_b, g.gate})
        SG_REQUIRE((reinterpret_cast<uintptr_t>(v) & 3u) == 0, SLICEGCN_EINVAL, "resnorm_bwd: misaligned gradient of a parameter");
    const bool any = g.post_w || g.post_b || g.pre_w || g.pre_b || g.gate;
    Args a = make_args(d, p, io);
    if (any) {
        const size_t need = slicegcn_resnorm_bwd_workspace_bytes(d->n, d->width);
        SG_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SLICEGCN_EINVAL, "resnorm_bwd: misaligned workspace");
        SG_REQUIRE(need == 0 || (ws && ws_bytes >= need), SLICEGCN_EWORKSPACE, "resnorm_bwd: workspace of %zu bytes, %zu needed", ws_bytes, need);
        // without du the norm before the next block gets no gradient: zeros, like every sum over no rows
        a.planes = (g.pre_w ? 1u : 0u) | (g.pre_b ? 2u : 0u) | (g.post_w || g.gate ? 4u : 0u) | (g.post_b || (g.gate && p->post_b) ? 8u : 0u);
        a.partial = static_cast<float *>(ws);
    }
    ProfScope prof(SLICEGCN_PROF_RESNORM, d->width, as_stream(stream));
    if (d->n > 0)
        if (int rc = launch<true>(a, d->type, as_stream(stream))) return rc;
    if (any) {
        const int32_t blocks = d->n > 0 ? (int32_t)bwd_blocks(d->n, d->width, d->type) : 0;
        resnorm_params_kernel<<<(d->width + FINAL_COLS - 1) / FINAL_COLS, FINAL_THREADS, 0, as_stream(stream)>>>(a, blocks, g);
        SG_LAUNCH_CHECK();
    }
    return SLICEGCN_OK;
}
