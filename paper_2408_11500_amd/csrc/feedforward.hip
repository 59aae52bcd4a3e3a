// Products of rows with a weight matrix (slicegcn_product_*) and gated projections (slicegcn_gated_*): the entry points, how a product is cut, and what goes round the
// products of a backward pass.
//
// A backward pass first forms the gradients before the activation in one pass over the rows (slope_kernel: dP, or dG and dU, rounded to the rows' type into
// the workspace; the column sums for the biases from the same values unrounded), then dX as one product (over both dG and dU) and the
// weights' gradients as one launch.
#include "product.h"

#include <cmath>

namespace slicegcn {

namespace {

constexpr int CUS = 256;
constexpr int64_t MOST_PARTIAL = (int64_t)256 << 20; // bytes of sums of parts of k
constexpr int64_t CHAIN = 1024;                      // steps of k that one sum runs over in fp32 at most

int tile_for(const ProductShape &s)
{
    if (s.M <= 32) return 2;
    const int64_t cols = s.gated ? TILE_N[0] / 2 : TILE_N[0];
    const int64_t large = (s.M + TILE_M[0] - 1) / TILE_M[0] * ((s.N + cols - 1) / cols) * s.sets;
    return large >= CUS ? 0 : 1;
}

} // namespace

ProductPlan plan_product(const ProductShape &s, bool aligned)
{
    ProductPlan p{};
    aligned = aligned && s.type != SLICEGCN_F32;
    p.kernel = aligned && s.by_rows && s.M <= ROWS_MOST ? BY_ROWS : aligned && s.M > ROWS_MOST && s.N > 64 ? BY_TILES : BY_REGISTERS;
    p.tile = tile_for(s);
    const int bk = p.kernel == BY_REGISTERS ? step_k(s.type) : DIRECT_K;
    const int bm = p.kernel == BY_ROWS ? ROWS_MOST : p.kernel == BY_TILES ? DIRECT_TILE : TILE_M[p.tile];
    const int both = p.kernel == BY_ROWS ? 64 : p.kernel == BY_TILES ? DIRECT_TILE : TILE_N[p.tile], bn = s.gated ? both / 2 : both;
    const int64_t tiles = (s.M + bm - 1) / bm * ((s.N + bn - 1) / bn) * s.sets;
    const int64_t steps = (s.K + bk - 1) / bk * s.segments, one = (int64_t)(s.gated ? 2 : s.sets) * s.M * s.N * 4;
    const int64_t want = p.kernel == BY_REGISTERS ? 2 * CUS : CUS;
    const int64_t least = p.kernel == BY_REGISTERS ? 4 : p.kernel == BY_TILES ? 16 : 64; // steps of a part
    int64_t splits = 2 * tiles > want ? 1 : want / (tiles > 0 ? tiles : 1);
    if (splits > steps / least) splits = steps / least;
    if (splits * one > MOST_PARTIAL) splits = MOST_PARTIAL / one;
    if (splits < (steps + CHAIN - 1) / CHAIN) splits = (steps + CHAIN - 1) / CHAIN;
    if (splits < 1) splits = 1;
    const int64_t each = (steps + splits - 1) / splits;
    p.steps_per_split = (int32_t)(each > 0 ? each : 1);
    p.splits = (int32_t)(steps > 0 ? (steps + p.steps_per_split - 1) / p.steps_per_split : 1);
    p.bytes = p.splits > 1 ? (size_t)round_up(p.splits * one, 256) : 0;
    return p;
}

namespace {

// What a call may need, however its operands lie
size_t partial_bytes(const ProductShape &s)
{
    const size_t x = plan_product(s, false).bytes, y = plan_product(s, true).bytes;
    return x > y ? x : y;
}

// Whether both operands can go straight into LDS: rows and columns in whole units of 16 bytes, offsets within a tile in 32 bits
bool on_units(const Operand &o) { return aligned16(o.p) && o.ld % 8 == 0 && o.ld <= 1 << 22; }
bool aligned_product(int layouts, const ProductShape &s, const ProductArgs &a)
{
    for (int i = 0; i < (s.segments > s.sets ? s.segments : s.sets); ++i)
        if (!on_units(a.a[i]) || !on_units(a.b[i])) return false;
    if (s.gated && !on_units(a.b[1])) return false;
    switch (layouts) {
    case PRODUCT_XW: return s.K % 8 == 0 && s.N % 8 == 0;
    case PRODUCT_GWT: return s.K % 8 == 0;
    default: return s.M % 8 == 0 && s.N % 8 == 0;
    }
}

int launch_product(const ProductShape &s, int layouts, int epilogue, ProductArgs &a, hipStream_t stream)
{
    const int32_t type = s.type;
    const ProductPlan plan = plan_product(s, aligned_product(layouts, s, a));
    return type == SLICEGCN_F32    ? launch_product_f32(layouts, epilogue, plan, a, stream)
           : type == SLICEGCN_BF16 ? launch_product_bf16(layouts, epilogue, plan, a, stream)
                                   : launch_product_f16(layouts, epilogue, plan, a, stream);
}

// ---- gradients before the activation ----------------------------------------------------------------------------------

// Rows of a backward pass.  GATED: g, u and d = dH give dg, du;  else p (act != none) and d = dY give dg = dP.  dr = residual * d.
struct SlopeArgs {
    Operand g, u, d;
    char *dg, *du, *dr;
    int64_t ldg, ldu, ldr, n;
    int32_t w, act;
    float residual;
    double *partial; // column sums of parts of the rows: [part][1 or 2][w], where biases have gradients
    int32_t parts;
    int64_t rows_per_part;
};

constexpr int SLOPE_V = 4, SLOPE_RUN = 32; // columns a thread owns; rows that are added in fp32 before they are added in fp64

// Workgroup (x, y): 64 x 4 columns, rows of part y; the four wavefronts take rows in turn
template <class T, bool GATED> __global__ __launch_bounds__(256) void slope_kernel(const SlopeArgs a)
{
    constexpr int V = SLOPE_V, Q = GATED ? 2 : 1;
    __shared__ double sums[3][Q * V][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t col = ((int64_t)blockIdx.x * 64 + lane) * V;
    const int left = a.w - col < V ? (int)(a.w - col) : V;
    const int64_t first = blockIdx.y * a.rows_per_part, last = first + a.rows_per_part < a.n ? first + a.rows_per_part : a.n;
    double total[Q][V] = {};
    float run[Q][V] = {};
    int in_run = 0;
    auto read = [&](const Operand &m, int64_t row, float (&v)[V]) {
        const T *p = reinterpret_cast<const T *>(m.p) + row * m.ld + col;
        if (left >= V) {
            const auto x = load_vec<T, V>(p);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = (float)x[i];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = i < left ? (float)p[i] : 0.f;
        }
    };
    auto write = [&](char *base, int64_t ld, int64_t row, const float (&v)[V]) {
        T *p = reinterpret_cast<T *>(base) + row * ld + col;
        if (left >= V) {
            store_vec<T, V>(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < left) p[i] = (T)v[i];
        }
    };
    if (left > 0) {
        for (int64_t row = first + wave; row < last; row += 4) {
            float d[V], g[V], u[V], o[Q][V];
            read(a.d, row, d);
            if (a.g.p) read(a.g, row, g);
            if (GATED) read(a.u, row, u);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float y = 0.f, slope = 1.f;
                if (a.g.p) activated_slope(a.act, g[i], y, slope);
                o[0][i] = GATED ? d[i] * u[i] * slope : d[i] * slope;
                if (GATED) o[Q - 1][i] = d[i] * y;
            }
            if (a.dg) write(a.dg, a.ldg, row, o[0]);
            if (GATED && a.du) write(a.du, a.ldu, row, o[Q - 1]);
            if (a.dr) {
#pragma unroll
                for (int i = 0; i < V; ++i) d[i] *= a.residual;
                write(a.dr, a.ldr, row, d);
            }
            if (a.partial) {
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int i = 0; i < V; ++i) run[q][i] += o[q][i];
                if (++in_run == SLOPE_RUN) {
                    in_run = 0;
#pragma unroll
                    for (int q = 0; q < Q; ++q)
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            total[q][i] += (double)run[q][i];
                            run[q][i] = 0.f;
                        }
                }
            }
        }
    }
    if (!a.partial) return; // the same for the workgroup
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            total[q][i] += (double)run[q][i];
            if (wave > 0) sums[wave - 1][q * V + i][lane] = total[q][i];
        }
    __syncthreads();
    if (wave > 0 || left <= 0) return;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (i >= left) continue;
            double t = total[q][i];
#pragma unroll
            for (int w = 0; w < 3; ++w) t += sums[w][q * V + i][lane];
            a.partial[((int64_t)blockIdx.y * Q + q) * a.w + col + i] = t;
        }
}

// db[q][j] = sum over the parts, in order; 64 columns and 4 shares of the parts a workgroup
__global__ __launch_bounds__(256) void bias_kernel(const double *__restrict__ partial, int32_t parts, int32_t q_count, int32_t w, float *__restrict__ db0,
                                                   float *__restrict__ db1)
{
    __shared__ double sums[4][64];
    const int lane = threadIdx.x % 64, share = threadIdx.x / 64, q = blockIdx.y;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    double t = 0.0;
    if (col < w)
        for (int32_t p = share; p < parts; p += 4) t += partial[((int64_t)p * q_count + q) * w + col];
    sums[share][lane] = t;
    __syncthreads();
    float *db = q ? db1 : db0;
    if (share == 0 && col < w && db) db[col] = (float)(((sums[0][lane] + sums[1][lane]) + sums[2][lane]) + sums[3][lane]);
}

int64_t slope_parts(int64_t n, int32_t w)
{
    const int64_t cols = ((int64_t)w + 64 * SLOPE_V - 1) / (64 * SLOPE_V);
    int64_t parts = (8 * CUS + cols - 1) / cols;
    if (parts > (n + 15) / 16) parts = (n + 15) / 16;
    return parts > 0 ? parts : 1;
}

// Workspace of a backward pass: gradients before the activation, their column sums, sums of parts of k
struct BwdWorkspace {
    int64_t ld; // of the gradients before the activation: rows on 16-byte boundaries
    size_t rows, sums, partial;
    size_t bytes(int q) const { return q * rows + sums + partial; }
};

ProductShape dx_shape(int64_t n, int32_t w_in, int32_t w_out, int32_t type, int q) { return ProductShape{n, w_out, w_in, q, 1, type, false, true}; }
ProductShape dw_shape(int64_t n, int32_t w_in, int32_t w_out, int32_t type, int q) { return ProductShape{w_in, n, w_out, 1, q, type, false, false}; }

BwdWorkspace bwd_workspace(int64_t n, int32_t w_in, int32_t w_out, int32_t type, int q)
{
    BwdWorkspace w;
    w.ld = round_up(w_out, 8);
    w.rows = (size_t)round_up(n * w.ld * type_bytes(type), 256);
    w.sums = (size_t)round_up(slope_parts(n, w_out) * q * (int64_t)w_out * 8, 256);
    const size_t x = partial_bytes(dx_shape(n, w_in, w_out, type, q)), y = partial_bytes(dw_shape(n, w_in, w_out, type, q));
    w.partial = x > y ? x : y;
    return w;
}

bool sizes_fit(int64_t n, int32_t w_in, int32_t w_out) { return n >= 0 && n <= INT32_MAX && w_in >= 1 && w_out >= 1 && w_in <= 1 << 24 && w_out <= 1 << 24; }

int check(const char *what, const slicegcn_product_desc *d)
{
    SG_REQUIRE(d, SLICEGCN_EINVAL, "%s: NULL descriptor", what);
    SG_REQUIRE(d->n >= 0 && d->w_in >= 1 && d->w_out >= 1, SLICEGCN_EINVAL, "%s: need n >= 0 and widths >= 1", what);
    SG_REQUIRE(known_type(d->type), SLICEGCN_EINVAL, "%s: unknown type", what);
    SG_REQUIRE(d->act >= SLICEGCN_ACT_NONE && d->act <= SLICEGCN_ACT_GELU, SLICEGCN_EINVAL, "%s: unknown activation", what);
    SG_REQUIRE(std::isfinite((float)d->residual), SLICEGCN_EINVAL, "%s: residual is not finite", what);
    SG_REQUIRE(sizes_fit(d->n, d->w_in, d->w_out), SLICEGCN_ERANGE, "%s: n or a width too large", what);
    return SLICEGCN_OK;
}

bool present(const slicegcn_matrix *m) { return m && m->data; }

int check_rows(const char *what, const char *name, const slicegcn_matrix *m, int32_t width, int32_t type, bool needed)
{
    SG_REQUIRE(!needed || present(m), SLICEGCN_EINVAL, "%s: NULL %s", what, name);
    SG_REQUIRE(!present(m) || (m->ld >= width && m->ld <= (int64_t)1 << 31 && aligned_for(m->data, type)), SLICEGCN_EINVAL,
               "%s: %s has an ld smaller than its width (or beyond 2^31), or a misaligned base", what, name);
    return SLICEGCN_OK;
}

int check_params(const char *what, int32_t type, std::initializer_list<const void *> weights, std::initializer_list<const float *> biases)
{
    for (const void *w : weights) SG_REQUIRE(!w || aligned_for(w, type), SLICEGCN_EINVAL, "%s: misaligned weights", what);
    for (const float *b : biases) SG_REQUIRE((reinterpret_cast<uintptr_t>(b) & 3u) == 0, SLICEGCN_EINVAL, "%s: misaligned bias", what);
    return SLICEGCN_OK;
}

int check_workspace(const char *what, const void *ws, size_t ws_bytes, size_t need)
{
    SG_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 255u) == 0, SLICEGCN_EINVAL, "%s: misaligned workspace", what);
    SG_REQUIRE(need == 0 || (ws && ws_bytes >= need), SLICEGCN_EWORKSPACE, "%s: workspace of %zu bytes, %zu needed", what, ws_bytes, need);
    return SLICEGCN_OK;
}

Operand operand(const slicegcn_matrix *m) { return present(m) ? Operand{static_cast<const char *>(m->data), m->ld} : Operand{nullptr, 0}; }
Operand weights(const void *w, int32_t w_out) { return Operand{static_cast<const char *>(w), w_out}; }

ProductShape fwd_shape(int64_t n, int32_t w_in, int32_t w_out, int32_t type, bool gated) { return ProductShape{n, w_in, w_out, 1, 1, type, gated, true}; }

// Both backward passes.  q = 2: gated
struct BwdCall {
    const slicegcn_product_desc *d;
    Operand x, w[2], g, u, dy;
    const slicegcn_matrix *dx, *dr;
    void *dw[2];
    float *db[2];
};

int backward(const char *what, const BwdCall &c, int q, void *ws, size_t ws_bytes, hipStream_t stream)
{
    const slicegcn_product_desc &d = *c.d;
    const BwdWorkspace w = bwd_workspace(d.n, d.w_in, d.w_out, d.type, q);
    if (int rc = check_workspace(what, ws, ws_bytes, w.bytes(q))) return rc;
    const bool want_x = present(c.dx) && d.n > 0, want_w = c.dw[0] || c.dw[1], want_b = c.db[0] || c.db[1], want_r = present(c.dr) && d.n > 0;
    char *at = static_cast<char *>(ws);
    const bool plain = q == 1 && d.act == SLICEGCN_ACT_NONE; // dP is dY itself
    Operand dg[2] = {c.dy, c.dy};
    SlopeArgs s{};
    s.g = plain ? Operand{nullptr, 0} : c.g;
    s.u = c.u;
    s.d = c.dy;
    s.n = d.n;
    s.w = d.w_out;
    s.act = d.act;
    s.residual = (float)d.residual;
    if (!plain && (want_x || want_w)) {
        s.dg = at;
        s.ldg = s.ldu = w.ld;
        if (q == 2) s.du = at + w.rows;
        dg[0] = Operand{s.dg, w.ld};
        dg[1] = Operand{s.du, w.ld};
    }
    if (want_r) {
        s.dr = static_cast<char *>(c.dr->data);
        s.ldr = c.dr->ld;
    }
    at += q * w.rows;
    if (want_b) s.partial = reinterpret_cast<double *>(at);
    at += w.sums;
    float *partial = reinterpret_cast<float *>(at);

    ProfScope prof(SLICEGCN_PROF_PRODUCT, d.w_out, stream);
    if (s.dg || s.dr || s.partial) {
        s.parts = (int32_t)slope_parts(d.n, d.w_out);
        s.rows_per_part = (d.n + s.parts - 1) / s.parts;
        const dim3 grid((d.w_out + 64 * SLOPE_V - 1) / (64 * SLOPE_V), (unsigned)s.parts);
        with_type(d.type, [&](auto t) {
            if (q == 2) slope_kernel<decltype(t), true><<<grid, 256, 0, stream>>>(s);
            else slope_kernel<decltype(t), false><<<grid, 256, 0, stream>>>(s);
        });
        SG_LAUNCH_CHECK();
        if (want_b) {
            bias_kernel<<<dim3((d.w_out + 63) / 64, q), 256, 0, stream>>>(s.partial, s.parts, q, d.w_out, c.db[0], c.db[1]);
            SG_LAUNCH_CHECK();
        }
    }
    if (want_x) {
        ProductArgs a{};
        for (int i = 0; i < q; ++i) {
            a.a[i] = dg[i];
            a.b[i] = c.w[i];
        }
        a.M = d.n;
        a.K = d.w_out;
        a.N = d.w_in;
        a.segments = q;
        a.sets = 1;
        a.out[0] = static_cast<char *>(c.dx->data);
        a.ldo[0] = c.dx->ld;
        a.partial = partial;
        if (int rc = launch_product(dx_shape(d.n, d.w_in, d.w_out, d.type, q), PRODUCT_GWT, EPI_STORE, a, stream)) return rc;
    }
    if (want_w) {
        ProductArgs a{};
        int sets = 0;
        for (int i = 0; i < q; ++i) {
            if (!c.dw[i]) continue;
            a.a[sets] = c.x;
            a.b[sets] = dg[i];
            a.out[sets] = static_cast<char *>(c.dw[i]);
            a.ldo[sets++] = d.w_out;
        }
        a.M = d.w_in;
        a.K = d.n;
        a.N = d.w_out;
        a.segments = 1;
        a.sets = sets;
        a.partial = partial;
        // one of the two alone: cut like both, so that the workspace suffices and its bits are the same
        if (int rc = launch_product(dw_shape(d.n, d.w_in, d.w_out, d.type, q), PRODUCT_XTG, EPI_STORE, a, stream)) return rc;
    }
    return SLICEGCN_OK;
}

} // namespace
} // namespace slicegcn

using namespace slicegcn;

extern "C" size_t slicegcn_product_fwd_workspace_bytes(int64_t n, int32_t w_in, int32_t w_out, int32_t type)
{
    if (!sizes_fit(n, w_in, w_out) || !known_type(type) || n == 0) return 0;
    return partial_bytes(fwd_shape(n, w_in, w_out, type, false));
}

extern "C" int slicegcn_product_fwd(const slicegcn_product_desc *d, const slicegcn_matrix *X, const void *W, const float *b, const slicegcn_matrix *R,
                                    const slicegcn_matrix *P, const slicegcn_matrix *Y, void *ws, size_t ws_bytes, void *stream)
{
    const char *what = "product_fwd";
    if (int rc = check(what, d)) return rc;
    SG_REQUIRE(W, SLICEGCN_EINVAL, "%s: NULL W", what);
    if (int rc = check_rows(what, "X", X, d->w_in, d->type, true)) return rc;
    if (int rc = check_rows(what, "Y", Y, d->w_out, d->type, true)) return rc;
    if (int rc = check_rows(what, "R", R, d->w_out, d->type, false)) return rc;
    if (int rc = check_rows(what, "P", P, d->w_out, d->type, false)) return rc;
    if (int rc = check_params(what, d->type, {W}, {b})) return rc;
    if (d->n == 0) return SLICEGCN_OK;
    SG_REQUIRE(Y->data != X->data, SLICEGCN_EINVAL, "%s: Y in the rows of X", what);
    const ProductShape shape = fwd_shape(d->n, d->w_in, d->w_out, d->type, false);
    if (int rc = check_workspace(what, ws, ws_bytes, partial_bytes(shape))) return rc;
    ProductArgs a{};
    a.a[0] = operand(X);
    a.b[0] = weights(W, d->w_out);
    a.M = d->n;
    a.K = d->w_in;
    a.N = d->w_out;
    a.segments = a.sets = 1;
    a.out[0] = static_cast<char *>(Y->data);
    a.ldo[0] = Y->ld;
    a.bias[0] = b;
    a.r = operand(R);
    if (present(P)) {
        a.keep[0] = static_cast<char *>(P->data);
        a.ldk[0] = P->ld;
    }
    a.residual = (float)d->residual;
    a.act = d->act;
    a.partial = static_cast<float *>(ws);
    ProfScope prof(SLICEGCN_PROF_PRODUCT, d->w_out, as_stream(stream));
    return launch_product(shape, PRODUCT_XW, EPI_FORWARD, a, as_stream(stream));
}

extern "C" size_t slicegcn_product_bwd_workspace_bytes(int64_t n, int32_t w_in, int32_t w_out, int32_t type)
{
    if (!sizes_fit(n, w_in, w_out) || !known_type(type)) return 0;
    return bwd_workspace(n, w_in, w_out, type, 1).bytes(1);
}

extern "C" int slicegcn_product_bwd(const slicegcn_product_desc *d, const slicegcn_matrix *X, const void *W, const slicegcn_matrix *P,
                                    const slicegcn_matrix *dY, const slicegcn_matrix *dX, void *dW, float *db, const slicegcn_matrix *dR, void *ws,
                                    size_t ws_bytes, void *stream)
{
    const char *what = "product_bwd";
    if (int rc = check(what, d)) return rc;
    const bool rows = d->n > 0, slope = d->act != SLICEGCN_ACT_NONE && (present(dX) || dW || db);
    if (int rc = check_rows(what, "X", X, d->w_in, d->type, rows && dW)) return rc;
    if (int rc = check_rows(what, "P", P, d->w_out, d->type, rows && slope)) return rc;
    if (int rc = check_rows(what, "dY", dY, d->w_out, d->type, rows)) return rc;
    if (int rc = check_rows(what, "dX", dX, d->w_in, d->type, false)) return rc;
    if (int rc = check_rows(what, "dR", dR, d->w_out, d->type, false)) return rc;
    SG_REQUIRE(W || !present(dX) || !rows, SLICEGCN_EINVAL, "%s: NULL W", what);
    if (int rc = check_params(what, d->type, {W, dW}, {db})) return rc;
    BwdCall c{};
    c.d = d;
    c.x = operand(X);
    c.w[0] = weights(W, d->w_out);
    c.g = operand(P);
    c.dy = operand(dY);
    c.dx = dX;
    c.dr = dR;
    c.dw[0] = dW;
    c.db[0] = db;
    return backward(what, c, 1, ws, ws_bytes, as_stream(stream));
}

extern "C" size_t slicegcn_gated_fwd_workspace_bytes(int64_t n, int32_t w_in, int32_t w_out, int32_t type)
{
    if (!sizes_fit(n, w_in, w_out) || !known_type(type) || n == 0) return 0;
    return partial_bytes(fwd_shape(n, w_in, w_out, type, true));
}

extern "C" int slicegcn_gated_fwd(const slicegcn_product_desc *d, const slicegcn_matrix *X, const void *Wg, const void *Wu, const float *bg,
                                  const float *bu, const slicegcn_matrix *G, const slicegcn_matrix *U, const slicegcn_matrix *H, void *ws,
                                  size_t ws_bytes, void *stream)
{
    const char *what = "gated_fwd";
    if (int rc = check(what, d)) return rc;
    SG_REQUIRE(Wg && Wu, SLICEGCN_EINVAL, "%s: NULL Wg or Wu", what);
    if (int rc = check_rows(what, "X", X, d->w_in, d->type, true)) return rc;
    if (int rc = check_rows(what, "H", H, d->w_out, d->type, true)) return rc;
    if (int rc = check_rows(what, "G", G, d->w_out, d->type, false)) return rc;
    if (int rc = check_rows(what, "U", U, d->w_out, d->type, false)) return rc;
    SG_REQUIRE(present(G) == present(U), SLICEGCN_EINVAL, "%s: G without U, or U without G", what);
    if (int rc = check_params(what, d->type, {Wg, Wu}, {bg, bu})) return rc;
    if (d->n == 0) return SLICEGCN_OK;
    SG_REQUIRE(H->data != X->data, SLICEGCN_EINVAL, "%s: H in the rows of X", what);
    const ProductShape shape = fwd_shape(d->n, d->w_in, d->w_out, d->type, true);
    if (int rc = check_workspace(what, ws, ws_bytes, partial_bytes(shape))) return rc;
    ProductArgs a{};
    a.a[0] = operand(X);
    a.b[0] = weights(Wg, d->w_out);
    a.b[1] = weights(Wu, d->w_out);
    a.M = d->n;
    a.K = d->w_in;
    a.N = d->w_out;
    a.segments = a.sets = 1;
    a.out[0] = static_cast<char *>(H->data);
    a.ldo[0] = H->ld;
    a.bias[0] = bg;
    a.bias[1] = bu;
    if (present(G)) {
        a.keep[0] = static_cast<char *>(G->data);
        a.ldk[0] = G->ld;
        a.keep[1] = static_cast<char *>(U->data);
        a.ldk[1] = U->ld;
    }
    a.act = d->act;
    a.partial = static_cast<float *>(ws);
    ProfScope prof(SLICEGCN_PROF_PRODUCT, d->w_out, as_stream(stream));
    return launch_product(shape, PRODUCT_XW, EPI_GATED, a, as_stream(stream));
}

extern "C" size_t slicegcn_gated_bwd_workspace_bytes(int64_t n, int32_t w_in, int32_t w_out, int32_t type)
{
    if (!sizes_fit(n, w_in, w_out) || !known_type(type)) return 0;
    return bwd_workspace(n, w_in, w_out, type, 2).bytes(2);
}

extern "C" int slicegcn_gated_bwd(const slicegcn_product_desc *d, const slicegcn_matrix *X, const void *Wg, const void *Wu, const slicegcn_matrix *G,
                                  const slicegcn_matrix *U, const slicegcn_matrix *dH, const slicegcn_matrix *dX, void *dWg, void *dWu, float *dbg,
                                  float *dbu, void *ws, size_t ws_bytes, void *stream)
{
    const char *what = "gated_bwd";
    if (int rc = check(what, d)) return rc;
    const bool rows = d->n > 0;
    if (int rc = check_rows(what, "X", X, d->w_in, d->type, rows && (dWg || dWu))) return rc;
    if (int rc = check_rows(what, "G", G, d->w_out, d->type, rows)) return rc;
    if (int rc = check_rows(what, "U", U, d->w_out, d->type, rows)) return rc;
    if (int rc = check_rows(what, "dH", dH, d->w_out, d->type, rows)) return rc;
    if (int rc = check_rows(what, "dX", dX, d->w_in, d->type, false)) return rc;
    SG_REQUIRE((Wg && Wu) || !present(dX) || !rows, SLICEGCN_EINVAL, "%s: NULL Wg or Wu", what);
    if (int rc = check_params(what, d->type, {Wg, Wu, dWg, dWu}, {dbg, dbu})) return rc;
    BwdCall c{};
    c.d = d;
    c.x = operand(X);
    c.w[0] = weights(Wg, d->w_out);
    c.w[1] = weights(Wu, d->w_out);
    c.g = operand(G);
    c.u = operand(U);
    c.dy = operand(dH);
    c.dx = dX;
    c.dw[0] = dWg;
    c.dw[1] = dWu;
    c.db[0] = dbg;
    c.db[1] = dbu;
    return backward(what, c, 2, ws, ws_bytes, as_stream(stream));
}
