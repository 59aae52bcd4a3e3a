// Norms before and after a block, fused with the block's gate and the residual: the calls, and the gradients of the parameters.
#include "resnorm.h"

#include <cfloat>
#include <cmath>
#include <initializer_list>

namespace slicegcn {

using namespace resnorm;

namespace {

// Sums over the workgroups in fp64, and from them the parameters' gradients.  A workgroup takes 8 columns, so that rows of a few hundred
// columns still occupy many of them; each plane has 32 threads a column.
constexpr int FINAL_COLS = 8, FINAL_PARTS = 32, FINAL_THREADS = PLANES * FINAL_PARTS * FINAL_COLS;
__global__ __launch_bounds__(FINAL_THREADS) void resnorm_params_kernel(const Args a, int32_t blocks, const slicegcn_resnorm_grads d)
{
    __shared__ double sums[PLANES][FINAL_PARTS][FINAL_COLS], total[PLANES][FINAL_COLS];
    const int c = threadIdx.x % FINAL_COLS, part = threadIdx.x / FINAL_COLS % FINAL_PARTS, q = threadIdx.x / (FINAL_COLS * FINAL_PARTS);
    const int32_t col = blockIdx.x * FINAL_COLS + c;
    double sum = 0.0;
    if (col < a.width && (a.planes >> q & 1)) {
#pragma unroll 8
        for (int32_t b = part; b < blocks; b += FINAL_PARTS) sum += (double)a.partial[((int64_t)b * PLANES + q) * a.width + col];
    }
    sums[q][part][c] = sum;
    __syncthreads();
    if (part == 0) {
        sum = 0.0;
#pragma unroll
        for (int i = 0; i < FINAL_PARTS; ++i) sum += sums[q][i][c];
        total[q][c] = sum;
    }
    __syncthreads();
    if (threadIdx.x >= FINAL_COLS || col >= a.width) return;
    if (d.pre_w) d.pre_w[col] = (float)total[0][c];
    if (d.pre_b) d.pre_b[col] = (float)total[1][c];
    double s = 1.0, slope = 1.0;
    if (a.gate_col) {
        s = a.gate_col[col];
        if (a.sigmoid) {
            const double e = exp(-s);
            s = 1.0 / (1.0 + e);
            slope = fmin(e, DBL_MAX) * s * s; // s (1 - s), in full where s is near 1
        }
    }
    if (d.post_w) d.post_w[col] = (float)(s * total[2][c]);
    if (d.post_b) d.post_b[col] = (float)(s * total[3][c]);
    if (d.gate) d.gate[col] = (float)(slope * ((a.post_w ? (double)a.post_w[col] : 1.0) * total[2][c] + (a.post_b ? (double)a.post_b[col] * total[3][c] : 0.0)));
}

// ---- host -----------------------------------------------------------------------------------------------------------------

// Workgroups of the backward pass: each leaves one set of sums.  A CU takes one where that has the operands of a row ahead in 32 KB, else (16-bit or
// narrow rows) two, and two where a gate per element makes the wavefronts compute for longer.  169 343 rows of 256 fp32 columns with one /
// two / three a CU 190 / 209 / 206 us, 60 000 of 1000 bf16 columns 196 / 146 / 153, 232 965 of 602 fp32 columns with such a gate 1375 / 864 / 1092.
int64_t bwd_blocks(int64_t n, int32_t width, int32_t type, bool matrix)
{
    constexpr int64_t CUS = 256, AHEAD = 32 << 10;
    const int v = access_elems(width, type);
    const Shape s(width, v);
    const int64_t rows = s.threads() / s.lanes, want = (n + rows - 1) / rows, ahead = (int64_t)s.threads() * s.accesses * v * type_bytes(type) * 4;
    const int64_t most = (s.threads() <= 256 && matrix) || ahead < AHEAD ? 2 * CUS : CUS;
    return want < most ? want : most;
}

template <bool BWD> int launch(Args &a, int32_t type, hipStream_t stream)
{
    const Shape s(a.width, access_elems(a.width, type));
    a.lanes = s.lanes;
    int64_t stored = 0; // rows of results, of all matrices together
    for (const RowPtr &m : BWD ? std::initializer_list<RowPtr>{a.dx, a.dy, a.dgate} : std::initializer_list<RowPtr>{a.h, a.u}) stored += m.data ? a.n : 0;
    a.past_cache = past_cache(stored, a.width, type);
    const int64_t rows = s.threads() / s.lanes, want = (a.n + rows - 1) / rows;
    const int v = access_elems(a.width, type);
    const bool loops = v > 1 && fwd_loops(s.lanes > 64, s.full(a.width, v), type_bytes(type));
    const int64_t most = BWD ? 0 : !loops ? 1 << 20 : s.lanes > 64 ? 4096 : 2048;
    const int64_t blocks = BWD ? bwd_blocks(a.n, a.width, type, a.gate.data != nullptr) : want < most ? want : most;
    with_type(type, [&](auto t) {
        if (BWD) launch_bwd<decltype(t)>(a, s, blocks, stream);
        else launch_fwd<decltype(t)>(a, s, blocks, stream);
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
    const int64_t a = bwd_blocks(n, width, SLICEGCN_F32, true), b = bwd_blocks(n, width, SLICEGCN_BF16, true);
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
        const int32_t blocks = d->n > 0 ? (int32_t)bwd_blocks(d->n, d->width, d->type, a.gate.data != nullptr) : 0;
        resnorm_params_kernel<<<(d->width + FINAL_COLS - 1) / FINAL_COLS, FINAL_THREADS, 0, as_stream(stream)>>>(a, blocks, g);
        SG_LAUNCH_CHECK();
    }
    return SLICEGCN_OK;
}
