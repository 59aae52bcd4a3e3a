// Products of rows with a weight matrix (slicegcn_product_*) and gated projections (slicegcn_gated_*): the entry points, how a product is cut, and what goes round the
// products of a backward pass.
//
// A backward pass first forms the gradients before the activation in one pass over the rows (slope_kernel: dP, or dG and dU, rounded to the rows' type into
// the workspace; the column sums for the biases from the same values unrounded), then dX as one product (over both dG and dU) and the
// weights' gradients as one launch.  Short passes form both in one launch (paired), narrow layers of 16 bits on many rows everything in one sweep (product_narrow.h).
#include "product.h"

#include <cmath>

namespace slicegcn {

namespace {

constexpr int CUS = 256;
constexpr int64_t MOST_PARTIAL = (int64_t)256 << 20; // bytes of sums of parts of k
constexpr int64_t CHAIN = 1024;                      // steps of k that one sum runs over in fp32 at most

// Tiles through registers.  Few rows: 32 x 128 (4 rows 535 -> 6038 fp32 11.7 us, in 64 x 64 12.3; 28 rows 3970 -> 1475 gated fp32 19.2 and 23.4).  fp32: 128 x 128 where that
// gives every CU a tile (16000 rows 1000 -> 1000 180 us, in 64 x 64 218), 64 x 64 where it does not (1000 rows 512 -> 512 15.9 us, in 128 x 128 19.5).  16-bit operands:
// 64 x 64 alone, since with 128 x 128 the epilogue of a forward pass does not fit the registers beside the sums (65536 rows 256 -> 64 bf16 gelu 68 us, in 64 x 64 13).
int tile_for(const ProductShape &s)
{
    if (s.M <= 32) return 2;
    if (s.type != SLICEGCN_F32) return 1;
    const int64_t cols = s.gated ? TILE_N[0] / 2 : TILE_N[0];
    const int64_t large = (s.M + TILE_M[0] - 1) / TILE_M[0] * ((s.N + cols - 1) / cols) * s.sets;
    return large >= CUS ? 0 : 1;
}

// 16-bit products that are worth tiles of 256 x 256, straight into LDS, and copies of operands that lie oddly.  A wavefront's epilogue alone takes 13 us there, with a gelu
// (4096 rows 1024 -> 1024 36 us, in 64 x 64 through registers 22; 4096 rows 1024 -> 4096 48 and 66; 8192 rows 1024 -> 1024 gated 34 and 61), and half-empty tiles do
// not pay (200 k rows 1024 -> 128 190 us and 145), but for sums over the rows, whose operands are read once then (dX and dW of 200 k rows 1000 -> 104 331 us and 407).
constexpr double TILES_LEAST = 1e10; // multiplications
double multiplications(const ProductShape &s) { return (double)s.M * (double)s.N * (double)s.K * (s.gated ? 2 : s.segments * s.sets); }
bool long_product(const ProductShape &s)
{
    return s.type != SLICEGCN_F32 && s.M > 128 && s.N * (s.gated ? 2 : 1) > (s.by_rows ? 128 : 64) && multiplications(s) >= TILES_LEAST;
}

// Few rows of 16 bits in strips of columns, where that is one launch for two: sums of up to 2048 (one row 2048 -> 2048 bf16 9.0 us, cut in parts through registers 12.7;
// 32 rows 1024 -> 2816 gated 9.5 and 12.3; one row 4096 -> 4096 16.5 and 13.6), and fewer columns than keep all CUs busy in another way (32 rows 2048 -> 5632 gated 19.8 and
// 18.5).  More rows go through registers (48 rows 2048 -> 2048 14.9 us in strips, 11.7).
int kernel_for(const ProductShape &s, bool aligned)
{
    if (!aligned || s.type == SLICEGCN_F32) return BY_REGISTERS;
    const int64_t steps = (s.K + DIRECT_K - 1) / DIRECT_K * s.segments, strips = (s.N * (s.gated ? 2 : 1) + 63) / 64;
    if (s.by_rows && s.M <= ROWS_MOST && steps <= 64 && strips <= CUS / 2) return BY_ROWS;
    return long_product(s) ? BY_TILES : BY_REGISTERS;
}

} // namespace

// Where the tiles of 256 x 256 are more than one round of the CUs and the last round would leave half of them or more idle, its tiles are cut along k and joined: 8192 rows 4096 ->
// 2304 161 us, whole 206; 8192 rows 2048 -> 2304 104 and 122; 20000 rows 1024 -> 1024 78 and 82, the shortest sum with which that was tried.
constexpr int64_t TAIL_LEAST = 32; // steps

// How k is cut: so that about `want` workgroups run, which are two a CU through registers (300 rows 4096 -> 512 bf16 14.6 us, with four 17.1; 300 rows 10240 -> 1024 31.5 and
// with one 33.8), in parts of `least` steps or more (300 rows 4096 -> 1024 in tiles of 256: 16 steps 29 us, 4 33, 64 51; 300 rows 700 -> 500 fp32 through registers: 4 steps 12.2,
// 1 14.4, 16 19.7).  Short sums are not cut, as the launch that joins the parts takes longer than they do (1000 rows 1024 -> 1024 bf16 11.7 us, in two parts 17.1; 2000 rows 256 ->
// 256 fp32 10.7 and 12.2); 16-bit operands that lie oddly are slower by the step and cut sooner (one row 1001 -> 1203 bf16 12.3 us, in one part 16.3; 300 rows 501 -> 701 13.1 and 10.4).
ProductPlan plan_product(const ProductShape &s, bool aligned)
{
    ProductPlan p{};
    p.kernel = kernel_for(s, aligned);
    p.tile = tile_for(s);
    const int bk = p.kernel == BY_REGISTERS ? step_k(s.type) : DIRECT_K;
    const int bm = p.kernel == BY_ROWS ? ROWS_MOST : p.kernel == BY_TILES ? DIRECT_TILE : TILE_M[p.tile];
    const int both = p.kernel == BY_ROWS ? 64 : p.kernel == BY_TILES ? DIRECT_TILE : TILE_N[p.tile], bn = s.gated ? both / 2 : both;
    const int64_t tiles = (s.M + bm - 1) / bm * ((s.N + bn - 1) / bn) * s.sets;
    const int64_t steps = (s.K + bk - 1) / bk * s.segments, one = (int64_t)(s.gated ? 2 : s.sets) * s.M * s.N * 4;
    const int64_t want = p.kernel == BY_REGISTERS ? 2 * CUS : CUS;
    const int64_t least = p.kernel == BY_REGISTERS ? 4 : 16; // steps of a part
    int64_t splits = 2 * tiles > want ? 1 : want / (tiles > 0 ? tiles : 1);
    if (splits > steps / least) splits = steps / least;
    if (p.kernel == BY_REGISTERS && steps < (s.type == SLICEGCN_F32 ? 16 : aligned ? 24 : 12)) splits = 1;
    if (splits * one > MOST_PARTIAL) splits = MOST_PARTIAL / one;
    if (splits < (steps + CHAIN - 1) / CHAIN) splits = (steps + CHAIN - 1) / CHAIN;
    if (splits < 1 || p.kernel == BY_ROWS) splits = 1;
    const int64_t each = (steps + splits - 1) / splits;
    p.steps_per_split = (int32_t)(each > 0 ? each : 1);
    p.splits = (int32_t)(steps > 0 ? (steps + p.steps_per_split - 1) / p.steps_per_split : 1);
    p.bytes = p.splits > 1 ? (size_t)round_up(p.splits * one, 256) : 0;
    if (p.kernel == BY_TILES && p.splits == 1 && tiles > CUS && steps >= TAIL_LEAST) {
        const int64_t rest = tiles % CUS, most = steps / 16;
        int64_t parts = rest > 0 ? CUS / rest : 0;
        parts = parts < most ? parts : most;
        parts = parts < 8 ? parts : 8;
        if (parts > 1) {
            p.tail = (int32_t)rest;
            p.steps_per_split = (int32_t)((steps + parts - 1) / parts);
            p.tail_splits = (int32_t)((steps + p.steps_per_split - 1) / p.steps_per_split);
            p.bytes = (size_t)rest * p.tail_splits * DIRECT_TILE * DIRECT_TILE * 4;
        }
    }
    return p;
}

namespace {

// Whether the products of a backward pass of these sizes share a launch, by the multiplications in both; and how each is cut then.  2048 rows 64 -> 170 gated fp32 17.7 us,
// in launches of their own 27.1; 2048 rows 256 -> 688 gated bf16 28 and 40, fp32 48 and 52; beyond: 4096 rows 256 -> 688 gated fp32 82 and 75, 8192 rows 512 -> 1024 bf16 69
// and 63.
constexpr int64_t PAIR_MOST_F32 = (int64_t)1 << 30, PAIR_MOST_16 = (int64_t)1 << 31;
constexpr int64_t PAIR_RESULTS = (int64_t)1 << 20; // elements of dX and of dW, which all go through memory as sums of parts: 1182 rows 2488 -> 13 gated fp32 31.5 us so, 26.2 apart
bool paired(int64_t n, int32_t w_in, int32_t w_out, int32_t type, int q)
{
    return n > 0 && (double)n * (double)w_in * (double)w_out * q <= (double)(type == SLICEGCN_F32 ? PAIR_MOST_F32 : PAIR_MOST_16) && n * w_in <= PAIR_RESULTS && (int64_t)w_in * w_out * q <= PAIR_RESULTS;
}
ProductPlan pair_plan(const ProductShape &s)
{
    ProductPlan p{};
    const int64_t tiles = (s.M + PAIR_TILE - 1) / PAIR_TILE * ((s.N + PAIR_TILE - 1) / PAIR_TILE) * s.sets;
    const int64_t bk = step_k(s.type), steps = (s.K + bk - 1) / bk * s.segments, one = s.sets * s.M * s.N * 4;
    int64_t splits = CUS / tiles;
    if (splits > steps / 2) splits = steps / 2;
    if (splits < (steps + CHAIN - 1) / CHAIN) splits = (steps + CHAIN - 1) / CHAIN;
    if (splits < 1) splits = 1;
    p.steps_per_split = (int32_t)((steps + splits - 1) / splits);
    p.splits = (int32_t)((steps + p.steps_per_split - 1) / p.steps_per_split);
    p.bytes = (size_t)round_up(p.splits * one, 256);
    return p;
}

// Whether the gradients before the activation are kept in two 16-bit terms: where there are so few of them that the errors of rounding them do not level out over a sum, and both
// products of them share a launch, in which the second term costs little (3 rows 2595 -> 8 gated bf16 gelu: errors of dX and dW 0.0031 of their norms in one term, 0.0017 in two).
constexpr int64_t TERMS_MOST = (int64_t)1 << 15; // elements
// Elsewhere a caller may ask for them, for twice the products (in one sweep over narrow layers they would need more registers than there are: 2.4 M rows 100 -> 256 bf16 gelu
// 0.96 ms in one term, 1.40 in two; gated 100 -> 128 0.69 and 1.87).
int terms_of(int64_t n, int32_t w_in, int32_t w_out, int32_t type, int q, bool two)
{
    return type != SLICEGCN_F32 && (two || (n * w_out * q <= TERMS_MOST && paired(n, w_in, w_out, type, q))) ? 2 : 1;
}

// What a call may need, however its operands lie
size_t partial_bytes(const ProductShape &s)
{
    const size_t x = plan_product(s, false).bytes, y = plan_product(s, true).bytes;
    return x > y ? x : y;
}

// Whether an operand can go straight into LDS: rows in whole units of 16 bytes
bool on_units(const Operand &o, int64_t width) { return aligned16(o.p) && o.ld % 8 == 0 && (width % 8 == 0 || o.padded); }
int operands(const ProductArgs &a) { return a.segments > a.sets ? a.segments : a.sets; } // on either side; GATED: one, and two on the N side
int64_t width_a(int layouts, const ProductShape &s) { return layouts == PRODUCT_XTG ? s.M : s.K; } // of a row as stored
int64_t width_b(int layouts, const ProductShape &s) { return layouts == PRODUCT_GWT ? s.K : s.N; }

bool aligned_product(int layouts, const ProductShape &s, const ProductArgs &a)
{
    for (int i = 0; i < operands(a); ++i)
        if (!on_units(a.a[i], width_a(layouts, s)) || !on_units(a.b[i], width_b(layouts, s))) return false;
    return !s.gated || on_units(a.b[1], width_b(layouts, s));
}

// ---- 16-bit operands whose rows are no whole units of 16 bytes: copied so that they are, where the product is long against a copy of its operands.

int64_t packed_bytes(int64_t rows, int64_t width) { return width % 8 == 0 ? 0 : round_up(rows * round_up(width, 8) * 2, 256); }
int64_t rows_a(int layouts, const ProductShape &s) { return layouts == PRODUCT_XTG ? s.K : s.M; }
int64_t rows_b(int layouts, const ProductShape &s) { return layouts == PRODUCT_GWT ? s.N : s.K; }
// Room for copies of the operands whose width asks for one (a, b: of the M side, of the N side; a backward pass has formed dP itself)
size_t pack_bytes(int layouts, const ProductShape &s, bool a, bool b)
{
    if (!long_product(s)) return 0;
    return (size_t)((a ? packed_bytes(rows_a(layouts, s), width_a(layouts, s)) : 0) +
                    (b ? packed_bytes(rows_b(layouts, s), width_b(layouts, s)) * (s.gated ? 2 : s.segments * s.sets) : 0));
}

typedef unsigned short ushort8 __attribute__((ext_vector_type(8)));
typedef unsigned short ushort8_packed __attribute__((ext_vector_type(8), aligned(2)));

// 8 elements a thread; zeros behind a row's last one
__global__ __launch_bounds__(256) void pack_kernel(const unsigned short *__restrict__ from, int64_t ld, int64_t rows, int32_t width, unsigned short *__restrict__ to,
                                                   int64_t first)
{
    const int64_t units = (width + 7) / 8, at = (first + blockIdx.x) * 256 + threadIdx.x;
    if (at >= units * rows) return;
    const int64_t row = at / units;
    const int32_t col = (int32_t)(at % units) * 8;
    const unsigned short *p = from + row * ld + col;
    ushort8 v;
    if (width - col >= 8) {
        v = *reinterpret_cast<const ushort8_packed *>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < width ? p[i] : (unsigned short)0;
    }
    *reinterpret_cast<ushort8 *>(to + at * 8) = v;
}

int pack(Operand &o, int64_t rows, int64_t width, char *&to, hipStream_t stream)
{
    const int64_t units = (width + 7) / 8 * rows;
    unsigned short *out = reinterpret_cast<unsigned short *>(to);
    const int rc = launch_parts((units + 255) / 256, [&](unsigned first, unsigned count) {
        pack_kernel<<<count, 256, 0, stream>>>(reinterpret_cast<const unsigned short *>(o.p), o.ld, rows, (int32_t)width, out, first);
    });
    o = Operand{to, round_up(width, 8), 1};
    to += packed_bytes(rows, width);
    return rc;
}

// Copies of the operands that need one into `room`.  Not where one that has no room kept (rows that lie oddly though their width is a multiple of 8) needs it too.
int pack_operands(int layouts, const ProductShape &s, ProductArgs &a, char *room, hipStream_t stream)
{
    const int64_t wa = width_a(layouts, s), wb = width_b(layouts, s);
    const int count = s.gated ? 2 : operands(a);
    bool fit = long_product(s);
    for (int i = 0; i < operands(a); ++i) fit = fit && (on_units(a.a[i], wa) || wa % 8);
    for (int i = 0; i < count; ++i) fit = fit && (on_units(a.b[i], wb) || wb % 8);
    if (!fit || aligned_product(layouts, s, a)) return SLICEGCN_OK;
    const Operand first = a.a[0];
    for (int i = 0; i < operands(a); ++i) {
        if (on_units(a.a[i], wa)) continue;
        if (i > 0 && a.a[i].p == first.p) a.a[i] = a.a[0]; // both products of one X
        else if (int rc = pack(a.a[i], rows_a(layouts, s), wa, room, stream)) return rc;
    }
    for (int i = 0; i < count; ++i)
        if (!on_units(a.b[i], wb))
            if (int rc = pack(a.b[i], rows_b(layouts, s), wb, room, stream)) return rc;
    return SLICEGCN_OK;
}

// Whether buffers can read both operands as they lie: their range checks go by words, so no word may hold an element that exists and one that does not
bool on_words(const Operand &o, int32_t type)
{
    return type == SLICEGCN_F32 || ((reinterpret_cast<uintptr_t>(o.p) & 3u) == 0 && o.ld % 2 == 0);
}
bool product_on_words(int layouts, const ProductShape &s, const ProductArgs &a)
{
    for (int i = 0; i < operands(a); ++i)
        if (!on_words(a.a[i], s.type) || !on_words(a.b[i], s.type)) return false;
    if (s.gated && !on_words(a.b[1], s.type)) return false;
    if (s.type == SLICEGCN_F32) return true;
    switch (layouts) {
    case PRODUCT_XW: return s.K % 2 == 0 && s.N % 2 == 0;
    case PRODUCT_GWT: return s.K % 2 == 0;
    default: return s.M % 2 == 0 && s.N % 2 == 0;
    }
}

// partial, room: parts of the workspace, for sums of parts of k and for copies of operands.  first_alone: the first set of two that s describes, without the second
int launch_product(const ProductShape &s, int layouts, int epilogue, ProductArgs &a, void *partial, char *room, hipStream_t stream, bool first_alone = false)
{
    const int32_t type = s.type;
    a.partial = static_cast<float *>(partial);
    if (int rc = pack_operands(layouts, s, a, room, stream)) return rc;
    ProductPlan plan = plan_product(s, aligned_product(layouts, s, a));
    // the tail is of the second set: of 2 t tiles, more than CUS, 2 t mod CUS are no more than t
    if (first_alone) plan.tail = 0;
    a.on_words = product_on_words(layouts, s, a);
    return type == SLICEGCN_F32    ? launch_product_f32(layouts, epilogue, plan, a, stream)
           : type == SLICEGCN_BF16 ? launch_product_bf16(layouts, epilogue, plan, a, stream)
                                   : launch_product_f16(layouts, epilogue, plan, a, stream);
}

// Products of gradients in two terms: the sums of either term's products, whole or in parts of k, are parts that are joined.  Each dW by itself; dX some rows at a time,
// so that the parts stay bounded.  Bound as the products are, of which there are twice as many, and by the parts' bytes: 8192 rows 4096 -> 10240 gated bf16 5.04 ms (one term 2.28; errors of
// dX and dW 0.0017 of their norms, 0.0023), 2.4 M rows 100 -> 256 gelu 3.79 ms (in one sweep and one term 0.96), 2048 rows 64 -> 170 gated 19.3 us (15.8).
int64_t rows_at_once(int64_t n, int32_t w_in)
{
    const int64_t most = MOST_PARTIAL / (8 * (int64_t)w_in) / DIRECT_TILE * DIRECT_TILE;
    return n <= most ? n : most > 0 ? most : DIRECT_TILE;
}
ProductPlan plan_terms(const ProductShape &s, bool aligned)
{
    ProductPlan p = plan_product(s, aligned);
    if (p.kernel == BY_ROWS) p = plan_product(s, false); // strips form whole results alone
    if (p.tail) p.steps_per_split = (int32_t)((s.K + DIRECT_K - 1) / DIRECT_K * s.segments);
    p.tail = p.tail_splits = 0;
    p.bytes = (size_t)round_up(2 * p.splits * s.M * s.N * 4, 256);
    return p;
}
size_t terms_bytes(ProductShape s, int layouts)
{
    s.sets = 1;
    const int64_t rows = s.M;
    if (layouts == PRODUCT_GWT) s.M = rows_at_once(rows, s.N);
    size_t most = 0;
    for (int last = 0; last < 2; ++last) {
        for (int aligned = 0; aligned < 2; ++aligned) {
            const size_t here = plan_terms(s, aligned).bytes;
            most = here > most ? here : most;
        }
        if (s.M == rows || rows % s.M == 0) break;
        s.M = rows % s.M;
    }
    return most;
}
// rest: how far the second term lies behind the first; it is that of the M side of dX (GWT), and of the N side of dW (XTG)
int launch_terms(ProductShape s, int layouts, ProductArgs &all, int64_t rest, void *partial, char *room, hipStream_t stream)
{
    if (int rc = pack_operands(layouts, s, all, room, stream)) return rc;
    const bool dx = layouts == PRODUCT_GWT;
    const auto launch = s.type == SLICEGCN_BF16 ? launch_product_bf16 : launch_product_f16;
    s.sets = 1;
    const int64_t rows = all.M, at_once = dx ? rows_at_once(rows, all.N) : rows;
    for (int set = 0; set < all.sets; ++set) {
        for (int64_t first = 0; first < rows; first += at_once) {
            ProductArgs a = all;
            s.M = a.M = rows - first < at_once ? rows - first : at_once;
            a.sets = 1;
            a.out[0] = all.out[set] + first * all.ldo[set] * 2;
            a.ldo[0] = all.ldo[set];
            if (dx) {
                for (int i = 0; i < a.segments; ++i) a.a[i].p += first * a.a[i].ld * 2;
            } else {
                a.a[0] = all.a[set];
                a.b[0] = all.b[set];
            }
            ProductPlan plan = plan_terms(s, aligned_product(layouts, s, a));
            a.on_words = product_on_words(layouts, s, a);
            plan.stage = SUMS_ALONE;
            for (int term = 0; term < 2; ++term) {
                a.partial = static_cast<float *>(partial) + term * plan.splits * a.M * a.N;
                if (int rc = launch(layouts, EPI_STORE, plan, a, stream)) return rc;
                if (dx) {
                    for (int i = 0; i < a.segments; ++i) a.a[i].p += rest;
                } else {
                    a.b[0].p += rest;
                }
            }
            plan.stage = JOIN_ALONE;
            plan.splits *= 2;
            a.partial = static_cast<float *>(partial);
            if (int rc = launch(layouts, EPI_STORE, plan, a, stream)) return rc;
        }
    }
    return SLICEGCN_OK;
}

// ---- gradients before the activation ----------------------------------------------------------------------------------

// Rows of a backward pass.  GATED: g, u and d = dH give dg, du;  else p (act != none) and d = dY give dg = dP.  dr = residual * d.
struct SlopeArgs {
    Operand g, u, d;
    char *dg, *du, *dr;
    int64_t ldg, ldu, ldr, n;
    int32_t w, lanes; // columns; threads that share a row out
    float residual;
    int64_t rest;    // where not 0: what rounding dg and du leaves, rounded too, goes that many bytes behind them
    double *partial; // column sums of parts of the rows: [part][1 or 2][w], where biases have gradients
    int64_t rows_per_part;
};

constexpr int SLOPE_RUN = 32; // rows that are added in fp32 before they are added in fp64

// Workgroup (x, y): `lanes` accesses of 16 bytes of the rows of part y, 256 / lanes rows at a time and ROWS such turns in flight.  Bound by bytes:
// 8192 rows of 10240 gated bf16 columns 178 us, 4.7 TB/s.
template <class T, bool GATED, int ACT> __global__ __launch_bounds__(256) void slope_kernel(const SlopeArgs a)
{
    constexpr int V = 16 / sizeof(T), Q = GATED ? 2 : 1, ROWS = GATED ? 2 : 4;
    constexpr bool SLOPES = GATED || ACT != SLICEGCN_ACT_NONE;
    __shared__ double sums[Q * V][257];
    const int groups = 256 / a.lanes, lane = threadIdx.x % a.lanes, group = threadIdx.x / a.lanes;
    const int64_t col = ((int64_t)blockIdx.x * a.lanes + lane) * V;
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
    // whole: rows have room for the access, and what is behind the last column (zeros: it was read as zeros) belongs to them
    auto write = [&](char *base, int64_t ld, int64_t row, const float (&v)[V], bool whole) {
        T *p = reinterpret_cast<T *>(base) + row * ld + col;
        if (left >= V || whole) {
            store_vec<T, V>(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i < left) p[i] = (T)v[i];
        }
    };
    if (left > 0) {
        for (int64_t row0 = first + group; row0 < last; row0 += (int64_t)groups * ROWS) {
            float d[ROWS][V], g[ROWS][V], u[ROWS][V];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const int64_t row = row0 + r * groups < last ? row0 + r * groups : row0; // the last turn reads a row again rather than branch
                read(a.d, row, d[r]);
                if (SLOPES) read(a.g, row, g[r]);
                if (GATED) read(a.u, row, u[r]);
            }
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const int64_t row = row0 + r * groups;
                if (row >= last) break;
                float o[Q][V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float y = 0.f, slope = 1.f;
                    if (SLOPES) activated_slope<ACT>(g[r][i], y, slope);
                    o[0][i] = through_slope<ACT>(GATED ? d[r][i] * u[r][i] : d[r][i], SLOPES ? g[r][i] : 0.f, slope);
                    if (GATED) o[Q - 1][i] = d[r][i] * y;
                }
                if (a.dg) write(a.dg, a.ldg, row, o[0], true);
                if (GATED && a.du) write(a.du, a.ldu, row, o[Q - 1], true);
                if constexpr (sizeof(T) == 2)
                    if (a.rest) {
                        float left_over[Q][V];
#pragma unroll
                        for (int q = 0; q < Q; ++q)
#pragma unroll
                            for (int i = 0; i < V; ++i) {
                                const float h = (float)(T)o[q][i];
                                left_over[q][i] = fabsf(h) < INFINITY ? o[q][i] - h : 0.f;
                            }
                        write(a.dg + a.rest, a.ldg, row, left_over[0], true);
                        if (GATED) write(a.du + a.rest, a.ldu, row, left_over[Q - 1], true);
                    }
                if (a.dr) {
#pragma unroll
                    for (int i = 0; i < V; ++i) d[r][i] *= a.residual;
                    write(a.dr, a.ldr, row, d[r], false);
                }
#pragma unroll
                for (int q = 0; q < Q; ++q)
#pragma unroll
                    for (int i = 0; i < V; ++i) run[q][i] += o[q][i];
            }
            if (a.partial && (in_run += ROWS) >= SLOPE_RUN) {
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
    if (!a.partial) return; // the same for the workgroup
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < V; ++i) sums[q * V + i][threadIdx.x] = total[q][i] + (double)run[q][i];
    __syncthreads();
    const int here = a.lanes * V;
    const int64_t col0 = (int64_t)blockIdx.x * here;
    for (int o = threadIdx.x; o < Q * here; o += 256) {
        const int q = o / here, c = o % here;
        if (col0 + c >= a.w) continue;
        double t = 0.0;
        for (int w = 0; w < groups; ++w) t += sums[q * V + c % V][w * a.lanes + c / V];
        a.partial[((int64_t)blockIdx.y * Q + q) * a.w + col0 + c] = t;
    }
}

__global__ __launch_bounds__(1024) void bias_kernel(const BiasSums b)
{
    __shared__ double sums[1024 + 1024 / BIAS_COLS];
    bias_sums<1024>(b, blockIdx.x, sums);
}

int launch_bias(const BiasSums &b, hipStream_t stream)
{
    if (!b.partial) return SLICEGCN_OK;
    bias_kernel<<<(unsigned)bias_workgroups(b), 1024, 0, stream>>>(b);
    SG_LAUNCH_CHECK();
    return SLICEGCN_OK;
}

struct SlopeGrid {
    int32_t lanes;
    int64_t cols, parts; // workgroups
};

SlopeGrid slope_grid(int64_t n, int32_t w, int32_t type)
{
    const int64_t accesses = ((int64_t)w * type_bytes(type) + 15) / 16;
    SlopeGrid g;
    g.lanes = 1;
    while (g.lanes < 64 && g.lanes < accesses) g.lanes *= 2;
    g.cols = (accesses + g.lanes - 1) / g.lanes;
    const int64_t rows = 256 / g.lanes;
    // eight workgroups a CU where a thread has eight rows or more then, else two (each leaves column sums): 16 k rows 512 -> 512 gated bf16 with biases 99 us, with eight 113; 100 k
    // rows 256 -> 688 495 and 460
    const int64_t most = (8 * CUS + g.cols - 1) / g.cols, few = (2 * CUS + g.cols - 1) / g.cols, long_ones = n / (8 * rows);
    g.parts = long_ones > few ? long_ones : few;
    if (g.parts > most) g.parts = most;
    if (g.parts > (n + rows - 1) / rows) g.parts = (n + rows - 1) / rows;
    if (g.parts < 1) g.parts = 1;
    return g;
}

// Whether a backward pass may go in one sweep over the rows, by its sizes, and with how many workgroups (0: it may not).  Many rows, since every workgroup leaves a
// dW of its own: 100 -> 256 columns bf16 gelu, 8192 rows 30 us, 22 in the general form; 16384 rows 28 and 37; 2.4 M rows 0.95 and 1.83 ms.
// Each has at most CHAIN blocks of rows, so that its sums are as short as those of the other forms: one workgroup a CU up to 8.4 M rows, then some each.
constexpr int64_t NARROW_LEAST = 16384;
unsigned narrow_blocks(int64_t n, int32_t w_in, int32_t w_out, int32_t type, int q)
{
    if (type == SLICEGCN_F32 || w_in > NARROW_WIDTH_IN || w_out * q > NARROW_WIDTH_OUT || w_in % 2 || w_out % 2 || n < NARROW_LEAST) return 0;
    const int64_t rows = CHAIN * NARROW_ROWS * CUS;
    return (unsigned)((n + rows - 1) / rows * CUS);
}
// ... and by how its rows lie: on boundaries of 4 bytes
bool narrow_rows_fit(const Operand &o) { return !o.p || ((reinterpret_cast<uintptr_t>(o.p) & 3u) == 0 && o.ld % 2 == 0); }

// Workspace of a backward pass: gradients before the activation, their column sums, sums of parts of k
struct BwdWorkspace {
    int64_t ld; // of the gradients before the activation: rows on 16-byte boundaries
    int terms;  // of them
    size_t rows, sums, partial, room;
    size_t bytes(int q) const { return terms * q * rows + sums + partial + room; }
};

ProductShape dx_shape(int64_t n, int32_t w_in, int32_t w_out, int32_t type, int q) { return ProductShape{n, w_out, w_in, q, 1, type, false, true}; }
ProductShape dw_shape(int64_t n, int32_t w_in, int32_t w_out, int32_t type, int q) { return ProductShape{w_in, n, w_out, 1, q, type, false, false}; }

BwdWorkspace bwd_workspace(int64_t n, int32_t w_in, int32_t w_out, int32_t type, int q, bool two)
{
    BwdWorkspace w;
    w.ld = round_up(w_out, 8);
    w.terms = terms_of(n, w_in, w_out, type, q, two);
    w.rows = (size_t)round_up(n * w.ld * type_bytes(type), 256);
    const int64_t parts = slope_grid(n, w_out, type).parts, blocks = narrow_blocks(n, w_in, w_out, type, q);
    w.sums = (size_t)round_up((parts > blocks ? parts : blocks) * q * (int64_t)w_out * 8, 256);
    const size_t x = partial_bytes(dx_shape(n, w_in, w_out, type, q)), y = partial_bytes(dw_shape(n, w_in, w_out, type, q));
    const size_t z = (size_t)round_up(blocks * q * w_in * (int64_t)w_out * 4, 256);
    w.partial = x > y ? x : y;
    w.partial = w.partial > z ? w.partial : z;
    if (paired(n, w_in, w_out, type, q)) {
        const size_t both = w.terms * (pair_plan(dx_shape(n, w_in, w_out, type, q)).bytes + pair_plan(dw_shape(n, w_in, w_out, type, q)).bytes);
        w.partial = w.partial > both ? w.partial : both;
    } else if (w.terms == 2) {
        const size_t a = terms_bytes(dx_shape(n, w_in, w_out, type, q), PRODUCT_GWT), b = terms_bytes(dw_shape(n, w_in, w_out, type, q), PRODUCT_XTG);
        w.partial = w.partial > a ? w.partial : a;
        w.partial = w.partial > b ? w.partial : b;
    }
    const size_t u = pack_bytes(PRODUCT_GWT, dx_shape(n, w_in, w_out, type, q), false, true), v = pack_bytes(PRODUCT_XTG, dw_shape(n, w_in, w_out, type, q), true, false);
    w.room = u > v ? u : v;
    return w;
}

// The kernels count k in 32 bits, up to some steps behind the last one: n is the k of dW
constexpr int64_t MOST_ROWS = ((int64_t)1 << 31) - (1 << 16);
bool sizes_fit(int64_t n, int32_t w_in, int32_t w_out) { return n >= 0 && n <= MOST_ROWS && w_in >= 1 && w_out >= 1 && w_in <= 1 << 20 && w_out <= 1 << 20; }

// The type of the elements alone
int32_t one_type(int32_t type) { return type & ~SLICEGCN_TWO_TERMS; }
slicegcn_product_desc of_one_type(slicegcn_product_desc d)
{
    d.type = one_type(d.type);
    return d;
}

int check(const char *what, const slicegcn_product_desc *d, const void *io)
{
    SG_REQUIRE(d && io, SLICEGCN_EINVAL, "%s: NULL descriptor or io", what);
    SG_REQUIRE(d->n >= 0 && d->w_in >= 1 && d->w_out >= 1, SLICEGCN_EINVAL, "%s: need n >= 0 and widths >= 1", what);
    SG_REQUIRE(known_type(one_type(d->type)), SLICEGCN_EINVAL, "%s: unknown type", what);
    SG_REQUIRE(d->act >= SLICEGCN_ACT_NONE && d->act <= SLICEGCN_ACT_GELU, SLICEGCN_EINVAL, "%s: unknown activation", what);
    SG_REQUIRE(std::isfinite((float)d->residual), SLICEGCN_EINVAL, "%s: residual is not finite", what);
    SG_REQUIRE(sizes_fit(d->n, d->w_in, d->w_out), SLICEGCN_ERANGE, "%s: n or a width too large", what);
    return SLICEGCN_OK;
}

constexpr int64_t MOST_LD = 1 << 21; // offsets within a tile fit 31 bits
int check_rows(const char *what, const char *name, const slicegcn_matrix &m, int64_t n, int32_t width, int32_t type, bool needed)
{
    SG_REQUIRE(!needed || m.data, SLICEGCN_EINVAL, "%s: NULL %s", what, name);
    SG_REQUIRE(!m.data || (m.ld >= width && aligned_for(m.data, type)), SLICEGCN_EINVAL, "%s: %s has an ld smaller than its width, or a misaligned base", what, name);
    SG_REQUIRE(!m.data || n <= 1 || m.ld <= MOST_LD, SLICEGCN_ERANGE, "%s: %s has an ld beyond 2^21", what, name);
    return SLICEGCN_OK;
}

// Outputs at the address of another operand (of any part of them an output may overlap nothing, but that is the caller's)
int check_apart(const char *what, std::initializer_list<const void *> outputs, std::initializer_list<const void *> inputs)
{
    for (auto o = outputs.begin(); o != outputs.end(); ++o) {
        if (!*o) continue;
        for (auto p = o + 1; p != outputs.end(); ++p) SG_REQUIRE(*o != *p, SLICEGCN_EINVAL, "%s: two outputs at one address", what);
        for (const void *i : inputs) SG_REQUIRE(*o != i, SLICEGCN_EINVAL, "%s: an output at the address of an input", what);
    }
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

// One row alone (the last token of a long sequence, say) may be said to be any distance from a next one that does not exist
int64_t ld_of(const slicegcn_matrix &m, int32_t width) { return m.ld <= MOST_LD ? m.ld : width; }
Operand operand(const slicegcn_matrix &m, int32_t width) { return Operand{static_cast<const char *>(m.data), ld_of(m, width), 0}; }
Operand weights(const void *w, int32_t w_out) { return Operand{static_cast<const char *>(w), w_out, 0}; }

ProductShape fwd_shape(int64_t n, int32_t w_in, int32_t w_out, int32_t type, bool gated) { return ProductShape{n, w_in, w_out, 1, 1, type, gated, true}; }

size_t fwd_bytes(const ProductShape &s) { return partial_bytes(s) + pack_bytes(PRODUCT_XW, s, true, true); }

// Both backward passes.  q = 2: gated
struct BwdCall {
    const slicegcn_product_desc *d;
    bool two; // whether the caller asks for two terms
    Operand x, w[2], g, u, dy;
    slicegcn_matrix dx, dr;
    void *dw[2];
    float *db[2];
};

int backward(const char *what, const BwdCall &c, int q, void *ws, size_t ws_bytes, hipStream_t stream)
{
    const slicegcn_product_desc &d = *c.d;
    const bool two = c.two && d.type != SLICEGCN_F32 && (q == 2 || d.act != SLICEGCN_ACT_NONE); // else dP is whole in one
    const BwdWorkspace w = bwd_workspace(d.n, d.w_in, d.w_out, d.type, q, two);
    if (int rc = check_workspace(what, ws, ws_bytes, w.bytes(q))) return rc;
    const bool want_x = c.dx.data && d.n > 0, want_w = c.dw[0] || c.dw[1], want_b = c.db[0] || c.db[1], want_r = c.dr.data && d.n > 0;
    char *at = static_cast<char *>(ws);
    // without an activation dP is dY itself, or a copy of it where its rows are no whole units and the products gain from that
    const bool plain = q == 1 && d.act == SLICEGCN_ACT_NONE &&
                       (on_units(c.dy, d.w_out) || !(long_product(dx_shape(d.n, d.w_in, d.w_out, d.type, q)) || long_product(dw_shape(d.n, d.w_in, d.w_out, d.type, q))));
    Operand dg[2] = {c.dy, c.dy};
    SlopeArgs s{};
    s.g = q == 1 && d.act == SLICEGCN_ACT_NONE ? Operand{nullptr, 0, 0} : c.g;
    s.u = c.u;
    s.d = c.dy;
    s.n = d.n;
    s.w = d.w_out;
    s.residual = (float)d.residual;
    if (!plain && (want_x || want_w)) {
        s.dg = at;
        s.ldg = s.ldu = w.ld;
        if (q == 2) s.du = at + w.rows;
        dg[0] = Operand{s.dg, w.ld, 1};
        dg[1] = Operand{s.du, w.ld, 1};
        s.rest = w.terms == 2 ? (int64_t)(q * w.rows) : 0;
    }
    if (want_r) {
        s.dr = static_cast<char *>(c.dr.data);
        s.ldr = c.dr.ld;
    }
    at += w.terms * q * w.rows;
    if (want_b) s.partial = reinterpret_cast<double *>(at);
    at += w.sums;
    float *partial = reinterpret_cast<float *>(at);
    char *room = at + w.partial;

    ProfScope prof(SLICEGCN_PROF_PRODUCT, d.w_out, stream);
    const Operand dx{static_cast<const char *>(c.dx.data), c.dx.ld, 0};
    const unsigned narrow = narrow_blocks(d.n, d.w_in, d.w_out, d.type, q);
    if (narrow && !two && (want_x || want_w) && !want_r && narrow_rows_fit(c.x) && narrow_rows_fit(c.g) && narrow_rows_fit(c.u) && narrow_rows_fit(c.dy) &&
        narrow_rows_fit(dx)) {
        NarrowArgs a{};
        a.x = c.x;
        a.w[0] = c.w[0];
        a.w[1] = c.w[1];
        a.g = c.g;
        a.u = c.u;
        a.d = c.dy;
        a.dx = want_x ? static_cast<char *>(c.dx.data) : nullptr;
        a.lddx = c.dx.ld;
        a.n = d.n;
        a.w_in = d.w_in;
        a.w_out = d.w_out;
        a.want_w = want_w;
        a.partial = partial;
        a.columns = s.partial;
        // one of two dW alone: the sums of both are formed, and its are joined
        ProductArgs join{};
        join.partial = c.dw[0] ? partial : partial + (int64_t)narrow * d.w_in * d.w_out;
        for (int i = 0; i < q; ++i) {
            if (!c.dw[i]) continue;
            join.out[join.sets] = static_cast<char *>(c.dw[i]);
            join.ldo[join.sets++] = d.w_out;
        }
        join.M = d.w_in;
        join.N = d.w_out;
        join.splits = (int32_t)narrow;
        const auto launch = d.type == SLICEGCN_BF16 ? launch_narrow_bf16 : launch_narrow_f16;
        if (int rc = launch(a, join, d.act, q == 2, narrow, stream)) return rc;
        return launch_bias(BiasSums{s.partial, (int32_t)narrow, q, d.w_out, {c.db[0], c.db[1]}}, stream);
    }
    BiasSums bias{};
    if (s.dg || s.dr || s.partial) {
        const SlopeGrid g = slope_grid(d.n, d.w_out, d.type);
        s.lanes = g.lanes;
        s.rows_per_part = (d.n + g.parts - 1) / g.parts;
        const dim3 grid((unsigned)g.cols, (unsigned)g.parts);
        with_type(d.type, [&](auto t) {
            with_act(s.g.p ? d.act : SLICEGCN_ACT_NONE, [&](auto act) {
                if (q == 2) slope_kernel<decltype(t), true, decltype(act)::value><<<grid, 256, 0, stream>>>(s);
                else slope_kernel<decltype(t), false, decltype(act)::value><<<grid, 256, 0, stream>>>(s);
            });
        });
        SG_LAUNCH_CHECK();
        bias = BiasSums{s.partial, (int32_t)g.parts, q, d.w_out, {c.db[0], c.db[1]}};
    }
    const ProductShape shape_x = dx_shape(d.n, d.w_in, d.w_out, d.type, q), shape_w = dw_shape(d.n, d.w_in, d.w_out, d.type, q);
    ProductArgs x{}, y{};
    if (want_x) {
        for (int i = 0; i < q; ++i) {
            x.a[i] = dg[i];
            x.b[i] = c.w[i];
        }
        x.M = d.n;
        x.K = d.w_out;
        x.N = d.w_in;
        x.segments = q;
        x.sets = 1;
        x.out[0] = static_cast<char *>(c.dx.data);
        x.ldo[0] = c.dx.ld;
    }
    if (want_w) {
        for (int i = 0; i < q; ++i) {
            if (!c.dw[i]) continue;
            y.a[y.sets] = c.x;
            y.b[y.sets] = dg[i];
            y.out[y.sets] = static_cast<char *>(c.dw[i]);
            y.ldo[y.sets++] = d.w_out;
        }
        y.M = d.w_in;
        y.K = d.n;
        y.N = d.w_out;
        y.segments = 1;
    }
    // one of two dW alone is cut like both, so that the workspace suffices and its bits are the same
    if (paired(d.n, d.w_in, d.w_out, d.type, q)) {
        x.on_words = !want_x || product_on_words(PRODUCT_GWT, shape_x, x);
        y.on_words = !want_w || product_on_words(PRODUCT_XTG, shape_w, y);
        const ProductPlan px = pair_plan(shape_x), pw = pair_plan(shape_w);
        const int terms = s.rest ? 2 : 1;
        x.splits = terms * px.splits;
        x.steps_per_split = px.steps_per_split;
        x.partial = partial;
        y.splits = terms * pw.splits;
        y.steps_per_split = pw.steps_per_split;
        y.partial = partial + terms * px.bytes / 4;
        x.terms = y.terms = terms;
        x.rest_a = y.rest_b = s.rest;
        const auto launch = d.type == SLICEGCN_F32 ? launch_pair_f32 : d.type == SLICEGCN_BF16 ? launch_pair_bf16 : launch_pair_f16;
        return launch(want_x ? &x : nullptr, want_w ? &y : nullptr, bias, stream);
    }
    if (int rc = launch_bias(bias, stream)) return rc;
    if (s.rest) {
        if (want_x)
            if (int rc = launch_terms(shape_x, PRODUCT_GWT, x, s.rest, partial, room, stream)) return rc;
        return want_w ? launch_terms(shape_w, PRODUCT_XTG, y, s.rest, partial, room, stream) : SLICEGCN_OK;
    }
    if (want_x)
        if (int rc = launch_product(shape_x, PRODUCT_GWT, EPI_STORE, x, partial, room, stream)) return rc;
    if (want_w)
        if (int rc = launch_product(shape_w, PRODUCT_XTG, EPI_STORE, y, partial, room, stream, q == 2 && !c.dw[1])) return rc;
    return SLICEGCN_OK;
}

} // namespace
} // namespace slicegcn

using namespace slicegcn;

extern "C" size_t slicegcn_product_fwd_workspace_bytes(int64_t n, int32_t w_in, int32_t w_out, int32_t type)
{
    if (!sizes_fit(n, w_in, w_out) || !known_type(one_type(type)) || n == 0) return 0;
    return fwd_bytes(fwd_shape(n, w_in, w_out, one_type(type), false));
}

extern "C" int slicegcn_product_fwd(const slicegcn_product_desc *desc, const slicegcn_product_io *io, void *ws, size_t ws_bytes, void *stream)
{
    const char *what = "product_fwd";
    if (int rc = check(what, desc, io)) return rc;
    const slicegcn_product_desc one = of_one_type(*desc), *d = &one;
    SG_REQUIRE(io->W, SLICEGCN_EINVAL, "%s: NULL W", what);
    if (int rc = check_rows(what, "X", io->X, d->n, d->w_in, d->type, true)) return rc;
    if (int rc = check_rows(what, "Y", io->Y, d->n, d->w_out, d->type, true)) return rc;
    if (int rc = check_rows(what, "R", io->R, d->n, d->w_out, d->type, false)) return rc;
    if (int rc = check_rows(what, "P", io->P, d->n, d->w_out, d->type, false)) return rc;
    if (int rc = check_params(what, d->type, {io->W}, {io->b})) return rc;
    if (d->n == 0) return SLICEGCN_OK;
    if (int rc = check_apart(what, {io->Y.data, io->P.data}, {io->X.data, io->W, io->b})) return rc;
    if (int rc = check_apart(what, {io->P.data}, {io->R.data})) return rc;
    SG_REQUIRE(io->Y.data != io->R.data || io->Y.ld == io->R.ld, SLICEGCN_EINVAL, "%s: Y in the rows of R with another ld", what);
    const ProductShape shape = fwd_shape(d->n, d->w_in, d->w_out, d->type, false);
    if (int rc = check_workspace(what, ws, ws_bytes, fwd_bytes(shape))) return rc;
    ProductArgs a{};
    a.a[0] = operand(io->X, d->w_in);
    a.b[0] = weights(io->W, d->w_out);
    a.M = d->n;
    a.K = d->w_in;
    a.N = d->w_out;
    a.segments = a.sets = 1;
    a.out[0] = static_cast<char *>(io->Y.data);
    a.ldo[0] = ld_of(io->Y, d->w_out);
    a.bias[0] = io->b;
    a.r = operand(io->R, d->w_out);
    a.keep[0] = static_cast<char *>(io->P.data);
    a.ldk[0] = ld_of(io->P, d->w_out);
    a.residual = (float)d->residual;
    a.act = d->act;
    ProfScope prof(SLICEGCN_PROF_PRODUCT, d->w_out, as_stream(stream));
    return launch_product(shape, PRODUCT_XW, EPI_FORWARD, a, ws, static_cast<char *>(ws) + partial_bytes(shape), as_stream(stream));
}

extern "C" size_t slicegcn_product_bwd_workspace_bytes(int64_t n, int32_t w_in, int32_t w_out, int32_t type)
{
    if (!sizes_fit(n, w_in, w_out) || !known_type(one_type(type))) return 0;
    return bwd_workspace(n, w_in, w_out, one_type(type), 1, type != one_type(type)).bytes(1);
}

extern "C" int slicegcn_product_bwd(const slicegcn_product_desc *desc, const slicegcn_product_io *io, void *ws, size_t ws_bytes, void *stream)
{
    const char *what = "product_bwd";
    if (int rc = check(what, desc, io)) return rc;
    const slicegcn_product_desc one = of_one_type(*desc), *d = &one;
    const bool rows = d->n > 0, slope = d->act != SLICEGCN_ACT_NONE && (io->dX.data || io->dW || io->db);
    if (int rc = check_rows(what, "X", io->X, d->n, d->w_in, d->type, rows && io->dW)) return rc;
    if (int rc = check_rows(what, "P", io->P, d->n, d->w_out, d->type, rows && slope)) return rc;
    if (int rc = check_rows(what, "dY", io->dY, d->n, d->w_out, d->type, rows)) return rc;
    if (int rc = check_rows(what, "dX", io->dX, d->n, d->w_in, d->type, false)) return rc;
    if (int rc = check_rows(what, "dR", io->dR, d->n, d->w_out, d->type, false)) return rc;
    SG_REQUIRE(io->W || !io->dX.data || !rows, SLICEGCN_EINVAL, "%s: NULL W", what);
    if (int rc = check_params(what, d->type, {io->W, io->dW}, {io->db})) return rc;
    if (rows)
        if (int rc = check_apart(what, {io->dX.data, io->dW, io->db, io->dR.data}, {io->X.data, io->W, io->P.data, io->dY.data})) return rc;
    BwdCall c{};
    c.d = d;
    c.two = desc->type != d->type;
    c.x = operand(io->X, d->w_in);
    c.w[0] = weights(io->W, d->w_out);
    c.g = operand(io->P, d->w_out);
    c.dy = operand(io->dY, d->w_out);
    c.dx = slicegcn_matrix{io->dX.data, ld_of(io->dX, d->w_in)};
    c.dr = slicegcn_matrix{io->dR.data, ld_of(io->dR, d->w_out)};
    c.dw[0] = io->dW;
    c.db[0] = io->db;
    return backward(what, c, 1, ws, ws_bytes, as_stream(stream));
}

extern "C" size_t slicegcn_gated_fwd_workspace_bytes(int64_t n, int32_t w_in, int32_t w_out, int32_t type)
{
    if (!sizes_fit(n, w_in, w_out) || !known_type(one_type(type)) || n == 0) return 0;
    return fwd_bytes(fwd_shape(n, w_in, w_out, one_type(type), true));
}

extern "C" int slicegcn_gated_fwd(const slicegcn_product_desc *desc, const slicegcn_gated_io *io, void *ws, size_t ws_bytes, void *stream)
{
    const char *what = "gated_fwd";
    if (int rc = check(what, desc, io)) return rc;
    const slicegcn_product_desc one = of_one_type(*desc), *d = &one;
    SG_REQUIRE(io->Wg && io->Wu, SLICEGCN_EINVAL, "%s: NULL Wg or Wu", what);
    if (int rc = check_rows(what, "X", io->X, d->n, d->w_in, d->type, true)) return rc;
    if (int rc = check_rows(what, "H", io->H, d->n, d->w_out, d->type, true)) return rc;
    if (int rc = check_rows(what, "G", io->G, d->n, d->w_out, d->type, false)) return rc;
    if (int rc = check_rows(what, "U", io->U, d->n, d->w_out, d->type, false)) return rc;
    SG_REQUIRE(!io->G.data == !io->U.data, SLICEGCN_EINVAL, "%s: G without U, or U without G", what);
    if (int rc = check_params(what, d->type, {io->Wg, io->Wu}, {io->bg, io->bu})) return rc;
    if (d->n == 0) return SLICEGCN_OK;
    if (int rc = check_apart(what, {io->H.data, io->G.data, io->U.data}, {io->X.data, io->Wg, io->Wu, io->bg, io->bu})) return rc;
    const ProductShape shape = fwd_shape(d->n, d->w_in, d->w_out, d->type, true);
    if (int rc = check_workspace(what, ws, ws_bytes, fwd_bytes(shape))) return rc;
    ProductArgs a{};
    a.a[0] = operand(io->X, d->w_in);
    a.b[0] = weights(io->Wg, d->w_out);
    a.b[1] = weights(io->Wu, d->w_out);
    a.M = d->n;
    a.K = d->w_in;
    a.N = d->w_out;
    a.segments = a.sets = 1;
    a.out[0] = static_cast<char *>(io->H.data);
    a.ldo[0] = ld_of(io->H, d->w_out);
    a.bias[0] = io->bg;
    a.bias[1] = io->bu;
    a.keep[0] = static_cast<char *>(io->G.data);
    a.ldk[0] = ld_of(io->G, d->w_out);
    a.keep[1] = static_cast<char *>(io->U.data);
    a.ldk[1] = ld_of(io->U, d->w_out);
    a.act = d->act;
    ProfScope prof(SLICEGCN_PROF_PRODUCT, d->w_out, as_stream(stream));
    return launch_product(shape, PRODUCT_XW, EPI_GATED, a, ws, static_cast<char *>(ws) + partial_bytes(shape), as_stream(stream));
}

extern "C" size_t slicegcn_gated_bwd_workspace_bytes(int64_t n, int32_t w_in, int32_t w_out, int32_t type)
{
    if (!sizes_fit(n, w_in, w_out) || !known_type(one_type(type))) return 0;
    return bwd_workspace(n, w_in, w_out, one_type(type), 2, type != one_type(type)).bytes(2);
}

extern "C" int slicegcn_gated_bwd(const slicegcn_product_desc *desc, const slicegcn_gated_io *io, void *ws, size_t ws_bytes, void *stream)
{
    const char *what = "gated_bwd";
    if (int rc = check(what, desc, io)) return rc;
    const slicegcn_product_desc one = of_one_type(*desc), *d = &one;
    const bool rows = d->n > 0;
    if (int rc = check_rows(what, "X", io->X, d->n, d->w_in, d->type, rows && (io->dWg || io->dWu))) return rc;
    if (int rc = check_rows(what, "G", io->G, d->n, d->w_out, d->type, rows)) return rc;
    if (int rc = check_rows(what, "U", io->U, d->n, d->w_out, d->type, rows)) return rc;
    if (int rc = check_rows(what, "dH", io->dH, d->n, d->w_out, d->type, rows)) return rc;
    if (int rc = check_rows(what, "dX", io->dX, d->n, d->w_in, d->type, false)) return rc;
    SG_REQUIRE((io->Wg && io->Wu) || !io->dX.data || !rows, SLICEGCN_EINVAL, "%s: NULL Wg or Wu", what);
    if (int rc = check_params(what, d->type, {io->Wg, io->Wu, io->dWg, io->dWu}, {io->dbg, io->dbu})) return rc;
    if (rows)
        if (int rc = check_apart(what, {io->dX.data, io->dWg, io->dWu, io->dbg, io->dbu}, {io->X.data, io->Wg, io->Wu, io->G.data, io->U.data, io->dH.data})) return rc;
    BwdCall c{};
    c.d = d;
    c.two = desc->type != d->type;
    c.x = operand(io->X, d->w_in);
    c.w[0] = weights(io->Wg, d->w_out);
    c.w[1] = weights(io->Wu, d->w_out);
    c.g = operand(io->G, d->w_out);
    c.u = operand(io->U, d->w_out);
    c.dy = operand(io->dH, d->w_out);
    c.dx = slicegcn_matrix{io->dX.data, ld_of(io->dX, d->w_in)};
    c.dw[0] = io->dWg;
    c.dw[1] = io->dWu;
    c.db[0] = io->dbg;
    c.db[1] = io->dbu;
    return backward(what, c, 2, ws, ws_bytes, as_stream(stream));
}
