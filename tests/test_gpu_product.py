"""Products with their epilogue and gated projections, forward and backward, against 64-bit references."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from product_util import ACTS, gated_bwd, gated_fwd, product_bwd, product_fwd
from train_util import F64, TYPES, assert_within, rows

pytestmark = pytest.mark.gpu
ACT = dict(none=B.ACT_NONE, relu=B.ACT_RELU, silu=B.ACT_SILU, gelu=B.ACT_GELU)

# rows, widths: single elements, less than a tile, whole tiles, one more, long sums that are cut, many rows
SIZES = [(1, 1, 1), (1, 64, 96), (1, 2000, 136), (2, 300, 1032), (3, 7, 5), (5, 1048, 40), (9, 520, 264), (17, 33, 31), (24, 1024, 200), (32, 128, 256),
         (33, 65, 129), (70, 2304, 64), (128, 64, 64), (200, 130, 70), (257, 520, 384), (300, 264, 520), (1000, 72, 40), (5000, 24, 8), (1, 8, 8), (64, 32, 16),
         # rows and columns in whole units of 16 bytes, tiles of 256: less than one, sums of one step, of an odd number, cut sums, ends within a step
         (129, 8, 72), (256, 64, 256), (300, 40, 72), (513, 1000, 776), (130, 2056, 136), (1040, 96, 264),
         # few rows of such operands: strips of 64 columns, k shared out among wavefronts and cut, more wavefronts than steps
         (1, 4104, 136), (16, 40, 64), (17, 2304, 72), (31, 5000, 24), (40, 264, 96), (64, 4096, 64), (65, 72, 200), (100, 2600, 136), (128, 1000, 40)]


def weights(gen, w_in, w_out, dtype):
    w = (torch.randn((w_in, w_out), generator=gen) / w_in ** 0.5).to(dtype)
    return w.cuda(), w.to(F64)


def vector(gen, width, present):
    if not present:
        return None, None
    v = torch.randn(width, generator=gen)
    return v.cuda(), v.to(F64)


def result(n, width, dtype, ld):
    """Rows that lie ld apart in a buffer of a value that no result has, and the buffer."""
    buf = torch.full((n, ld), 777.0, dtype=dtype, device="cuda")
    return buf[:, :width], buf


def assert_padding(buf, width):
    assert (buf[:, width:] == 777.0).all(), "written behind the last column"


def workspace(count):
    return torch.full((count,), 0xFF, dtype=torch.uint8, device="cuda")  # NaN in every type


def lds(n, w, kind):
    return {"dense": w, "lines": -(-w // 64) * 64, "odd": w + 3}[kind]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("name", ACTS)
def test_product(size, name, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    case = SIZES.index(size) + ACTS.index(name)
    gen = torch.Generator().manual_seed(case)
    ld = ("dense", "lines", "odd")[case % 3]
    offset = (0, 8, 1)[case % 3]
    residual, with_r, with_b, with_p = (1.0, 0.5, 0.0, -2.0)[case % 4], case % 2 == 0, case % 3 != 1, case % 2 == 1 or name != "none"
    x, x64 = rows(gen, n, wi, dtype, lds(n, wi, ld), offset)
    w, w64 = weights(gen, wi, wo, dtype)
    b, b64 = vector(gen, wo, with_b)
    r, r64 = rows(gen, n, wo, dtype, lds(n, wo, ld), offset) if with_r else (None, None)
    y, ybuf = result(n, wo, dtype, lds(n, wo, ld))
    p, pbuf = result(n, wo, dtype, lds(n, wo, "odd")) if with_p else (None, None)
    ws = workspace(B.slicegcn_product_fwd_workspace_bytes(n, wi, wo, dtype))
    B.slicegcn_product_fwd(x, w, y, ws, b=b, R=r, P=p, act=ACT[name], residual=residual)
    want = product_fwd(x64, w64, b64, r64, residual, name, dtype)
    assert_within(y, *want["Y"], "Y")
    assert_padding(ybuf, wo)
    if with_p:
        assert_within(p, *want["P"], "P")
        assert_padding(pbuf, wo)

    kept, k64 = rows(gen, n, wo, dtype, lds(n, wo, ld), offset, std=1.5)
    dy, d64 = rows(gen, n, wo, dtype, lds(n, wo, ld), offset)
    dx, dxbuf = result(n, wi, dtype, lds(n, wi, ld))
    dr, drbuf = result(n, wo, dtype, lds(n, wo, "odd"))
    dw, db = torch.full_like(w, 777.0), torch.full((wo,), 777.0, device="cuda")
    ws = workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype))
    B.slicegcn_product_bwd(x, w, kept if name != "none" else None, dy, ws, dX=dx, dW=dw, db=db, dR=dr, act=ACT[name], residual=residual)
    want = product_bwd(x64, w64, k64, d64, residual, name, dtype)
    for got, key in ((dx, "dX"), (dw, "dW"), (db, "db"), (dr, "dR")):
        assert_within(got, *want[key], key)
    assert_padding(dxbuf, wi)
    assert_padding(drbuf, wo)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("name", ACTS)
def test_gated(size, name, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    case = SIZES.index(size) + 2 * ACTS.index(name)
    gen = torch.Generator().manual_seed(100 + case)
    ld = ("dense", "lines", "odd")[case % 3]
    offset = (0, 8, 1)[case % 3]
    x, x64 = rows(gen, n, wi, dtype, lds(n, wi, ld), offset)
    (wg, wg64), (wu, wu64) = weights(gen, wi, wo, dtype), weights(gen, wi, wo, dtype)
    bg, bg64 = vector(gen, wo, case % 2 == 0)
    bu, bu64 = vector(gen, wo, case % 3 == 0)
    h, hbuf = result(n, wo, dtype, lds(n, wo, ld))
    (g, gbuf), (u, ubuf) = (result(n, wo, dtype, lds(n, wo, k)) if case % 4 else (None, None) for k in ("odd", ld))
    ws = workspace(B.slicegcn_gated_fwd_workspace_bytes(n, wi, wo, dtype))
    B.slicegcn_gated_fwd(x, wg, wu, h, ws, bg=bg, bu=bu, G=g, U=u, act=ACT[name])
    want = gated_fwd(x64, wg64, wu64, bg64, bu64, name, dtype)
    for got, buf, key in ((h, hbuf, "H"), (g, gbuf, "G"), (u, ubuf, "U")):
        if got is not None:
            assert_within(got, *want[key], key)
            assert_padding(buf, wo)

    g, g64 = rows(gen, n, wo, dtype, lds(n, wo, ld), offset, std=1.5)
    u, u64 = rows(gen, n, wo, dtype, lds(n, wo, "odd"), offset)
    dh, d64 = rows(gen, n, wo, dtype, lds(n, wo, ld), offset)
    dx, dxbuf = result(n, wi, dtype, lds(n, wi, ld))
    dwg, dwu = torch.full_like(wg, 777.0), torch.full_like(wu, 777.0)
    dbg, dbu = (torch.full((wo,), 777.0, device="cuda") for _ in range(2))
    ws = workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype))
    B.slicegcn_gated_bwd(x, wg, wu, g, u, dh, ws, dX=dx, dWg=dwg, dWu=dwu, dbg=dbg, dbu=dbu, act=ACT[name])
    want = gated_bwd(x64, wg64, wu64, g64, u64, d64, name, dtype)
    for got, key in ((dx, "dX"), (dwg, "dWg"), (dwu, "dWu"), (dbg, "dbg"), (dbu, "dbu")):
        assert_within(got, *want[key], key)
    assert_padding(dxbuf, wi)


@pytest.mark.parametrize("size", [(40, 24, 16), (3, 600, 48), (700, 40, 136)], ids=str)
@pytest.mark.parametrize("kind", TYPES)
def test_gradients_that_are_not_wanted(size, kind):
    """Each gradient alone, in the bits that it has among all of them."""
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(7)
    x, g, u, dh = (rows(gen, n, w, dtype)[0] for w in (wi, wo, wo, wo))
    (wg, _), (wu, _) = weights(gen, wi, wo, dtype), weights(gen, wi, wo, dtype)
    ws = workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype))
    empty = dict(dX=(n, wi), dWg=(wi, wo), dWu=(wi, wo), dbg=(wo,), dbu=(wo,))
    make = lambda names: {k: torch.full(empty[k], 777.0, dtype=torch.float32 if k in ("dbg", "dbu") else dtype, device="cuda") for k in names}
    every = make(empty)
    B.slicegcn_gated_bwd(x, wg, wu, g, u, dh, ws, **every)
    for k in empty:
        alone = make([k])
        needed = dict(X=x if k in ("dWg", "dWu") else None)
        B.slicegcn_gated_bwd(needed["X"], wg, wu, g, u, dh, ws, **alone)
        assert torch.equal(alone[k], every[k]), k
    ws = workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype))
    every = {k: torch.full(s, 777.0, dtype=torch.float32 if k == "db" else dtype, device="cuda")
             for k, s in dict(dX=(n, wi), dW=(wi, wo), db=(wo,), dR=(n, wo)).items()}
    B.slicegcn_product_bwd(x, wg, g, dh, ws, act=B.ACT_GELU, residual=3.0, **every)
    for k, t in every.items():
        alone = torch.full_like(t, 777.0)
        B.slicegcn_product_bwd(x if k == "dW" else None, wg, g if k != "dR" else None, dh, ws, act=B.ACT_GELU, residual=3.0, **{k: alone})
        assert torch.equal(alone, t), k


@pytest.mark.parametrize("kind", TYPES)
def test_no_rows(kind):
    dtype = TYPES[kind]
    e = lambda w: torch.empty((0, w), dtype=dtype, device="cuda")
    w, w2 = torch.ones((5, 7), dtype=dtype, device="cuda"), torch.ones((5, 7), dtype=dtype, device="cuda")
    assert B.slicegcn_product_fwd_workspace_bytes(0, 5, 7, dtype) == 0
    B.slicegcn_product_fwd(e(5), w, e(7), R=e(7), P=e(7), act=B.ACT_GELU)
    B.slicegcn_gated_fwd(e(5), w, w2, e(7))
    for t in (w, w2):
        t.fill_(777.0)
    db, db2 = torch.full((7,), 777.0, device="cuda"), torch.full((7,), 777.0, device="cuda")
    ws = workspace(B.slicegcn_gated_bwd_workspace_bytes(0, 5, 7, dtype))
    weight = torch.ones((5, 7), dtype=dtype, device="cuda")
    B.slicegcn_gated_bwd(e(5), weight, weight, e(7), e(7), e(7), ws, dX=e(5), dWg=w, dWu=w2, dbg=db, dbu=db2)
    for t in (w, w2, db, db2):
        assert (t == 0).all()
        t.fill_(777.0)
    ws = workspace(B.slicegcn_product_bwd_workspace_bytes(0, 5, 7, dtype))
    B.slicegcn_product_bwd(e(5), weight, e(7), e(7), ws, dX=e(5), dW=w, db=db, dR=e(7), act=B.ACT_SILU)
    assert (w == 0).all() and (db == 0).all()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", [(3, 900, 40), (150, 64, 200)], ids=str)
def test_result_in_the_rows_of_the_residual(size, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(5)
    x, _ = rows(gen, n, wi, dtype)
    w, _ = weights(gen, wi, wo, dtype)
    r, _ = rows(gen, n, wo, dtype, wo + 5)
    ws = workspace(B.slicegcn_product_fwd_workspace_bytes(n, wi, wo, dtype))
    y = torch.empty((n, wo), dtype=dtype, device="cuda")
    B.slicegcn_product_fwd(x, w, y, ws, R=r, act=B.ACT_SILU, residual=0.5)
    B.slicegcn_product_fwd(x, w, r, ws, R=r, act=B.ACT_SILU, residual=0.5)
    assert torch.equal(r, y)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", [(5, 1024, 136), (200, 128, 128), (129, 65, 40)], ids=str)
def test_values_that_are_not_finite_stay_in_their_rows_and_columns(size, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(6)
    x, _ = rows(gen, n, wi, dtype)
    (wg, _), (wu, _) = weights(gen, wi, wo, dtype), weights(gen, wi, wo, dtype)
    ws = workspace(B.slicegcn_gated_fwd_workspace_bytes(n, wi, wo, dtype))
    h, h2 = (torch.empty((n, wo), dtype=dtype, device="cuda") for _ in range(2))
    B.slicegcn_gated_fwd(x, wg, wu, h, ws)
    x[n // 2, wi - 1] = float("inf")
    wg[wi // 2, wo - 1] = float("nan")
    B.slicegcn_gated_fwd(x, wg, wu, h2, ws)
    assert not torch.isfinite(h2[n // 2]).any() and torch.isnan(h2[:, wo - 1]).all()
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[n // 2] = False
    assert torch.equal(h2[keep, :wo - 1], h[keep, :wo - 1])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", [(300, 40, 72), (2000, 1100, 136), (16_500, 64, 64)], ids=str)
def test_what_lies_behind_the_flat_part_of_a_relu_is_not_looked_at(size, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(7)
    x, g, d, u = (rows(gen, n, w, dtype)[0] for w in (wi, wo, wo, wo))
    (wg, _), (wu, _) = weights(gen, wi, wo, dtype), weights(gen, wi, wo, dtype)

    def grads(d, u):
        dx, dx2 = (torch.empty((n, wi), dtype=dtype, device="cuda") for _ in range(2))
        dw, dwg, dwu = (torch.empty_like(wg) for _ in range(3))
        db, dbg = (torch.empty(wo, device="cuda") for _ in range(2))
        B.slicegcn_product_bwd(x, wg, g, d, workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype)), dX=dx, dW=dw, db=db, act=B.ACT_RELU)
        B.slicegcn_gated_bwd(x, wg, wu, g, u, d.nan_to_num(0.0, 0.0, 0.0), workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype)), dX=dx2, dWg=dwg,
                             dWu=dwu, dbg=dbg, act=B.ACT_RELU)
        return dx, dw, db, dx2, dwg, dwu, dbg
    flat = g <= 0
    want = grads(d.masked_fill(flat, 0.0), u.masked_fill(flat, 0.0))
    d[flat] = float("inf")
    u[flat] = float("nan")
    for a, b in zip(grads(d, u), want):
        assert torch.isfinite(b).all() and torch.equal(a, b)


def test_large_and_small_fp32_operands():
    """Values over the whole range of exponents: each product by itself (a sum of one)."""
    gen = torch.Generator().manual_seed(8)
    n = 64
    x = (torch.randn((n, 1), generator=gen) * torch.exp2(torch.randint(-60, 60, (n, 1), generator=gen).float()))
    w = (torch.randn((1, n), generator=gen) * torch.exp2(torch.randint(-60, 60, (1, n), generator=gen).float()))
    y = torch.empty((n, n), device="cuda")
    B.slicegcn_product_fwd(x.cuda(), w.cuda(), y, workspace(B.slicegcn_product_fwd_workspace_bytes(n, 1, n, torch.float32)))
    want = x.double() * w.double()
    assert_within(y, want, 16 * 2.0 ** -24 * want.abs(), "products")


def test_same_bits_again_and_on_another_stream():
    gen = torch.Generator().manual_seed(9)
    n, wi, wo = 333, 264, 200
    x, g, u, dh = (rows(gen, n, w, torch.bfloat16)[0] for w in (wi, wo, wo, wo))
    (wg, _), (wu, _) = weights(gen, wi, wo, torch.bfloat16), weights(gen, wi, wo, torch.bfloat16)

    def once():
        ws = workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, torch.bfloat16))
        out = [torch.empty_like(t) for t in (x, wg, wu)] + [torch.empty(wo, device="cuda")]
        B.slicegcn_gated_bwd(x, wg, wu, g, u, dh, ws, dX=out[0], dWg=out[1], dWu=out[2], dbg=out[3])
        return out
    first = once()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = once()
    torch.cuda.current_stream().wait_stream(s)
    for a, b in zip(first, other):
        assert torch.equal(a, b)


@pytest.mark.parametrize("kind", TYPES)
def test_a_block_in_a_graph(kind):
    """Forward and backward of a feed-forward block captured and replayed with new rows, beside eager calls."""
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(10)
    n, w, f = 70, 96, 264
    x, dy = rows(gen, n, w, dtype)[0], rows(gen, n, w, dtype)[0]
    (wg, _), (wu, _), (wd, _) = weights(gen, w, f, dtype), weights(gen, w, f, dtype), weights(gen, f, w, dtype)

    def block(x):
        e = lambda *s: torch.empty(s, dtype=dtype, device="cuda")
        t = dict(h=e(n, f), g=e(n, f), u=e(n, f), y=e(n, w), dh=e(n, f), dwd=e(f, w), dx=e(n, w), dwg=e(w, f), dwu=e(w, f))
        sizes = [B.slicegcn_gated_fwd_workspace_bytes(n, w, f, dtype), B.slicegcn_gated_bwd_workspace_bytes(n, w, f, dtype),
                 B.slicegcn_product_fwd_workspace_bytes(n, f, w, dtype), B.slicegcn_product_bwd_workspace_bytes(n, f, w, dtype)]
        ws = torch.empty(max(sizes), dtype=torch.uint8, device="cuda")

        def run():
            B.slicegcn_gated_fwd(x, wg, wu, t["h"], ws, G=t["g"], U=t["u"])
            B.slicegcn_product_fwd(t["h"], wd, t["y"], ws, R=x)
            B.slicegcn_product_bwd(t["h"], wd, None, dy, ws, dX=t["dh"], dW=t["dwd"])
            B.slicegcn_gated_bwd(x, wg, wu, t["g"], t["u"], t["dh"], ws, dX=t["dx"], dWg=t["dwg"], dWu=t["dwu"])
        return run, t, ws
    captured, t, _ = block(x)
    captured()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured()
    for seed in range(3):
        x.copy_(torch.randn((n, w), generator=torch.Generator().manual_seed(seed)).to(dtype))
        eager, e, _ = block(x)
        eager()
        for v in t.values():
            v.fill_(777.0)
        graph.replay()
        torch.cuda.synchronize()
        for k in t:
            assert torch.equal(t[k], e[k]), k


def test_gradients_against_differences():
    """dX and dWg of a small block against central differences of the block in 64 bits."""
    gen = torch.Generator().manual_seed(11)
    n, w, f = 4, 6, 5
    x, x64 = rows(gen, n, w, torch.float32)
    (wg, wg64), (wu, wu64) = weights(gen, w, f, torch.float32), weights(gen, w, f, torch.float32)
    dh, d64 = rows(gen, n, f, torch.float32)
    h, g, u = (torch.empty((n, f), device="cuda") for _ in range(3))
    B.slicegcn_gated_fwd(x, wg, wu, h, workspace(B.slicegcn_gated_fwd_workspace_bytes(n, w, f, torch.float32)), G=g, U=u, act=B.ACT_GELU)
    dx, dwg = torch.empty_like(x), torch.empty_like(wg)
    B.slicegcn_gated_bwd(x, wg, wu, g, u, dh, workspace(B.slicegcn_gated_bwd_workspace_bytes(n, w, f, torch.float32)), dX=dx, dWg=dwg,
                         act=B.ACT_GELU)

    def loss():
        return float((gated_fwd(x64, wg64, wu64, None, None, "gelu", torch.float32)["H"][0] * d64).sum())
    step = 1e-5  # error of the differences: step^2 times third derivatives of order 1, 1e-10
    for t64, grad in ((x64, dx.cpu()), (wg64, dwg.cpu())):
        for i in range(t64.shape[0]):
            for j in range(t64.shape[1]):
                old = float(t64[i, j])
                t64[i, j] = old + step
                up = loss()
                t64[i, j] = old - step
                down = loss()
                t64[i, j] = old
                assert abs((up - down) / (2 * step) - float(grad[i, j])) < 1e-5  # sums of at most 30 products of order 1 in fp32: 30 * 2^-20


NARROW = [(16384, 100, 256), (20_011, 128, 126), (17_000, 6, 2), (16_500, 64, 64), (16_390, 34, 250), (33_333, 72, 40)]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", NARROW, ids=str)
@pytest.mark.parametrize("gated", [False, True])
def test_narrow_backward_passes_of_many_rows(size, kind, gated):
    """In one sweep over the rows where they lie on boundaries of 4 bytes, and in the general form where they do not."""
    n, wi, wo = size
    dtype = TYPES[kind]
    case = NARROW.index(size)
    if gated:
        wo = min(wo, 128)
    gen = torch.Generator().manual_seed(200 + case)
    name = ACTS[(case + gated) % 4]
    x, x64 = rows(gen, n, wi, dtype, wi + (0, 2, 30)[case % 3], (0, 2, 8)[case % 3])
    w = [weights(gen, wi, wo, dtype) for _ in range(2)]
    g, g64 = rows(gen, n, wo, dtype, wo + (2, 0, 6)[case % 3], std=1.5)
    u, u64 = rows(gen, n, wo, dtype, wo, 2)
    d, d64 = rows(gen, n, wo, dtype, wo + (0, 4, 2)[case % 3])
    if gated:
        want = gated_bwd(x64, w[0][1], w[1][1], g64, u64, d64, name, dtype)
        call, keys = (lambda ws, x=x, **out: B.slicegcn_gated_bwd(x, w[0][0], w[1][0], g, u, d, ws, act=ACT[name], **out)), ("dX", "dWg", "dWu", "dbg", "dbu")
        ws = workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype))
    else:
        want = product_bwd(x64, w[0][1], g64, d64, 1.0, name, dtype)
        call, keys = (lambda ws, x=x, **out: B.slicegcn_product_bwd(x, w[0][0], g if name != "none" else None, d, ws, act=ACT[name], **out)), ("dX", "dW", "db")
        ws = workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype))

    def outputs(ld):
        dx, buf = result(n, wi, dtype, ld)
        return {k: dx if k == "dX" else torch.full((wi, wo) if k[1] == "W" else (wo,), 777.0, dtype=dtype if k[1] == "W" else torch.float32, device="cuda")
                for k in keys}, buf
    first, buf = outputs(wi + 2)
    call(ws, **first)
    for k in keys:
        assert_within(first[k], *want[k], k)
    assert_padding(buf, wi)
    again, _ = outputs(wi)
    call(ws, **again)
    assert all(torch.equal(first[k], again[k]) for k in keys)
    for some in (("dX",), tuple(k for k in keys if k[1] == "W"), ("dX", keys[-1])):  # without the others, and without X where dW is not wanted
        few = {k: v for k, v in outputs(wi)[0].items() if k in some}
        call(ws, x=x if any(k[1] == "W" for k in some) else None, **few)
        assert all(torch.equal(few[k], first[k]) for k in some if k != "X"), some
    general, buf = outputs(wi + 3)  # rows of dX on odd elements
    call(ws, **general)
    for k in keys:
        assert_within(general[k], *want[k], k)
    assert_padding(buf, wi)


# rows that are no whole units of 16 bytes, through registers: odd widths, even ones, one of the two
UNEVEN = [(2050, 1003, 1021), (1500, 1026, 1401), (2100, 1016, 1001), (3000, 701, 1024), (140, 4001, 4103)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size", UNEVEN, ids=str)
@pytest.mark.parametrize("ld", ["dense", "lines", "odd"])
def test_large_products_of_rows_that_lie_oddly(size, ld, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(sum(size))
    x, x64 = rows(gen, n, wi, dtype, lds(n, wi, ld))
    (wg, wg64), (wu, wu64) = weights(gen, wi, wo, dtype), weights(gen, wi, wo, dtype)
    g, g64 = rows(gen, n, wo, dtype, lds(n, wo, ld))
    u, u64 = rows(gen, n, wo, dtype, lds(n, wo, ld))
    d, d64 = rows(gen, n, wo, dtype, lds(n, wo, ld))
    for name in ("none", "silu"):
        y, ybuf = result(n, wo, dtype, lds(n, wo, ld))
        B.slicegcn_product_fwd(x, wg, y, workspace(B.slicegcn_product_fwd_workspace_bytes(n, wi, wo, dtype)), R=u, act=ACT[name])
        assert_within(y, *product_fwd(x64, wg64, None, u64, 1.0, name, dtype)["Y"], "Y")
        assert_padding(ybuf, wo)
        dx, dxbuf = result(n, wi, dtype, lds(n, wi, ld))
        dw, db = torch.full_like(wg, 777.0), torch.full((wo,), 777.0, device="cuda")
        B.slicegcn_product_bwd(x, wg, g, d, workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype)), dX=dx, dW=dw, db=db, act=ACT[name])
        want = product_bwd(x64, wg64, g64, d64, 1.0, name, dtype)
        for got, key in ((dx, "dX"), (dw, "dW"), (db, "db")):
            assert_within(got, *want[key], key)
        assert_padding(dxbuf, wi)
    h, hbuf = result(n, wo, dtype, lds(n, wo, ld))
    B.slicegcn_gated_fwd(x, wg, wu, h, workspace(B.slicegcn_gated_fwd_workspace_bytes(n, wi, wo, dtype)))
    assert_within(h, *gated_fwd(x64, wg64, wu64, None, None, "silu", dtype)["H"], "H")
    assert_padding(hbuf, wo)
    dx, dxbuf = result(n, wi, dtype, lds(n, wi, ld))
    dwg, dwu = torch.full_like(wg, 777.0), torch.full_like(wu, 777.0)
    ws = workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype))
    B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, dX=dx, dWg=dwg, dWu=dwu)
    want = gated_bwd(x64, wg64, wu64, g64, u64, d64, "silu", dtype)
    for got, key in ((dx, "dX"), (dwg, "dWg"), (dwu, "dWu")):
        assert_within(got, *want[key], key)
    assert_padding(dxbuf, wi)
    alone = torch.full_like(wu, 777.0)
    B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, dWu=alone)
    assert torch.equal(alone, dwu)


@pytest.mark.parametrize("kind", TYPES)
def test_rows_of_more_than_4_gb_give_the_bits_of_close_rows(kind):
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(12)
    n, wi, wo, ld = 70_000, 64, 136, (1 << 15) if dtype != torch.float32 else 1 << 14  # 4.6 GB
    gaps = [torch.empty((n, ld), dtype=dtype, device="cuda") for _ in range(2)]
    assert gaps[0].numel() * gaps[0].element_size() > 1 << 32
    (wg, _), (wu, _) = weights(gen, wi, wo, dtype), weights(gen, wi, wo, dtype)
    x, g, u, d = (rows(gen, n, w, dtype)[0] for w in (wi, wo, wo, wo))

    def far(t, i, col):
        v = gaps[i][:, col:col + t.shape[1]]
        return v.copy_(t)
    # 8 columns apart, so that rows lie on the boundaries that close ones lie on
    fx, fg, fu, fd = far(x, 0, 0), far(g, 0, 72), far(u, 0, 216), far(d, 0, 360)
    empty = lambda i, w, col: gaps[i][:, col:col + w]
    close = lambda w: torch.empty((n, w), dtype=dtype, device="cuda")
    h, ks, dx, y = close(wo), [close(wo), close(wo)], close(wi), close(wo)
    fh, fks, fdx, fy = empty(1, wo, 0), [empty(1, wo, 144), empty(1, wo, 288)], empty(1, wi, 432), empty(1, wo, 504)
    ws = workspace(max(f(n, wi, wo, dtype) for f in (B.slicegcn_gated_fwd_workspace_bytes, B.slicegcn_gated_bwd_workspace_bytes,
                                                     B.slicegcn_product_fwd_workspace_bytes, B.slicegcn_product_bwd_workspace_bytes)))
    dw = [torch.empty_like(wg) for _ in range(6)]
    B.slicegcn_gated_fwd(x, wg, wu, h, ws, G=ks[0], U=ks[1])
    B.slicegcn_gated_fwd(fx, wg, wu, fh, ws, G=fks[0], U=fks[1])
    B.slicegcn_product_fwd(x, wg, y, ws, R=u, act=B.ACT_GELU)
    B.slicegcn_product_fwd(fx, wg, fy, ws, R=fu, act=B.ACT_GELU)
    assert torch.equal(h, fh) and torch.equal(ks[0], fks[0]) and torch.equal(ks[1], fks[1]) and torch.equal(y, fy)
    B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, dX=dx, dWg=dw[0], dWu=dw[1])
    B.slicegcn_gated_bwd(fx, wg, wu, fg, fu, fd, ws, dX=fdx, dWg=dw[2], dWu=dw[3])
    assert torch.equal(dx, fdx) and torch.equal(dw[0], dw[2]) and torch.equal(dw[1], dw[3])
    B.slicegcn_product_bwd(x, wg, None, d, ws, dX=dx, dW=dw[4])
    B.slicegcn_product_bwd(fx, wg, None, fd, ws, dX=fdx, dW=dw[5])
    assert torch.equal(dx, fdx) and torch.equal(dw[4], dw[5])


@pytest.mark.parametrize("kind", TYPES)
def test_calls_at_the_same_time(kind):
    """Two streams with a workspace each; what either forms is what it forms alone."""
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(13)
    n, w, f = 700, 264, 712
    (wg, _), (wu, _), (wd, _) = weights(gen, w, f, dtype), weights(gen, w, f, dtype), weights(gen, f, w, dtype)
    calls = []
    for _ in range(2):
        x, dy = rows(gen, n, w, dtype)[0], rows(gen, n, w, dtype)[0]
        e = lambda *s: torch.empty(s, dtype=dtype, device="cuda")
        ws = workspace(max(fn(n, a, b, dtype) for fn in (B.slicegcn_gated_fwd_workspace_bytes, B.slicegcn_gated_bwd_workspace_bytes,
                                                         B.slicegcn_product_fwd_workspace_bytes, B.slicegcn_product_bwd_workspace_bytes)
                           for a, b in ((w, f), (f, w))))
        calls.append((x, dy, ws, dict(h=e(n, f), g=e(n, f), u=e(n, f), y=e(n, w), dh=e(n, f), dwd=e(f, w), dx=e(n, w), dwg=e(w, f), dwu=e(w, f))))

    def block(x, dy, ws, t):
        B.slicegcn_gated_fwd(x, wg, wu, t["h"], ws, G=t["g"], U=t["u"])
        B.slicegcn_product_fwd(t["h"], wd, t["y"], ws, R=x)
        B.slicegcn_product_bwd(t["h"], wd, None, dy, ws, dX=t["dh"], dW=t["dwd"])
        B.slicegcn_gated_bwd(x, wg, wu, t["g"], t["u"], t["dh"], ws, dX=t["dx"], dWg=t["dwg"], dWu=t["dwu"])
    alone = []
    for c in calls:
        block(*c)
        alone.append({k: v.clone() for k, v in c[3].items()})
    streams = [torch.cuda.Stream() for _ in calls]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                block(*c)
    torch.cuda.synchronize()
    for c, want in zip(calls, alone):
        assert all(torch.equal(c[3][k], want[k]) for k in want)


# on either side of where both products of a backward pass share a launch: by the multiplications in them, by the elements of dX, by those of dW
SHORT = [(2048, 512, 128), (2049, 512, 128), (2048, 512, 130), (1030, 1018, 120), (40, 1400, 740), (40, 1400, 760), (1000, 2, 3), (1200, 301, 13)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", SHORT, ids=str)
@pytest.mark.parametrize("q", [1, 2])
def test_short_backward_passes(size, q, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(14)
    x, x64 = rows(gen, n, wi, dtype)
    (wg, wg64), (wu, wu64) = weights(gen, wi, wo, dtype), weights(gen, wi, wo, dtype)
    g, g64 = rows(gen, n, wo, dtype, std=1.5)
    u, u64 = rows(gen, n, wo, dtype)
    d, d64 = rows(gen, n, wo, dtype)
    dx, dxbuf = result(n, wi, dtype, wi + 1)
    dwg, dwu = torch.full_like(wg, 777.0), torch.full_like(wu, 777.0)
    db = torch.full((wo,), 777.0, device="cuda")
    if q == 2:
        ws = workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype))
        B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, dX=dx, dWg=dwg, dWu=dwu, dbu=db)
        want = gated_bwd(x64, wg64, wu64, g64, u64, d64, "silu", dtype)
        got = ((dx, "dX"), (dwg, "dWg"), (dwu, "dWu"), (db, "dbu"))
    else:
        ws = workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype))
        B.slicegcn_product_bwd(x, wg, g, d, ws, dX=dx, dW=dwg, db=db, act=B.ACT_GELU)
        want = product_bwd(x64, wg64, g64, d64, 1.0, "gelu", dtype)
        got = ((dx, "dX"), (dwg, "dW"), (db, "db"))
    for t, key in got:
        assert_within(t, *want[key], key)
    assert_padding(dxbuf, wi)


# 16-bit products that go in tiles of 256 x 256: cut sums, ends within a step and an odd number of steps, one tile of rows, a sum of many rows, columns behind a tile; and with
# operands that are copied first
LONG = [(513, 5000, 4104), (130, 9000, 9032), (8200, 9064, 136), (20_000, 72, 7000), (2500, 2056, 2000), (2050, 2003, 2521), (9001, 1026, 1101), (140, 8401, 9103),
        # more than a round of tiles, the last of which are cut: in dX and both dW of a gated projection, in all but the latter, and with an end within four columns
        (4100, 4400, 3768), (4100, 4400, 4616), (4100, 4401, 4611),
        # copied: rows on odd elements, gradients without an activation
        (1500, 3026, 2401), (2100, 2203, 2301)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size", LONG, ids=str)
def test_long_products(size, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    case = LONG.index(size)
    gen = torch.Generator().manual_seed(300 + case)
    ld = ("dense", "lines", "odd" if wi % 8 else "dense")[case % 3]
    on_gpu = lambda t, t64: (t, t64.cuda())  # references in 64 bits on the device: 1e10 multiplications each
    x, x64 = on_gpu(*rows(gen, n, wi, dtype, lds(n, wi, ld)))
    (wg, wg64), (wu, wu64) = (on_gpu(*weights(gen, wi, wo, dtype)) for _ in range(2))
    g, g64 = on_gpu(*rows(gen, n, wo, dtype, lds(n, wo, ld), std=1.5))
    u, u64 = on_gpu(*rows(gen, n, wo, dtype, lds(n, wo, ld)))
    d, d64 = on_gpu(*rows(gen, n, wo, dtype, lds(n, wo, ld)))
    b = torch.randn(wo, generator=gen).cuda()
    name = ACTS[case % 4]
    y, ybuf = result(n, wo, dtype, lds(n, wo, ld))
    p, pbuf = result(n, wo, dtype, lds(n, wo, "odd"))
    dx, dxbuf = result(n, wi, dtype, lds(n, wi, ld))
    dwg, dwu, db = torch.full_like(wg, 777.0), torch.full_like(wu, 777.0), torch.full((wo,), 777.0, device="cuda")

    def check(got, want, key):
        assert_within(got, *(t.cpu() for t in want[key]), key)
    B.slicegcn_product_fwd(x, wg, y, workspace(B.slicegcn_product_fwd_workspace_bytes(n, wi, wo, dtype)), b=b, R=u, P=p, act=ACT[name], residual=0.5)
    want = product_fwd(x64, wg64, b.to(F64), u64, 0.5, name, dtype)
    check(y, want, "Y")
    check(p, want, "P")
    assert_padding(ybuf, wo)
    assert_padding(pbuf, wo)
    B.slicegcn_product_bwd(x, wg, g, d, workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype)), dX=dx, dW=dwg, db=db, act=ACT[name])
    want = product_bwd(x64, wg64, g64, d64, 1.0, name, dtype)
    for got, key in ((dx, "dX"), (dwg, "dW"), (db, "db")):
        check(got, want, key)
    assert_padding(dxbuf, wi)
    B.slicegcn_gated_fwd(x, wg, wu, y, workspace(B.slicegcn_gated_fwd_workspace_bytes(n, wi, wo, dtype)), bg=b, act=ACT[name])
    check(y, gated_fwd(x64, wg64, wu64, b.to(F64), None, name, dtype), "H")
    assert_padding(ybuf, wo)
    B.slicegcn_gated_bwd(x, wg, wu, g, u, d, workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype)), dX=dx, dWg=dwg, dWu=dwu, dbu=db, act=ACT[name])
    want = gated_bwd(x64, wg64, wu64, g64, u64, d64, name, dtype)
    for got, key in ((dx, "dX"), (dwg, "dWg"), (dwu, "dWu"), (db, "dbu")):
        check(got, want, key)
    assert_padding(dxbuf, wi)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size", [(33, 65, 129), (200, 131, 71), (7, 333, 45), (64, 63, 65), (300, 129, 201), (1, 1, 1), (1300, 901, 303)], ids=str)
@pytest.mark.parametrize("offset", [0, 1])
def test_operands_of_odd_widths_amid_nan(size, offset, kind):
    """Elements before and behind an operand share words with its own: of a pair of weights one begins on a word, the other within one."""
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(400 + offset)

    def amid(rows, width, offset, std=1.0):
        buf = torch.full((rows * width + offset + 9,), float("nan"), dtype=dtype)
        view = buf[offset:offset + rows * width].view(rows, width)
        view.copy_((torch.randn((rows, width), generator=gen) * std).to(dtype))
        return buf.cuda()[offset:offset + rows * width].view(rows, width), view.to(F64)
    x, x64 = amid(n, wi, offset)
    wg, wg64 = amid(wi, wo, offset, wi ** -0.5)
    wu, wu64 = amid(wi, wo, 1 - offset, wi ** -0.5)
    g, g64 = amid(n, wo, 1 - offset, 1.5)
    u, u64 = amid(n, wo, offset)
    d, d64 = amid(n, wo, 1)
    ws = workspace(max(f(n, wi, wo, dtype) for f in (B.slicegcn_gated_fwd_workspace_bytes, B.slicegcn_gated_bwd_workspace_bytes,
                                                     B.slicegcn_product_fwd_workspace_bytes, B.slicegcn_product_bwd_workspace_bytes)))
    y, ybuf = result(n, wo, dtype, wo + 1)
    dx, dxbuf = result(n, wi, dtype, wi + 2)
    dwg, dwu, db = torch.full((wi, wo), 777.0, dtype=dtype, device="cuda"), torch.full((wi, wo), 777.0, dtype=dtype, device="cuda"), torch.zeros(wo, device="cuda")
    B.slicegcn_product_fwd(x, wg, y, ws, R=u)
    assert_within(y, *product_fwd(x64, wg64, None, u64, 1.0, "none", dtype)["Y"], "Y")
    assert_padding(ybuf, wo)
    B.slicegcn_gated_fwd(x, wg, wu, y, ws)
    assert_within(y, *gated_fwd(x64, wg64, wu64, None, None, "silu", dtype)["H"], "H")
    assert_padding(ybuf, wo)
    B.slicegcn_product_bwd(x, wg, None, d, ws, dX=dx, dW=dwg, db=db)
    want = product_bwd(x64, wg64, None, d64, 1.0, "none", dtype)
    for got, key in ((dx, "dX"), (dwg, "dW"), (db, "db")):
        assert_within(got, *want[key], key)
    B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, dX=dx, dWg=dwg, dWu=dwu, dbg=db)
    want = gated_bwd(x64, wg64, wu64, g64, u64, d64, "silu", dtype)
    for got, key in ((dx, "dX"), (dwg, "dWg"), (dwu, "dWu"), (db, "dbg")):
        assert_within(got, *want[key], key)
    assert_padding(dxbuf, wi)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size", [(3, 259, 8), (1, 40, 24), (2, 15, 593), (60, 100, 200), (1300, 33, 12), (7, 1000, 501)], ids=str)
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_gradients_of_few_elements_keep_two_terms(size, name, kind):
    """Bounds without the rounding of the gradients before the activation: a sum of both terms has twice the products, in parts that are added in fp64."""
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(15)
    x, x64 = rows(gen, n, wi, dtype)
    (wg, wg64), (wu, wu64) = weights(gen, wi, wo, dtype), weights(gen, wi, wo, dtype)
    g, g64 = rows(gen, n, wo, dtype, wo + 3, std=1.5)
    u, u64 = rows(gen, n, wo, dtype)
    d, d64 = rows(gen, n, wo, dtype)
    dx, dxbuf = result(n, wi, dtype, wi + 1)
    dwg, dwu = torch.full_like(wg, 777.0), torch.full_like(wu, 777.0)
    B.slicegcn_product_bwd(x, wg, g, d, workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype)), dX=dx, dW=dwg, act=ACT[name])
    want = product_bwd(x64, wg64, g64, d64, 1.0, name, dtype, terms=2)
    for got, key in ((dx, "dX"), (dwg, "dW")):
        assert_within(got, *want[key], key)
    ws = workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype))
    B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, dX=dx, dWg=dwg, dWu=dwu, act=ACT[name])
    want = gated_bwd(x64, wg64, wu64, g64, u64, d64, name, dtype, terms=2)
    for got, key in ((dx, "dX"), (dwg, "dWg"), (dwu, "dWu")):
        assert_within(got, *want[key], key)
    assert_padding(dxbuf, wi)
    alone = torch.full_like(wu, 777.0)
    B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, dWu=alone, act=ACT[name])
    assert torch.equal(alone, dwu)


def test_gradients_beyond_fp16_stay_infinite():
    one = lambda v, *shape: torch.full(shape, v, dtype=torch.float16, device="cuda")
    x, w, g, u, d = one(2.0, 1, 8), one(0.5, 8, 16), one(3.0, 1, 16), one(60.0, 1, 16), one(-60000.0, 1, 16)
    dx, dwg, dwu = one(0.0, 1, 8), one(0.0, 8, 16), one(0.0, 8, 16)
    B.slicegcn_gated_bwd(x, w, w, g, u, d, workspace(B.slicegcn_gated_bwd_workspace_bytes(1, 8, 16, torch.float16)), dX=dx, dWg=dwg, dWu=dwu)
    assert (dwg == -float("inf")).all() and (dx == -float("inf")).all()
