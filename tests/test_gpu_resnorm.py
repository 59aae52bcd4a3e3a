"""Norms around a block with its gate and residual, forward and backward, against plain 64-bit forms: every combination of norms, gates and
absent operands, at widths, types and strides where they can go wrong."""
import itertools

import pytest
import torch

from paper_2408_11500_amd import binding as B
from train_util import F64, LAYER, NONE, RMS, TYPES, U, Resnorm, assert_within, half_step, rows

pytestmark = pytest.mark.gpu

# Additions in a row: 16 of a lane, 6 over a wavefront, 16 over wavefronts; a column sum 64 in these tests; the chain of a formula 20 operations.
# Each of the two norms of a result passes its error on once.
C = 256


class Call:
    """Operands of one call on the device and in 64 bits."""

    def __init__(self, n, width, kind, post=RMS, pre=RMS, gate="column", sigmoid=False, x=True, y=True, bias=True, weight=True, residual=1.0,
                 eps=1e-6, ld=None, offset=0, seed=0, shift=0.0):
        gen = torch.Generator().manual_seed(seed + 131 * width + n)
        self.n, self.width, self.dtype, self.ld, self.offset = n, width, TYPES[kind], ld or width, offset
        self.dev, self.f64 = {}, {}

        def put(name, there, mean=0.0, std=1.0):
            self.dev[name], self.f64[name] = rows(gen, n, width, self.dtype, self.ld, offset, std) if there else (None, None)
            if there and mean:
                self.dev[name] += mean
                self.f64[name] = self.dev[name].cpu().to(F64)

        def param(name, there, mean, std):
            t = (mean + std * torch.randn(width, generator=gen)) if there else None
            self.dev[name], self.f64[name] = (None, None) if t is None else (t.cuda(), t.to(F64))
        put("x", x, shift)
        put("y", y, shift, 2.0)
        post = post if y else NONE
        gate = gate if y else "none"
        param("post_w", weight and post != NONE, 1.0, 0.3)
        param("post_b", bias and post != NONE, 0.0, 0.3)
        param("pre_w", weight and pre != NONE, 1.0, 0.3)
        param("pre_b", bias and pre != NONE, 0.0, 0.3)
        param("gate", gate == "column", 0.5, 0.5)
        if gate == "matrix":
            put("gate", True)
        self.sigmoid = sigmoid and gate != "none"
        self.args = dict(post=post, pre=pre, sigmoid=self.sigmoid, residual=residual, eps=eps)
        self.gen = gen
        self.want = Resnorm(**self.f64, **self.args)

    def like(self, fill=float("nan")):
        buf = torch.full((self.n * self.ld + self.offset,), fill, dtype=self.dtype, device="cuda")
        return buf[self.offset:].view(self.n, self.ld)[:, :self.width]

    def forward(self, h=True, u=True, stats=True):
        self.h, self.u = self.like() if h else None, self.like() if u else None
        self.stats = torch.full((self.n, 4), float("nan"), device="cuda") if stats else None
        B.slicegcn_resnorm_fwd(self.dev["x"], self.dev["y"], self.h, self.u, stats=self.stats, **self.params(), **self.args)

    def params(self):
        return {k: self.dev[k] for k in ("post_w", "post_b", "pre_w", "pre_b", "gate")}

    def check_forward(self):
        w = self.want
        if self.h is not None:
            assert_within(self.h, w.h, C * U * w.h_size, "h")
        if self.u is not None:
            assert_within(self.u, w.u, C * U * w.u_size, "u")

    def backward(self, dh=True, du=True, rows_wanted=True, params_wanted=True):
        self.dh, dh64 = rows(self.gen, self.n, self.width, self.dtype, self.ld, self.offset) if dh else (None, None)
        self.du, du64 = rows(self.gen, self.n, self.width, self.dtype, self.ld, self.offset) if du else (None, None)
        g = {"d" + k: torch.full_like(v, float("nan")) if v.dim() == 1 else self.like()
             for k, v in self.params().items() if v is not None and (params_wanted if v.dim() == 1 else rows_wanted)}
        self.dx = self.like() if self.dev["x"] is not None and rows_wanted else None
        self.dy = self.like() if self.dev["y"] is not None and rows_wanted else None
        ws = torch.empty(B.slicegcn_resnorm_bwd_workspace_bytes(self.n, self.width), dtype=torch.uint8, device="cuda")
        B.slicegcn_resnorm_bwd(self.dev["x"], self.dev["y"], self.stats, self.dh, self.du, self.dx, self.dy, ws, **g, **self.params(), **self.args)
        self.g = dict(g, dx=self.dx, dy=self.dy)
        want, size = self.want.backward(dh64, du64)
        for name, got in self.g.items():
            if got is not None:
                assert_within(got, want[name].reshape(got.shape), C * U * size[name].reshape(got.shape), name)


SHAPES = [(1, 1), (3, 2), (5, 3), (2, 4), (7, 5), (9, 7), (70, 8), (33, 9), (260, 16), (300, 31), (65, 33), (130, 64), (50, 100), (41, 129),
          (37, 256), (20, 257), (19, 511), (17, 512), (21, 513), (12, 602), (9, 1000), (9, 1024), (7, 1025), (6, 1500), (5, 2048), (5, 2049),
          (5, 4096), (4, 4100), (3, 5003), (3, 8192), (3, 8193), (2, 12_345), (2, 16_383), (2, 16_384)]


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,width", SHAPES)
def test_widths(n, width, kind):
    for post, pre, gate, ld, offset in ((RMS, RMS, "column", width, 0), (LAYER, LAYER, "matrix", width + 3, 1), (NONE, RMS, "none", width, 0)):
        c = Call(n, width, kind, post, pre, gate, sigmoid=gate == "matrix", ld=ld, offset=offset, residual=0.75, eps=1e-3)
        c.forward()
        c.check_forward()
        c.backward()


@pytest.mark.parametrize("post,pre", list(itertools.product((NONE, RMS, LAYER), repeat=2)))
@pytest.mark.parametrize("gate,sigmoid", [("none", False), ("column", False), ("column", True), ("matrix", False), ("matrix", True)])
@pytest.mark.parametrize("kind,width", [("f32", 72), ("bf16", 200), ("f16", 1040)])
def test_norms_and_gates(post, pre, gate, sigmoid, kind, width):
    for weight, bias in ((True, True), (True, False), (False, False), (False, True)):
        c = Call(23, width, kind, post, pre, gate, sigmoid, weight=weight, bias=bias, residual=1.25)
        c.forward()
        c.check_forward()
        c.backward()


@pytest.mark.parametrize("kind,width", [("f32", 60), ("bf16", 1100)])
@pytest.mark.parametrize("pre", [NONE, LAYER])
@pytest.mark.parametrize("x,y,h,u", [(True, False, False, True), (True, False, True, True), (False, True, True, True), (True, True, False, True),
                                     (True, True, True, False), (False, True, True, False)])
def test_absent_rows(x, y, h, u, pre, kind, width):
    c = Call(19, width, kind, LAYER, pre, "column", x=x, y=y, residual=0.5)
    c.forward(h=h, u=u, stats=u or pre == NONE)
    c.check_forward()
    if u or pre == NONE:
        c.backward(dh=h, du=u)
        if h and u:
            c.backward(dh=False)
            c.backward(du=False)
            c.backward(rows_wanted=False)
            c.backward(params_wanted=False)


@pytest.mark.parametrize("width", [48, 2000])
def test_far_means_and_rows_without_variance(width):
    """Rows of one value (variance zero), rows of zeros, and values far from zero, where a sum of squares minus a square would cancel."""
    c = Call(12, width, "f32", LAYER, LAYER, "none", shift=300.0, eps=1e-2)
    c.forward()
    c.check_forward()
    c.backward()
    x = torch.zeros(4, width, device="cuda")
    x[1], x[2] = 5.0, -1e-20
    for norm in (RMS, LAYER):
        u = torch.empty_like(x)
        B.slicegcn_resnorm_fwd(x, None, None, u, pre=norm, eps=1e-6)
        w = Resnorm(x.cpu().to(F64), None, pre=norm, eps=1e-6)
        assert_within(u, w.u, C * U * w.u_size, "u")


def test_non_finite_values_stay_in_their_rows():
    c = Call(40, 96, "f32", RMS, LAYER, "column")
    c.dev["y"][7, 3], c.dev["x"][20, 90] = float("inf"), float("nan")
    c.forward()
    good = torch.ones(40, dtype=torch.bool)
    good[7] = good[20] = False
    assert c.u[good.cuda()].isfinite().all() and c.h[good.cuda()].isfinite().all()
    assert c.u[20].isnan().all() and not c.u[7].isfinite().any()
    c.h, c.u, c.want.h, c.want.u, c.want.h_size, c.want.u_size = (t[good.cuda() if t.is_cuda else good] for t in
                                                                  (c.h, c.u, c.want.h, c.want.u, c.want.h_size, c.want.u_size))
    c.check_forward()


@pytest.mark.parametrize("n", [0, 1, 255, 100_003])
def test_many_rows_and_none(n):
    """Column sums over as many rows as there are: each workgroup adds up to 100 of them in turn."""
    c = Call(n, 24, "f32", RMS, RMS, "column", residual=1.0)
    c.forward()
    c.check_forward()
    c.backward()
    if n == 0:
        assert all((c.g[k] == 0).all() for k in ("dpost_w", "dpost_b", "dpre_w", "dpre_b", "dgate"))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("width", [602, 2049, 4097, 5120, 8192])
@pytest.mark.parametrize("norm,gate", [(RMS, "column"), (LAYER, "column"), (LAYER, "matrix")])
def test_wide_rows_in_turn(width, kind, norm, gate):
    """More rows than workgroups, so that each takes several in turn: the row requested ahead, sums kept over rows."""
    n = {602: 12_000, 2049: 2100, 4097: 1100, 5120: 600, 8192: 600}[width]
    c = Call(n, width, kind, norm, norm, gate, sigmoid=gate == "matrix", residual=0.75)
    c.forward()
    c.check_forward()
    c.backward()


@pytest.mark.parametrize("kind,width", [("f32", 64), ("f32", 301), ("bf16", 1001), ("f32", 1333), ("f16", 5001)])
def test_rows_in_place(kind, width):
    """Outputs in the rows of inputs give the same bits; nothing beside the rows is written."""
    for post, pre, gate in ((RMS, LAYER, "matrix"), (NONE, NONE, "column"), (NONE, RMS, "none"), (RMS, NONE, "matrix")):
        c = Call(13, width, kind, post, pre, gate, ld=width + 5)
        c.forward()
        c.backward()
        wide = lambda t: t.as_strided((t.shape[0], width + 5), t.stride(), t.storage_offset())
        d = {k: wide(v).clone()[:, :width] if v is not None and v.dim() == 2 else v for k, v in c.dev.items()}
        B.slicegcn_resnorm_fwd(d["x"], d["y"], d["x"], d["y"], **{k: d[k] for k in c.params()}, **c.args)
        assert torch.equal(d["x"], c.h) and torch.equal(d["y"], c.u)
        d = {k: wide(v).clone()[:, :width] if v is not None and v.dim() == 2 else v for k, v in c.dev.items()}
        dh, du = wide(c.dh).clone()[:, :width], wide(c.du).clone()[:, :width]
        dgate = d["gate"] if gate == "matrix" else None
        B.slicegcn_resnorm_bwd(d["x"], d["y"], c.stats, dh, du, dh, du, None, dgate=dgate, **{k: d[k] for k in c.params()}, **c.args)
        assert torch.equal(dh, c.dx) and torch.equal(du, c.dy) and (dgate is None or torch.equal(dgate, c.g["dgate"]))
        assert wide(dh)[:, width:].isnan().all() and wide(du)[:, width:].isnan().all()


def test_beyond_32_bit_offsets():
    n, ld, width = 60_000, 40_000, 32
    x = torch.zeros((n, ld), dtype=torch.bfloat16, device="cuda")
    x[:, :width] = torch.randn(n, width, device="cuda")
    u = torch.empty((n, ld), dtype=torch.bfloat16, device="cuda")
    small = torch.empty((n, width), dtype=torch.bfloat16, device="cuda")
    B.slicegcn_resnorm_fwd(x[:, :width], None, None, u[:, :width], pre=RMS)
    B.slicegcn_resnorm_fwd(x[:, :width].contiguous(), None, None, small, pre=RMS)
    assert torch.equal(u[:, :width], small)


@pytest.mark.parametrize("gate,sigmoid", [("column", True), ("matrix", False)])
def test_gradients_against_differences(gate, sigmoid):
    """<gradients, direction> against the slope of <h, dh> + <u, du> of the 64-bit forward form along the direction."""
    c = Call(11, 50, "f32", LAYER, RMS, gate, sigmoid, residual=0.8, eps=1e-3)
    c.forward()
    c.backward()
    dh, du = c.dh.cpu().to(F64), c.du.cpu().to(F64)
    way = {k: torch.randn(v.shape, generator=c.gen, dtype=F64) for k, v in c.f64.items() if v is not None}

    def value(t):
        r = Resnorm(**{k: None if v is None else v + t * way[k] for k, v in c.f64.items()}, **c.args)
        return float((r.h * dh).sum() + (r.u * du).sum())
    step = 1e-4
    slope = (8 * (value(step) - value(-step)) - (value(2 * step) - value(-2 * step))) / (12 * step)  # error of order step^4
    got = sum(float((c.g["d" + k].cpu().to(F64) * w).sum()) for k, w in way.items())
    size = sum(float((c.g["d" + k].cpu().to(F64) * w).abs().sum()) for k, w in way.items())
    assert abs(got - slope) <= (C * U + 1e-9) * size


def test_same_bits_on_any_stream_and_in_graphs():
    c = Call(5000, 160, "bf16", RMS, LAYER, "column", True)
    c.forward()
    c.backward()
    ws = torch.empty(B.slicegcn_resnorm_bwd_workspace_bytes(c.n, c.width), dtype=torch.uint8, device="cuda")

    def step():
        B.slicegcn_resnorm_fwd(c.dev["x"], c.dev["y"], c.h, c.u, stats=c.stats, **c.params(), **c.args)
        B.slicegcn_resnorm_bwd(c.dev["x"], c.dev["y"], c.stats, c.dh, c.du, c.dx, c.dy, ws, **{k: v for k, v in c.g.items() if k not in ("dx", "dy")},
                               **c.params(), **c.args)
    outs = [c.h, c.u, c.stats, *c.g.values()]
    first = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, outs))
    from paper_2408_11500_amd.stack import GraphedStep
    graph = GraphedStep(step)
    for i in range(4):
        c.dev["x"].normal_()
        c.dh.normal_()
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), i


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("width", [3, 9, 66, 100, 257, 602, 1001, 4097, 5001, 8193])
def test_one_infinity_in_a_row(width, kind):
    """A root mean square of infinity leaves zeros and, in the infinity's own column, NaN, wherever in the row it stands: also in columns that two
    lanes hold, where a row does not fill its lanes."""
    places = sorted({0, 1, width // 2, *range(max(width - 17, 0), width)})
    v = torch.randn((len(places), width), generator=torch.Generator().manual_seed(width)).to(TYPES[kind])
    for row, place in enumerate(places):
        v[row, place] = float("inf") if row % 2 else float("-inf")
    want = torch.zeros(v.shape)
    want[v.isinf()] = float("nan")
    u = torch.full_like(v, 5.0, device="cuda")
    same = lambda got: torch.equal(got.cpu().float().nan_to_num(9.0, 8.0, 7.0), want.nan_to_num(9.0))
    B.slicegcn_resnorm_fwd(v.cuda(), None, None, u, pre=RMS)
    assert same(u), "before a block"
    B.slicegcn_resnorm_fwd(None, v.cuda(), u, None, post=RMS)
    assert same(u), "after a block"
    B.slicegcn_resnorm_fwd(None, v.cuda(), u, None, post=RMS, post_b=torch.zeros(width, device="cuda"), post_w=torch.ones(width, device="cuda"))
    assert same(u), "with a bias"
    B.slicegcn_resnorm_fwd(v.cuda(), None, None, u, pre=LAYER)
    assert u.isnan().all(), "layer norm"


def large(n, width, kind, norm, gate, sigmoid, seed=0):
    """Operands of a call made on the device: rows of x, y, dh, du, and the parameters."""
    gen = torch.Generator(device="cuda").manual_seed(seed + n + width)
    values = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
    t = {k: values(n, width).to(TYPES[kind]) for k in ("x", "y", "dh", "du")}
    p = {"post_w": 1 + 0.3 * values(width), "pre_w": 1 + 0.3 * values(width)}
    if norm == LAYER:
        p.update(post_b=0.3 * values(width), pre_b=0.3 * values(width))
    p["gate"] = values(n, width).to(TYPES[kind]) if gate == "matrix" else 0.5 + 0.5 * values(width)
    return t, p, dict(post=norm, pre=norm, sigmoid=sigmoid, residual=0.75, eps=1e-3)


def run_large(t, p, args, params=True):
    """All results of the forward and the backward pass."""
    n, width = t["x"].shape
    out = {k: torch.full_like(t["x"], float("nan")) for k in ("h", "u", "dx", "dy")}
    out.update({"d" + k: torch.full_like(v, float("nan")) for k, v in p.items() if params or v.dim() == 2})
    stats = torch.full((n, 4), float("nan"), device="cuda")
    ws = torch.empty(B.slicegcn_resnorm_bwd_workspace_bytes(n, width), dtype=torch.uint8, device="cuda")
    B.slicegcn_resnorm_fwd(t["x"], t["y"], out["h"], out["u"], stats=stats, **p, **args)
    B.slicegcn_resnorm_bwd(t["x"], t["y"], stats, t["dh"], t["du"], out["dx"], out["dy"], ws,
                           **{k: v for k, v in out.items() if k not in ("h", "u", "dx", "dy")}, **p, **args)
    return out


# Rows so many that every lane group of the backward pass takes more than 32 of them, twice what it adds up before it sets a sum aside (on rows of up
# to 4096 columns); above that, several for every workgroup.
MANY = [("f32", 256, RMS, "column", 70_000), ("f32", 64, LAYER, "column", 280_001), ("bf16", 100, LAYER, "column", 280_001), ("bf16", 64, RMS, "matrix", 560_001),
        ("f32", 602, LAYER, "matrix", 36_001), ("f32", 1500, RMS, "column", 8_800), ("f16", 2048, RMS, "column", 17_600), ("bf16", 2500, LAYER, "matrix", 8_801),
        ("f32", 3, LAYER, "column", 1_120_001), ("f32", 5000, RMS, "column", 8_800), ("bf16", 5000, LAYER, "column", 8_800), ("bf16", 8192, LAYER, "matrix", 2_000)]
MANY += [(kind, width, norm, "column", 801) for kind in ("f32", "bf16") for width in (8193, 16_384) for norm in (RMS, LAYER)]


@pytest.mark.parametrize("kind,width,norm,gate,n", MANY)
def test_sums_over_many_rows_in_turn(kind, width, norm, gate, n):
    # A column's sum: 16 rows and 3 sums of those in a lane, up to 64 rows beside each other; the rest as above: within C
    t, p, args = large(n, width, kind, norm, gate, gate == "matrix")
    got = run_large(t, p, args)
    with torch.device("cuda"):
        f64 = {k: v.to(F64) for k, v in {**t, **p}.items()}
        dh, du = f64.pop("dh"), f64.pop("du")
        w = Resnorm(**f64, **args)
        want, size = w.backward(dh, du)
        want.update(h=w.h, u=w.u)
        size.update(h=w.h_size, u=w.u_size)
        for name, g in got.items():
            tol = C * U * size[name].reshape(g.shape) + half_step(want[name].reshape(g.shape), g.dtype)
            err = (g.to(F64) - want[name].reshape(g.shape)).abs()
            assert bool((err <= tol).all()), f"{name}: {float((err / tol).max()):.2f} of the bound"


@pytest.mark.parametrize("kind,width,norm,gate", [("f32", 256, RMS, "column"), ("bf16", 100, LAYER, "column"), ("f32", 602, LAYER, "matrix"), ("bf16", 64, RMS, "matrix"),
                                                  ("f32", 3, RMS, "column"), ("bf16", 2500, RMS, "column"), ("f16", 5000, LAYER, "column"), ("f32", 9000, RMS, "column")])
def test_rows_beyond_the_caches_have_the_bits_of_smaller_calls(kind, width, norm, gate):
    """Results of 256 MB and more are stored past the caches; rows do not depend on each other."""
    n = (256 << 20) // (2 * width * (4 if kind == "f32" else 2)) + 1001
    t, p, args = large(n, width, kind, norm, gate, gate == "matrix")
    whole = run_large(t, p, args, params=False)
    for a in range(0, n, n // 3 + 1):
        part = slice(a, a + n // 3 + 1)
        got = run_large({k: v[part] for k, v in t.items()}, {k: v[part] if v.dim() == 2 else v for k, v in p.items()}, args, params=False)
        for name, g in got.items():
            assert torch.equal(g, whole[name][part]), (name, a)


@pytest.mark.parametrize("width", [3, 64, 101, 602, 5000, 9000])
@pytest.mark.parametrize("post", [NONE, LAYER])
def test_gradients_of_gates_that_are_wide_open_or_shut(width, post):
    """s (1 - s) of a gate near 1 keeps its relative precision, as that of one near 0 does."""
    n = 40
    gate = torch.linspace(-80, 80, n)[:, None] + torch.linspace(0, 4, width)[None]
    gen = torch.Generator().manual_seed(width)
    y, dh = (torch.randn((n, width), generator=gen) for _ in range(2))
    h, dgate = (torch.empty((n, width), device="cuda") for _ in range(2))
    stats = torch.empty((n, 4), device="cuda")
    args = dict(post=post, gate=gate.cuda(), sigmoid=True, eps=1e-3)
    B.slicegcn_resnorm_fwd(None, y.cuda(), h, None, stats=stats, **args)
    B.slicegcn_resnorm_bwd(None, y.cuda(), stats, dh.cuda(), None, None, None, None, dgate=dgate, **args)
    g = gate.to(F64)
    small = torch.exp(-g.abs()) / (1 + torch.exp(-g.abs()))
    p = y.to(F64) if post == NONE else (y.to(F64) - stats.cpu().to(F64)[:, :1]) * stats.cpu().to(F64)[:, 1:2]
    size = p.abs() if post == NONE else (y.to(F64).abs() + stats.cpu().to(F64)[:, :1].abs()) * stats.cpu().to(F64)[:, 1:2]
    # exp within a unit in the last place (2), its sum, quotient and products (4 roundings of it, each twice in the slope), three products more
    bound = 16 * U * dh.to(F64).abs() * size * small * (1 - small)
    assert_within(dgate, dh.to(F64) * p * small * (1 - small), bound, "dgate")


def test_gradients_of_column_gates_that_are_wide_open_or_shut():
    n, width = 40, 161
    gate = torch.linspace(-80, 80, width)
    gen = torch.Generator().manual_seed(width)
    y, dh = (torch.randn((n, width), generator=gen) for _ in range(2))
    h, dgate = torch.empty((n, width), device="cuda"), torch.full((width,), float("nan"), device="cuda")
    stats = torch.empty((n, 4), device="cuda")
    ws = torch.empty(B.slicegcn_resnorm_bwd_workspace_bytes(n, width), dtype=torch.uint8, device="cuda")
    args = dict(gate=gate.cuda(), sigmoid=True)
    B.slicegcn_resnorm_fwd(None, y.cuda(), h, None, stats=stats, **args)
    B.slicegcn_resnorm_bwd(None, y.cuda(), stats, dh.cuda(), None, None, None, ws, dgate=dgate, **args)
    small = torch.exp(-gate.to(F64).abs()) / (1 + torch.exp(-gate.to(F64).abs()))
    terms = dh.to(F64) * y.to(F64) * small * (1 - small)
    assert_within(dgate, terms.sum(0), C * U * terms.abs().sum(0), "dgate")
