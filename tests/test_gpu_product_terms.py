"""Backward passes that keep the gradients before the activation in two terms because the caller asks for it."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from product_util import STEPS, act, depth
from test_gpu_product_guards import Guarded
from test_gpu_product_rounded import ACT, check
from train_util import F64, TYPES, U, half_step

pytestmark = pytest.mark.gpu


def make(gen, rows, cols, dtype, std=1.0, ld=0):
    return (torch.randn((rows, cols + ld), generator=gen, device="cuda") * std).to(dtype)[:, :cols]


def in_two(v, off, dtype):
    """What two terms hold of a number within `off` of v: all but half a step of a second term, which is at most half a step of the first."""
    return v, off + U * v.abs() + half_step(half_step(v.abs() + off, dtype), dtype)


# short passes; through registers with sums whole and cut, few rows, odd widths; narrow layers of many rows; tiles of 256 x 256, whole, cut, with more tiles than a round; operands
# that are copied; rows of dX that do not fit one turn
SIZES = [(3, 7, 5), (33, 65, 129), (700, 264, 300), (3000, 300, 136), (12_000, 400, 200), (2050, 701, 331), (20, 4096, 3000), (16_384, 100, 128), (33_333, 72, 40), (20_000, 72, 7000),
         (4100, 4400, 4616), (513, 5000, 4104), (2050, 2003, 2521), (140, 8401, 9103), (200_001, 200, 24)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("name", ACT)
def test_gradients(size, name, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator(device="cuda").manual_seed(SIZES.index(size))
    ld = (0, 3, 8)[SIZES.index(size) % 3]
    x, g, u, d = make(gen, n, wi, dtype, ld=ld), make(gen, n, wo, dtype, 1.5, ld), make(gen, n, wo, dtype), make(gen, n, wo, dtype, ld=ld)
    wg, wu = (make(gen, wi, wo, dtype, wi ** -0.5) for _ in range(2))
    x64, g64, u64, d64, wg64, wu64 = (t.to(F64) for t in (x, g, u, d, wg, wu))
    none = torch.zeros_like
    y, slope = act(g64, name)
    t = Guarded(dtype)
    dx, dw, dwu, db = t.rows(n, wi, wi + ld), t.flat(wi, wo), t.flat(wi, wo), t.flat(wo, dtype=torch.float32)
    ws = t.workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype, two_terms=True))
    B.slicegcn_product_bwd(x, wg, g, d, ws, dX=dx, dW=dw, db=db, act=ACT[name], two_terms=True)
    dp, ep = in_two(d64 * slope, d64.abs() * U * (STEPS * (1 + g64.abs()) + 2), dtype)
    check(dx, [(dp, ep, wg64.t(), none(wg64.t()))], dtype, "dX")
    check(dw, [(x64.t(), none(x64.t()), dp, ep)], dtype, "dW")
    plain = torch.empty_like(db)
    B.slicegcn_product_bwd(x, wg, g, d, torch.empty_like(ws), db=plain, act=ACT[name])
    assert ((db - plain).abs() <= 2.0 ** -20 * (1 + d64.abs().sum(0))).all()
    ws = t.workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype, two_terms=True))
    B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, dX=dx, dWg=dw, dWu=dwu, act=ACT[name], two_terms=True)
    dg, eg = in_two(d64 * u64 * slope, d64.abs() * u64.abs() * U * (STEPS * (1 + g64.abs()) + 2), dtype)
    du, eu = in_two(d64 * y, d64.abs() * U * (STEPS + 2) * g64.abs(), dtype)
    check(dx, [(dg, eg, wg64.t(), none(wg64.t())), (du, eu, wu64.t(), none(wu64.t()))], dtype, "dX")
    check(dw, [(x64.t(), none(x64.t()), dg, eg)], dtype, "dWg")
    check(dwu, [(x64.t(), none(x64.t()), du, eu)], dtype, "dWu")
    for k, both in (("dX", dx), ("dWg", dw), ("dWu", dwu)):
        alone = torch.full_like(both, 777.0)
        B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, act=ACT[name], two_terms=True, **{k: alone})
        assert torch.equal(alone, both), k
    for buf, count, width in t.buffers:  # written again since: only what lies behind is looked at
        assert (buf[count:] == (0xA5 if buf.dtype is torch.uint8 else 777.0)).all()
        assert width is None or (buf[:count, width:] == 777.0).all()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", [(40, 96, 64), (16_384, 100, 128), (2050, 2003, 2521)], ids=str)
def test_where_one_term_is_all_there_is(size, kind):
    """Without an activation, and of fp32 rows, asking for two terms changes no bit; nor does it in a forward pass."""
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, g, d, wg, wu = make(gen, n, wi, dtype), make(gen, n, wo, dtype), make(gen, n, wo, dtype), make(gen, wi, wo, dtype), make(gen, wi, wo, dtype)
    ws = torch.empty(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype, two_terms=True), dtype=torch.uint8, device="cuda")

    def run(two):
        out = [torch.empty_like(t) for t in (x, wg, x, wg, wg)]
        B.slicegcn_product_bwd(x, wg, None, d, ws, dX=out[0], dW=out[1], two_terms=two)
        if dtype is torch.float32:
            B.slicegcn_gated_bwd(x, wg, wu, g, d, d, ws, dX=out[2], dWg=out[3], dWu=out[4], two_terms=two)
        return out[:5 if dtype is torch.float32 else 2]
    for a, b in zip(run(False), run(True)):
        assert torch.equal(a, b)


def test_no_rows():
    e = lambda w: torch.empty((0, w), dtype=torch.bfloat16, device="cuda")
    w = torch.ones((5, 7), dtype=torch.bfloat16, device="cuda")
    dwg, dwu = (torch.full_like(w, 777.0) for _ in range(2))
    ws = torch.empty(B.slicegcn_gated_bwd_workspace_bytes(0, 5, 7, torch.bfloat16, two_terms=True), dtype=torch.uint8, device="cuda")
    B.slicegcn_gated_bwd(e(5), w, w, e(7), e(7), e(7), ws, dX=e(5), dWg=dwg, dWu=dwu, two_terms=True)
    assert (dwg == 0).all() and (dwu == 0).all()


@pytest.mark.parametrize("size", [(70, 96, 264), (3000, 300, 136)], ids=str)
def test_captured(size):
    n, wi, wo = size
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, g, u, d, wg, wu = (make(gen, *s, torch.bfloat16) for s in ((n, wi), (n, wo), (n, wo), (n, wo), (wi, wo), (wi, wo)))

    def call(out, ws):
        B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, dX=out[0], dWg=out[1], dWu=out[2], two_terms=True)
    buffers = lambda: ([torch.empty_like(t) for t in (x, wg, wu)],
                       torch.empty(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, torch.bfloat16, two_terms=True), dtype=torch.uint8, device="cuda"))
    captured, eager = buffers(), buffers()
    call(*captured)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(*captured)
    for seed in range(3):
        d.copy_(make(torch.Generator(device="cuda").manual_seed(seed), n, wo, torch.bfloat16))
        call(*eager)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured[0], eager[0]))
