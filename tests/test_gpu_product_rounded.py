"""Backward passes through an activation whose gradients before it are rounded once: dX and dW against the products of gradients that are rounded too, so that what is left is
the kernels' own error, not half a step of each gradient."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from product_util import STEPS, act, depth
from train_util import F64, TYPES, U, assert_within

pytestmark = pytest.mark.gpu
ACT = dict(silu=B.ACT_SILU, gelu=B.ACT_GELU)


def rounded(v, off, dtype):
    """The middle of what a number within `off` of v can be rounded to, and how far that reaches to either side."""
    off = off + U * v.abs()  # and the way to the type through fp32
    lo, hi = ((v + s * off).to(dtype).to(F64) for s in (-1, 1))
    return (lo + hi) / 2, (hi - lo) / 2


def check(got, pairs, dtype, what):
    """got = sum of a @ b over (a, its error, b, its error)."""
    want = sum(a @ b for a, ea, b, eb in pairs)
    k = sum(a.shape[1] for a, *_ in pairs)
    bound = sum(ea @ b.abs() + a.abs() @ eb + depth(k, dtype) * ((a.abs() + ea) @ (b.abs() + eb)) for a, ea, b, eb in pairs)
    assert_within(got, want.cpu(), bound.cpu(), what)


# one sweep over many rows; through registers; in tiles of 256 x 256, whole, cut and with a last round cut along k; operands that are copied.  More gradients than are kept in two terms
SIZES = [(16_384, 100, 256), (33_333, 72, 40), (60_000, 34, 126), (3000, 300, 136), (12_000, 400, 200), (2050, 701, 331), (20_000, 72, 7000), (4100, 4400, 4616),
         (513, 5000, 4104), (2050, 2003, 2521)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("name", ACT)
def test_backward(size, name, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    assert n * wo > 1 << 15
    gen = torch.Generator(device="cuda").manual_seed(SIZES.index(size))
    make = lambda rows, cols, std=1.0: (torch.randn((rows, cols), generator=gen, device="cuda") * std).to(dtype)
    x, g, u, d, wg, wu = make(n, wi), make(n, wo, 1.5), make(n, wo), make(n, wo), make(wi, wo, wi ** -0.5), make(wi, wo, wi ** -0.5)
    x64, g64, u64, d64, wg64, wu64 = (t.to(F64) for t in (x, g, u, d, wg, wu))
    zero = lambda t: torch.zeros_like(t)
    ws = lambda count: torch.full((count,), 0xFF, dtype=torch.uint8, device="cuda")
    y, slope = act(g64, name)
    dx, dw, dwu = (torch.full_like(t, 777.0) for t in (x, wg, wg))
    B.slicegcn_product_bwd(x, wg, g, d, ws(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype)), dX=dx, dW=dw, act=ACT[name])
    dp, ep = rounded(d64 * slope, d64.abs() * U * (STEPS * (1 + g64.abs()) + 2), dtype)
    check(dx, [(dp, ep, wg64.t(), zero(wg64.t()))], dtype, "dX")
    check(dw, [(x64.t(), zero(x64.t()), dp, ep)], dtype, "dW")
    del dp, ep
    B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype)), dX=dx, dWg=dw, dWu=dwu, act=ACT[name])
    dg, eg = rounded(d64 * u64 * slope, d64.abs() * u64.abs() * U * (STEPS * (1 + g64.abs()) + 2), dtype)
    du, eu = rounded(d64 * y, d64.abs() * U * (STEPS + 2) * g64.abs(), dtype)
    check(dx, [(dg, eg, wg64.t(), zero(wg64.t())), (du, eu, wu64.t(), zero(wu64.t()))], dtype, "dX")
    check(dw, [(x64.t(), zero(x64.t()), dg, eg)], dtype, "dWg")
    check(dwu, [(x64.t(), zero(x64.t()), du, eu)], dtype, "dWu")
