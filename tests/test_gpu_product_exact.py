"""Products of small integers, whose sums are integers below 2^24: every sum in fp32 is exact, in whatever order, and a result is that of the formula rounded once.  Rows or
terms that are left out, or counted twice, show whatever their number."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from train_util import F64, TYPES

pytestmark = pytest.mark.gpu


def integers(gen, rows, cols, dtype, most=2, ld=None):
    """(matrix of the type, the same in 64 bits): integers from -most to most, all exact in any of the types."""
    ld = cols if ld is None else ld
    buf = torch.full((rows, ld), float("nan"), dtype=dtype, device="cuda")
    v = torch.randint(-most, most + 1, (rows, cols), generator=gen, device="cuda").to(dtype)
    buf[:, :cols] = v
    return buf[:, :cols], v.to(F64)


def products_exact(*pairs):
    """Sums of a @ b in 64 bits, whose every partial sum fp32 holds exactly."""
    assert float(sum((a.abs() @ b.abs()).max() for a, b in pairs)) < 2 ** 24
    return sum(a @ b for a, b in pairs)


def assert_rounded(got, want, what):
    want = want.to(torch.float32).to(got.dtype)  # exact in fp32
    assert torch.equal(got, want), f"{what}: {int((got != want).sum())} of {want.numel()} differ"


def workspace(count):
    return torch.full((count,), 0xFF, dtype=torch.uint8, device="cuda")


def check(n, wi, wo, dtype, relu, seed=0, ld=0, forward=True, gated=True):
    """Both operators, forward and backward.  ld: elements behind each row."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    make = lambda cols, most=2: integers(gen, n, cols, dtype, most, cols + ld)
    x, x64 = make(wi, 1)
    (wg, wg64), (wu, wu64) = (integers(gen, wi, wo, dtype, 1) for _ in range(2))
    b = torch.randint(-3, 4, (wo,), generator=gen, device="cuda").float()
    act, positive = (B.ACT_RELU, lambda t: t.clamp(min=0)) if relu else (B.ACT_NONE, lambda t: t)
    out = lambda cols: torch.full((n, cols + ld), 777.0, dtype=dtype, device="cuda")[:, :cols]
    if forward:
        r, r64 = make(wo)
        y, p = out(wo), out(wo)
        B.slicegcn_product_fwd(x, wg, y, workspace(B.slicegcn_product_fwd_workspace_bytes(n, wi, wo, dtype)), b=b, R=r, P=p, act=act, residual=2.0)
        p64 = products_exact((x64, wg64)) + b
        assert_rounded(p, p64, "P")
        assert_rounded(y, positive(p64) + 2 * r64, "Y")
        if gated:
            u64 = products_exact((x64, wu64))
            assert (p64 * u64).abs().max() < 2 ** 24
            B.slicegcn_gated_fwd(x, wg, wu, y, workspace(B.slicegcn_gated_fwd_workspace_bytes(n, wi, wo, dtype)), bg=b, G=p, U=r, act=act)
            assert_rounded(y, positive(p64) * u64, "H")
            assert_rounded(p, p64, "G")
            assert_rounded(r, u64, "U")
        del r, y, p, r64, p64
    d, d64 = make(wo)
    g, g64 = make(wo)
    dx, dw, db = out(wi), torch.full_like(wg, 777.0), torch.full((wo,), 777.0, device="cuda")
    B.slicegcn_product_bwd(x, wg, g if relu else None, d, workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype)), dX=dx, dW=dw, db=db, act=act)
    dp = d64 * (g64 > 0) if relu else d64
    assert_rounded(dx, products_exact((dp, wg64.t())), "dX")
    assert_rounded(dw, products_exact((x64.t(), dp)), "dW")
    assert_rounded(db, dp.sum(0), "db")
    if gated:
        u, u64 = make(wo)
        dwu, dbu = torch.full_like(wg, 777.0), torch.full((wo,), 777.0, device="cuda")
        B.slicegcn_gated_bwd(x, wg, wu, g, u, d, workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype)), dX=dx, dWg=dw, dWu=dwu, dbg=db, dbu=dbu, act=act)
        dg, du = d64 * u64 * (g64 > 0 if relu else 1), d64 * positive(g64)
        assert_rounded(dx, products_exact((dg, wg64.t()), (du, wu64.t())), "dX")
        assert_rounded(dw, products_exact((x64.t(), dg)), "dWg")
        assert_rounded(dwu, products_exact((x64.t(), du)), "dWu")
        assert_rounded(db, dg.sum(0), "dbg")
        assert_rounded(dbu, du.sum(0), "dbu")


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size", [(1024 * 32 * 256 + 1, 4, 8), (1024 * 32 * 256 + 32 * 256 + 5, 34, 6), (3 * 1024 * 32 * 256 - 31, 2, 2)], ids=str)
def test_one_sweep_over_more_rows_than_a_workgroup_a_cu_takes(size, kind):
    check(*size, TYPES[kind], True, forward=False)
