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


# through registers in each tile shape, with sums whole and cut, on whole units, even and odd widths; few rows in strips; both products in one launch
SIZES = [(1, 1, 1), (1, 64, 96), (1, 4104, 136), (3, 7, 5), (16, 40, 64), (17, 2304, 72), (24, 1024, 200), (32, 2048, 1001), (33, 65, 129), (65, 72, 200), (128, 1000, 40),
         (257, 520, 384), (300, 264, 520), (300, 1003, 71), (1000, 72, 40), (2048, 64, 170), (2049, 512, 128), (5000, 24, 8), (5000, 1001, 333), (16_383, 100, 256),
         (9000, 700, 260)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("relu", [False, True])
def test_short_and_middling_products(size, relu, kind):
    check(*size, TYPES[kind], relu, seed=SIZES.index(size), ld=(0, 3, 8)[SIZES.index(size) % 3])


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", [(16_384, 100, 256), (16_385, 100, 128), (33_333, 72, 40), (20_011, 128, 126), (17_000, 6, 2), (60_001, 34, 250)], ids=str)
@pytest.mark.parametrize("relu", [False, True])
def test_narrow_layers_of_many_rows(size, relu, kind):
    check(*size, TYPES[kind], relu, ld=2)


# tiles of 256 x 256: sums cut, whole, of an odd number of steps, a last round cut along k in dX, in one dW and in both, sums over many rows, operands that are copied
LONG = [(513, 5000, 4104), (20_000, 72, 7000), (2500, 2056, 2000), (4100, 4400, 4616), (4100, 4400, 3768), (8200, 9064, 136), (2050, 2003, 2521), (9001, 1026, 1101), (40_000, 512, 520)]


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size", LONG, ids=str)
@pytest.mark.parametrize("relu", [False, True])
def test_long_products(size, relu, kind):
    check(*size, TYPES[kind], relu, seed=LONG.index(size))


# widths in whole units, rows that are none: leading dimensions and bases off 16 bytes
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("size,ld", [((2500, 2056, 2000), 1), ((2500, 2056, 2000), 4), ((4100, 2400, 1808), 3)], ids=str)
def test_long_products_of_rows_that_lie_oddly_at_widths_in_whole_units(size, ld, kind):
    check(*size, TYPES[kind], True, ld=ld)


@pytest.mark.parametrize("size", [(60_000, 300, 130), (3000, 1200, 700)], ids=str)
def test_fp32_in_large_tiles(size):
    check(*size, torch.float32, True, ld=1)
