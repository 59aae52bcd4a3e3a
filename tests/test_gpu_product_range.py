"""Products of fp32 operands at the lower end of their range."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from product_util import depth
from train_util import F64, assert_within

pytestmark = pytest.mark.gpu
LEAST = 2.0 ** -134  # half of the smallest 16-bit term


@pytest.mark.parametrize("exponent", [-100, -110, -112, -118, -126, -131])
@pytest.mark.parametrize("size", [(64, 1, 64), (5, 300, 40), (300, 700, 200)], ids=str)
def test_small_operands(size, exponent):
    n, wi, wo = size
    gen = torch.Generator().manual_seed(-exponent)
    x = torch.randn((n, wi), generator=gen) * 2.0 ** exponent
    w = torch.randn((wi, wo), generator=gen) * 2.0 ** 20
    y = torch.empty((n, wo), device="cuda")
    B.slicegcn_product_fwd(x.cuda(), w.cuda(), y, torch.empty(B.slicegcn_product_fwd_workspace_bytes(n, wi, wo, torch.float32), dtype=torch.uint8, device="cuda"))
    x, w = x.to(F64), w.to(F64)
    # the products of what is left of an operand, and a term of a product is 2^-126 at least or may be taken for 0
    bound = depth(wi, torch.float32) * (x.abs() @ w.abs()) + LEAST * w.abs().sum(0) + wi * 6 * 2.0 ** -126
    assert_within(y, x @ w, bound, "Y")
