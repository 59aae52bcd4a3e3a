"""What lies behind the last row of a result, behind gradients of weights and biases and behind the workspace stays as it was."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from train_util import TYPES

pytestmark = pytest.mark.gpu
ACT = (B.ACT_NONE, B.ACT_RELU, B.ACT_SILU, B.ACT_GELU)
ROWS, MORE = 260, 1 << 16  # rows behind the last one (more than the tallest tile has), elements behind others


class Guarded:
    """Tensors of a call, each amid 777 (bytes: 0xA5)."""

    def __init__(self, dtype):
        self.dtype, self.buffers = dtype, []

    def rows(self, n, width, ld):
        buf = torch.full((n + ROWS, ld), 777.0, dtype=self.dtype, device="cuda")
        self.buffers.append((buf, n, width))
        return buf[:n, :width]

    def flat(self, *shape, dtype=None):
        count = torch.Size(shape).numel()
        buf = torch.full((count + MORE,), 777.0, dtype=dtype or self.dtype, device="cuda")
        self.buffers.append((buf, count, None))
        return buf[:count].view(shape)

    def workspace(self, count):
        buf = torch.full((count + MORE,), 0xA5, dtype=torch.uint8, device="cuda")
        buf[:count] = 0xFF
        self.buffers.append((buf, count, None))
        return buf[:count]

    def check(self, what):
        for i, (buf, n, width) in enumerate(self.buffers):
            guard = 0xA5 if buf.dtype is torch.uint8 else 777.0
            assert (buf[n:] == guard).all(), (what, i, "behind the end")
            if width is not None:
                assert (buf[:n, width:] == guard).all(), (what, i, "behind the last column")
                assert (buf[:n, :width] != guard).all(), (what, i, "not written")
        self.buffers.clear()


# all forms, with few rows in the last tile
SIZES = [(1, 8, 8), (1, 64, 96), (1, 1001, 35), (1, 4104, 136), (17, 40, 64), (17, 2304, 1032), (31, 700, 75), (33, 65, 129), (33, 4096, 256), (65, 72, 200), (65, 513, 70),
         (129, 264, 1032), (257, 520, 384), (257, 1001, 333), (2049, 64, 170), (16_385, 100, 128), (16_389, 34, 126), (40_001, 256, 130),
         (257, 9000, 5000), (4097, 4400, 2600), (2049, 2003, 2521), (20_001, 72, 7000)]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("ld", [0, 5])
def test_nothing_is_written_behind_the_end(size, ld, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    act = ACT[(SIZES.index(size) + ld) % 4]
    gen = torch.Generator(device="cuda").manual_seed(2)
    make = lambda rows, cols: torch.randn((rows, cols + ld), generator=gen, device="cuda").to(dtype)[:, :cols]
    x, r, g, u, d = make(n, wi), *(make(n, wo) for _ in range(4))
    wg, wu = ((torch.randn((wi, wo), generator=gen, device="cuda") / wi ** 0.5).to(dtype) for _ in range(2))
    bias = torch.randn(wo, generator=gen, device="cuda")
    t = Guarded(dtype)
    B.slicegcn_product_fwd(x, wg, t.rows(n, wo, wo + ld), t.workspace(B.slicegcn_product_fwd_workspace_bytes(n, wi, wo, dtype)), b=bias, R=r, P=t.rows(n, wo, wo + 3), act=act)
    t.check("product_fwd")
    B.slicegcn_gated_fwd(x, wg, wu, t.rows(n, wo, wo + ld), t.workspace(B.slicegcn_gated_fwd_workspace_bytes(n, wi, wo, dtype)), bg=bias, G=t.rows(n, wo, wo),
                         U=t.rows(n, wo, wo + 1), act=act)
    t.check("gated_fwd")
    B.slicegcn_product_bwd(x, wg, g, d, t.workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype)), dX=t.rows(n, wi, wi + ld), dW=t.flat(wi, wo),
                           db=t.flat(wo, dtype=torch.float32), act=act)
    t.check("product_bwd")
    B.slicegcn_product_bwd(x, wg, g, d, t.workspace(B.slicegcn_product_bwd_workspace_bytes(n, wi, wo, dtype)), dX=t.rows(n, wi, wi + ld), dR=t.rows(n, wo, wo + ld), act=act)
    t.check("product_bwd with dR")
    B.slicegcn_gated_bwd(x, wg, wu, g, u, d, t.workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype)), dX=t.rows(n, wi, wi + ld), dWg=t.flat(wi, wo),
                         dWu=t.flat(wi, wo), dbg=t.flat(wo, dtype=torch.float32), dbu=t.flat(wo, dtype=torch.float32), act=act)
    t.check("gated_bwd")
    for alone in ("dWg", "dWu"):
        B.slicegcn_gated_bwd(x, wg, wu, g, u, d, t.workspace(B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype)), **{alone: t.flat(wi, wo)}, act=act)
        t.check(alone)
