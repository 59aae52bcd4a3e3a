"""One row whose leading dimension says nothing: the last of a long sequence, as hidden[:, -1] has it."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from train_util import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("wi,wo", [(1024, 2816), (4096, 136), (1000, 1000), (77, 35)], ids=str)
def test_the_last_row_of_a_sequence_gives_the_bits_of_a_row_by_itself(wi, wo, kind):
    dtype = TYPES[kind]
    gen = torch.Generator(device="cuda").manual_seed(1)
    steps = (1 << 21) // min(wi, wo) + 2
    make = lambda cols: torch.randn((1, cols), generator=gen, device="cuda").to(dtype)
    rows = dict(x=make(wi), r=make(wo), g=make(wo), u=make(wo), d=make(wo))
    wg, wu = ((torch.randn((wi, wo), generator=gen, device="cuda") / wi ** 0.5).to(dtype) for _ in range(2))
    ws = torch.empty(max(f(1, wi, wo, dtype) for f in (B.slicegcn_product_fwd_workspace_bytes, B.slicegcn_product_bwd_workspace_bytes,
                                                       B.slicegcn_gated_fwd_workspace_bytes, B.slicegcn_gated_bwd_workspace_bytes)), dtype=torch.uint8, device="cuda")

    def run(place):
        t = {k: place(v.shape[1]).copy_(v) for k, v in rows.items()}
        o = {k: place(w) for k, w in dict(y=wo, p=wo, h=wo, kg=wo, ku=wo, dx=wi, dr=wo, dx2=wi).items()}
        dw = [torch.empty_like(wg) for _ in range(3)]
        B.slicegcn_product_fwd(t["x"], wg, o["y"], ws, R=t["r"], P=o["p"], act=B.ACT_GELU)
        B.slicegcn_gated_fwd(t["x"], wg, wu, o["h"], ws, G=o["kg"], U=o["ku"])
        B.slicegcn_product_bwd(t["x"], wg, t["g"], t["d"], ws, dX=o["dx"], dW=dw[0], dR=o["dr"], act=B.ACT_GELU, residual=0.5)
        B.slicegcn_gated_bwd(t["x"], wg, wu, t["g"], t["u"], t["d"], ws, dX=o["dx2"], dWg=dw[1], dWu=dw[2])
        return [*o.values(), *dw]
    far = lambda cols: torch.empty((1, steps, cols), dtype=dtype, device="cuda")[:, -1]
    assert far(min(wi, wo)).stride(0) > 1 << 21
    # a row that begins where rows of a sequence do: whether that is on 16 bytes decides between forms of the 16-bit products
    near = lambda cols: torch.empty((steps, cols), dtype=dtype, device="cuda")[-1].view(1, cols)
    for a, b in zip(run(far), run(near)):
        assert torch.equal(a, b)
