"""Either gradient of a gated projection's weights alone, in the bits that it has beside the other."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from train_util import TYPES

pytestmark = pytest.mark.gpu


# one sweep over many rows; a last round of tiles of 256 x 256 that is cut along k (320 tiles of both, of 64 in one round more; 648; with an end within a tile); sums that are cut;
# through registers; in one launch with dX
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("size", [(16_384, 100, 128), (33_333, 34, 42), (4100, 4096, 2560), (4100, 4400, 4616), (8200, 3340, 3001), (9000, 700, 260), (3000, 1000, 130),
                                  (2048, 64, 170), (40, 96, 64)], ids=str)
def test_weights_gradients(size, kind):
    n, wi, wo = size
    dtype = TYPES[kind]
    gen = torch.Generator(device="cuda").manual_seed(1)
    make = lambda rows, cols, std=1.0: (torch.randn((rows, cols), generator=gen, device="cuda") * std).to(dtype)
    x, g, u, d, wg, wu = make(n, wi), make(n, wo, 1.5), make(n, wo), make(n, wo), make(wi, wo, wi ** -0.5), make(wi, wo, wi ** -0.5)
    ws = torch.full((B.slicegcn_gated_bwd_workspace_bytes(n, wi, wo, dtype),), 0xFF, dtype=torch.uint8, device="cuda")

    def form(*names):
        out = {k: torch.full_like(x if k == "dX" else wg, 777.0) for k in names}
        B.slicegcn_gated_bwd(x, wg, wu, g, u, d, ws, **out)
        return out
    both = form("dX", "dWg", "dWu")
    for names in (("dWg",), ("dWu",), ("dWg", "dWu"), ("dX", "dWg"), ("dX", "dWu")):
        for k, t in form(*names).items():
            assert torch.equal(t, both[k]), (names, k, int((t != both[k]).sum()))
