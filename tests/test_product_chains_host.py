"""How far the sums of products run before they are joined in fp64, without a GPU: by the room that their parts take."""
import pytest

from paper_2408_11500_amd import binding as B
from test_abi_host import L  # noqa: F401  (a fixture)


@pytest.mark.parametrize("type", [B.BF16, B.F16])
@pytest.mark.parametrize("n", [1024 * 32 * 256, 1024 * 32 * 256 + 1, 100_000_000, 2**31 - 2**16])
@pytest.mark.parametrize("w_in,w_out", [(100, 256), (128, 128), (2, 2)])
def test_one_sweep_over_many_rows_has_chains_of_1024_steps(L, w_in, w_out, n, type):  # noqa: F811
    """A sum of dW for every 1024 blocks of 32 rows, and column sums of as many parts, beside the gradients before the activation."""
    parts = -(-n // (1024 * 32))
    for q, size in ((1, L.slicegcn_product_bwd_workspace_bytes), (2, L.slicegcn_gated_bwd_workspace_bytes)):
        if w_out * q > 256:
            continue
        rows = q * n * -(-w_out // 8) * 8 * 2
        assert size(n, w_in, w_out, type) - rows >= parts * q * w_out * (4 * w_in + 8)
