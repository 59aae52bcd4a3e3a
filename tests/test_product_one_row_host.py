"""Which leading dimensions products take, without a GPU."""
import pytest

from paper_2408_11500_amd import binding as B
from test_abi_host import L  # noqa: F401  (a fixture)
from test_block_host import GOOD, call, desc


@pytest.mark.parametrize("op,way", GOOD)
def test_one_row_may_be_any_distance_from_the_next(L, op, way):  # noqa: F811
    wide = dict(w_in=4096, w_out=512)  # sums that are cut: without a workspace the call ends there, with all other checks behind it
    for ld in ((1 << 21) + 1, 1 << 40):
        assert call(L, op, way, d=desc(n=1, **wide), ld=ld, ws=None, ws_bytes=0) == B.EWORKSPACE
        assert call(L, op, way, d=desc(n=2, **wide), ld=ld, ws=None, ws_bytes=0) == B.ERANGE
    assert call(L, op, way, d=desc(n=1, **wide), ld=511, ws=None, ws_bytes=0) == B.EINVAL
