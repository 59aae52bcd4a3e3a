"""Asking for two terms of the gradients before the activation, without a GPU: types and workspaces."""
import pytest

from paper_2408_11500_amd import binding as B
from test_abi_host import L  # noqa: F401  (a fixture)
from test_block_host import GOOD, call, desc


@pytest.mark.parametrize("op,way", GOOD)
def test_types(L, op, way):  # noqa: F811
    wide = dict(w_in=4096, w_out=512)
    for t in (B.F32, B.BF16, B.F16):
        assert call(L, op, way, d=desc(3, **wide, type=t | B.TWO_TERMS), ld=4096, ws=None, ws_bytes=0) == B.EWORKSPACE
    for t in (3 | B.TWO_TERMS, B.BF16 | 2 * B.TWO_TERMS, -1 & ~B.TWO_TERMS):
        assert call(L, op, way, d=desc(type=t)) == B.EINVAL
        assert getattr(L, f"slicegcn_{op}_{way}_workspace_bytes")(3, 8, 8, t) == 0


@pytest.mark.parametrize("n", [0, 1, 3, 2048, 16_384, 2_449_029, 2**31 - 2**16])
@pytest.mark.parametrize("w_in,w_out", [(1, 1), (64, 170), (100, 128), (4096, 1024), (10240, 4096)])
def test_workspaces(L, n, w_in, w_out):  # noqa: F811
    for op in ("product", "gated"):
        fwd, bwd = (getattr(L, f"slicegcn_{op}_{way}_workspace_bytes") for way in ("fwd", "bwd"))
        for t in (B.F32, B.BF16, B.F16):
            assert fwd(n, w_in, w_out, t | B.TWO_TERMS) == fwd(n, w_in, w_out, t)
        assert bwd(n, w_in, w_out, B.F32 | B.TWO_TERMS) == bwd(n, w_in, w_out, B.F32)
        q = 2 if op == "gated" else 1
        rows = q * n * -(-w_out // 8) * 8 * 2
        for t in (B.BF16, B.F16):
            one, two = bwd(n, w_in, w_out, t), bwd(n, w_in, w_out, t | B.TWO_TERMS)
            assert two % 256 == 0 and two >= one and two >= 2 * rows
            # the second term, sums of two parts of a turn of dX, and two for one of each part of dW
            assert two <= 2 * one + rows + (512 << 20) + 2 * q * 4 * w_in * w_out * (1 + n // 32768) + 4096


@pytest.mark.parametrize("op", ["product", "gated"])
def test_a_workspace_for_one_term_is_refused(L, op):  # noqa: F811
    n, w_in, w_out = 3000, 300, 136
    one = getattr(L, f"slicegcn_{op}_bwd_workspace_bytes")(n, w_in, w_out, B.BF16)
    d = desc(n, w_in, w_out, B.BF16 | B.TWO_TERMS, act=B.ACT_GELU)
    assert call(L, op, "bwd", d=d, ld=300, ws_bytes=one) == B.EWORKSPACE
