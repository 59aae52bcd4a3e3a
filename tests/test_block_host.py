"""Products, gated projections and AdamW without a GPU: exported symbols, workspace sizes, and refusals before any device work."""
import ctypes

import pytest
import torch

from paper_2408_11500_amd import binding as B
from test_abi_host import L, declared_symbols  # noqa: F401  (L is a fixture)

ONE = 1 << 20  # an aligned non-NULL address: validation must fail before anything dereferences it


def test_every_declared_symbol_is_exported(L):  # noqa: F811
    names = set(declared_symbols("slicegcn_train.h"))
    assert {"slicegcn_product_fwd", "slicegcn_product_bwd", "slicegcn_gated_fwd", "slicegcn_gated_bwd", "slicegcn_adamw_step"} <= names
    for n in names:
        assert getattr(L, n).argtypes is not None, n


def desc(n=4, w_in=8, w_out=8, type=B.F32, act=B.ACT_NONE, residual=1.0):
    return B._PRODUCT_DESC.pack(n, w_in, w_out, type, act, residual)


FIELDS = {"product": ("X", "W", "b", "R", "P", "Y", "dY", "dX", "dW", "db", "dR"),
          "gated": ("X", "Wg", "Wu", "bg", "bu", "G", "U", "H", "dH", "dX", "dWg", "dWu", "dbg", "dbu")}
MATRICES = {"X", "R", "P", "Y", "dY", "dX", "dR", "G", "U", "H", "dH"}


def io(op, ld=8, **given):
    """Packed io: absent but for what is given, an address or (address, ld)."""
    values = []
    for f in FIELDS[op]:
        v = given.pop(f, 0)
        values += (v if isinstance(v, tuple) else (v, ld if v else 0)) if f in MATRICES else (v,)
    assert not given
    return {"product": B._PRODUCT_IO, "gated": B._GATED_IO}[op].pack(*values)


GOOD = {("product", "fwd"): dict(X=ONE, W=ONE, Y=2 * ONE), ("product", "bwd"): dict(X=ONE, W=ONE, P=ONE, dY=ONE, dX=2 * ONE, dW=3 * ONE, db=4 * ONE),
        ("gated", "fwd"): dict(X=ONE, Wg=ONE, Wu=ONE, H=2 * ONE),
        ("gated", "bwd"): dict(X=ONE, Wg=ONE, Wu=ONE, G=ONE, U=ONE, dH=ONE, dX=2 * ONE, dWg=3 * ONE, dWu=4 * ONE)}


def call(L, op, way, d=None, ws=ONE, ws_bytes=1 << 40, raw=None, **changes):  # noqa: F811
    fields = {**GOOD[op, way], **changes}
    ld = fields.pop("ld", 8)
    return getattr(L, f"slicegcn_{op}_{way}")(desc() if d is None else d, io(op, ld, **fields) if raw is None else raw, ws, ws_bytes, None)


@pytest.mark.parametrize("op,way", GOOD)
def test_refusals_of_sizes_types_and_descriptors(L, op, way):  # noqa: F811
    refused = lambda rc, **kw: call(L, op, way, **kw) == rc
    assert getattr(L, f"slicegcn_{op}_{way}")(None, io(op, **GOOD[op, way]), None, 0, None) == B.EINVAL
    assert getattr(L, f"slicegcn_{op}_{way}")(desc(), None, None, 0, None) == B.EINVAL
    for d in (desc(n=-1), desc(w_in=0), desc(w_out=0), desc(type=3), desc(type=-1), desc(act=4), desc(act=-1), desc(residual=float("nan")),
              desc(residual=float("inf")), desc(residual=1e300)):
        assert refused(B.EINVAL, d=d)
    for d in (desc(n=1 << 31), desc(n=2**31 - 2**16 + 1), desc(w_in=(1 << 20) + 1), desc(w_out=(1 << 20) + 1)):
        assert refused(B.ERANGE, d=d)
    out = {"fwd": "Y" if op == "product" else "H", "bwd": "dX"}[way]
    assert refused(B.EINVAL, ld=7) and refused(B.ERANGE, ld=(1 << 21) + 1)
    assert refused(B.EINVAL, **{out: 2 * ONE + 2}) and refused(B.EINVAL, X=ONE + 1)
    assert refused(B.EINVAL, d=desc(type=B.BF16), X=ONE + 1)


@pytest.mark.parametrize("op,way,name", [(o, w, f) for (o, w), g in GOOD.items() for f in g if f[0] != "d" or f in ("dY", "dH")])
def test_refusals_of_missing_operands(L, op, way, name):  # noqa: F811
    assert call(L, op, way, d=desc(act=B.ACT_GELU), **{name: 0}) == B.EINVAL


def test_refusals_of_combinations(L):  # noqa: F811
    assert call(L, "gated", "fwd", G=ONE) == B.EINVAL and call(L, "gated", "fwd", U=ONE) == B.EINVAL
    assert call(L, "product", "fwd", Y=ONE) == B.EINVAL and call(L, "gated", "fwd", H=ONE) == B.EINVAL  # in the rows of X
    assert call(L, "product", "fwd", b=ONE + 2) == B.EINVAL and call(L, "product", "bwd", db=ONE + 1) == B.EINVAL
    assert call(L, "gated", "bwd", dbu=ONE + 1) == B.EINVAL and call(L, "gated", "bwd", dWg=ONE + 1) == B.EINVAL


OUTPUTS = {("product", "fwd"): ("Y", "P"), ("product", "bwd"): ("dX", "dW", "db", "dR"), ("gated", "fwd"): ("H", "G", "U"),
           ("gated", "bwd"): ("dX", "dWg", "dWu", "dbg", "dbu")}


@pytest.mark.parametrize("op,way", GOOD)
def test_refusals_of_outputs_at_the_address_of_another_operand(L, op, way):  # noqa: F811
    apart = {f: (10 + i) * ONE for i, f in enumerate(FIELDS[op]) if way == "bwd" or f[0] != "d"}
    if way == "bwd":
        apart = {f: a for f, a in apart.items() if f not in ("Y", "H", "R", "b", "bg", "bu")}
    for out in OUTPUTS[op, way]:
        for other, at in apart.items():
            if other != out and (out, other) != ("Y", "R"):
                assert call(L, op, way, d=desc(act=B.ACT_GELU), **{**apart, out: at}) == B.EINVAL, (out, other)
    if (op, way) == ("product", "fwd"):
        assert call(L, op, way, d=desc(n=3, w_in=4096, w_out=512), ws_bytes=0, **{**apart, "ld": 4096, "Y": apart["R"]}) == B.EWORKSPACE  # allowed as such
        assert call(L, op, way, **{**apart, "Y": (apart["R"], 9)}) == B.EINVAL


@pytest.mark.parametrize("op,way", GOOD)
@pytest.mark.parametrize("type", [B.F32, B.BF16, B.F16])
def test_workspaces(L, op, way, type):  # noqa: F811
    size = getattr(L, f"slicegcn_{op}_{way}_workspace_bytes")
    assert size(-1, 8, 8, type) == size(4, 0, 8, type) == size(4, 8, 0, type) == size(4, 8, 8, 3) == size(1 << 31, 8, 8, type) == size(2**31 - 2**16 + 1, 8, 8, type) == 0
    n, w_in, w_out = 3, 4096, 512  # few rows: the sum is cut
    need = size(n, w_in, w_out, type)
    assert need > 0 and need % 256 == 0
    d = desc(n, w_in, w_out, type)
    assert call(L, op, way, d=d, ld=4096, ws=None, ws_bytes=0) == B.EWORKSPACE
    assert call(L, op, way, d=d, ld=4096, ws_bytes=need - 1) == B.EWORKSPACE
    assert call(L, op, way, d=d, ld=4096, ws=ONE + 128) == B.EINVAL
    if way == "fwd":
        assert size(0, w_in, w_out, type) == 0
        assert call(L, op, way, d=desc(0, w_in, w_out, type), ld=4096, ws=None, ws_bytes=0) == 0  # nothing to do
    else:
        rows = n * w_out * (4 if type == B.F32 else 2)
        assert need >= rows * (2 if op == "gated" else 1)


@pytest.mark.parametrize("n", [1, 2, 31, 128, 129, 5000, 16384, 169_343, 2_449_029, 2**31 - 2**16])
@pytest.mark.parametrize("w_in,w_out", [(1, 1), (100, 256), (256, 680), (10240, 4096), (1 << 20, 8)])
def test_sums_of_parts_stay_bounded(L, n, w_in, w_out):  # noqa: F811
    """Parts of long sums: a few hundred MB at most, but for sums of so many rows that their chains would grow too long."""
    for type in (B.F32, B.BF16):
        size = L.slicegcn_product_fwd_workspace_bytes(n, w_in, w_out, type)
        assert size <= max(256 << 20, n * w_out * 4 * -(-w_in // (32 * 1024)))


def adam(**changes):
    t = B._AdamTensor(param=ONE, grad=ONE, m=ONE, v=ONE, scales=ONE, count=10, decay=0.0, param_type=B.F32, grad_type=B.F32)
    for k, v in changes.items():
        setattr(t, k, v)
    return (B._AdamTensor * 1)(t)


@pytest.mark.parametrize("changes", [dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(scales=None), dict(count=-1), dict(count=(1 << 40) + 1),
                                     dict(decay=float("nan")), dict(decay=float("inf")), dict(param_type=3), dict(grad_type=-1), dict(master=ONE),
                                     dict(param=ONE + 2), dict(grad=ONE + 1), dict(scales=ONE + 1), dict(param_type=B.BF16, master=ONE + 2)], ids=str)
def test_refusals_of_adam_tensors(L, changes):  # noqa: F811
    assert L.slicegcn_adamw_step(adam(**changes), 1, 8, 0.1, 0.9, 0.999, 1e-8, 1, None, 0, None) == B.EINVAL


def test_refusals_of_adamw(L):  # noqa: F811
    ok = dict(t=adam(count=0), count=1, states=32, lr=0.1, b1=0.9, b2=0.999, eps=1e-8, step=1)
    run = lambda **kw: L.slicegcn_adamw_step(*{**ok, **kw}.values(), None, 0, None)
    assert run() == 0 and run(t=None, count=0) == 0  # nothing to do
    for kw in (dict(t=None), dict(count=-1), dict(states=16), dict(lr=float("nan")), dict(lr=float("inf")), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=-1.0),
               dict(eps=0.0), dict(eps=-1.0), dict(eps=1e-60), dict(eps=float("nan")), dict(step=0)):
        assert run(**kw) == B.EINVAL, kw
    assert L.slicegcn_adamw_step(adam(m=ONE + 2), 1, 32, 0.1, 0.9, 0.999, 1e-8, 1, None, 0, None) == B.EINVAL


def test_structures_match_the_header(L):  # noqa: F811
    assert B._PRODUCT_DESC.size == 32 and B._PRODUCT_IO.size == 7 * 16 + 4 * 8 and B._GATED_IO.size == 6 * 16 + 8 * 8
    assert ctypes.sizeof(B._AdamTensor) == 64


def test_the_binding_refuses_what_does_not_fit():
    x, w, y = torch.zeros(4, 8), torch.zeros(8, 6), torch.zeros(4, 6)
    with pytest.raises(TypeError):
        B.slicegcn_product_fwd(x, w, y)  # host tensors
    with pytest.raises(ValueError):
        B.slicegcn_product_fwd(torch.zeros(4, 9), w, y)
    with pytest.raises(ValueError):
        B.slicegcn_gated_fwd(x, torch.zeros(8), w, y)
    with pytest.raises(TypeError):
        B.slicegcn_product_fwd_workspace_bytes(4, 8, 6, torch.float64)
    p = [torch.zeros(5)]
    with pytest.raises(ValueError):
        B.AdamList(p, p, p, [])
    with pytest.raises(TypeError):
        B.AdamList(p, p, p, [torch.zeros(5, dtype=torch.float16)])
    with pytest.raises(ValueError):
        B.AdamList(p, p, [torch.zeros(6)], p)
