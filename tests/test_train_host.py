"""The operators of slicegcn_train.h without a GPU: exported symbols, workspace sizes, and refusals before any device work."""
import ctypes

import pytest
import torch

from paper_2408_11500_amd import binding as B
from test_abi_host import L, declared_symbols  # noqa: F401  (L is a fixture)

ONE = 1 << 20  # an aligned non-NULL address: validation must fail before anything dereferences it


def test_every_declared_symbol_is_exported(L):  # noqa: F811
    names = declared_symbols("slicegcn_train.h")
    assert {"slicegcn_embed_fwd", "slicegcn_embed_sort", "slicegcn_embed_bwd", "slicegcn_resnorm_fwd", "slicegcn_resnorm_bwd",
            "slicegcn_global_norm", "slicegcn_clip", "slicegcn_adam_step_scaled"} <= set(names)
    for n in names:
        assert getattr(L, n).argtypes is not None, n


def embed(n=4, vocab=4, width=4, table=B.F32, rows=B.F32, scale=1.0, pad=0, flags=0):
    return B._EMBED_DESC.pack(n, vocab, pad, scale, width, table, rows, flags)


BAD_EMBED = [(dict(n=-1), B.EINVAL), (dict(vocab=0), B.EINVAL), (dict(n=2**31), B.ERANGE), (dict(vocab=2**31 - 1), B.ERANGE), (dict(flags=8), B.EINVAL)]
BAD_ROWS = [(dict(width=0), B.EINVAL), (dict(table=3), B.EINVAL), (dict(rows=-1), B.EINVAL), (dict(table=B.BF16, rows=B.F16), B.EINVAL),
            (dict(scale=float("inf")), B.EINVAL), (dict(scale=float("nan")), B.EINVAL), (dict(scale=1e39), B.EINVAL), (dict(width=5), B.EINVAL)]


@pytest.mark.parametrize("change,status", BAD_EMBED + BAD_ROWS)
def test_embed_fwd_refuses(L, change, status):  # noqa: F811
    assert L.slicegcn_embed_fwd(embed(**change), ONE, ONE, 4, ONE, 4, None) == status


def test_embed_calls_refuse_bad_pointers(L):  # noqa: F811
    d = embed()
    wide = embed(flags=B.EMBED_IDS64)
    half = embed(table=B.BF16, rows=B.F32)
    for args in ((None, ONE, ONE, 4, ONE, 4), (d, None, ONE, 4, ONE, 4), (d, ONE, None, 4, ONE, 4), (d, ONE, ONE, 4, None, 4), (d, ONE + 2, ONE, 4, ONE, 4),
                 (wide, ONE + 4, ONE, 4, ONE, 4), (d, ONE, ONE + 2, 4, ONE, 4), (half, ONE, ONE + 1, 4, ONE, 4), (d, ONE, ONE, 3, ONE, 4), (d, ONE, ONE, 4, ONE, 3)):
        assert L.slicegcn_embed_fwd(*args, None) == B.EINVAL
    for args in ((None, ONE, ONE, ONE), (d, None, ONE, ONE), (d, ONE, None, ONE), (d, ONE, ONE, None), (d, ONE, ONE + 2, ONE), (d, ONE, ONE, ONE + 1)):
        assert L.slicegcn_embed_sort(*args, None, 0, None) == B.EINVAL
    big = embed(n=5000)
    need = L.slicegcn_embed_sort_workspace_bytes(5000, 4)
    assert need > 0
    assert L.slicegcn_embed_sort(big, ONE, ONE, ONE, None, 0, None) == B.EWORKSPACE
    assert L.slicegcn_embed_sort(big, ONE, ONE, ONE, ONE, need - 1, None) == B.EWORKSPACE
    assert L.slicegcn_embed_sort(big, ONE, ONE, ONE, ONE + 64, need, None) == B.EINVAL
    for args in ((None, ONE, ONE, ONE, 4, ONE, 4), (d, None, ONE, ONE, 4, ONE, 4), (d, ONE, None, ONE, 4, ONE, 4), (d, ONE, ONE, None, 4, ONE, 4),
                 (d, ONE, ONE, ONE, 4, None, 4), (d, ONE, ONE, ONE, 3, ONE, 4), (d, ONE, ONE, ONE, 4, ONE, 3), (d, ONE + 2, ONE, ONE, 4, ONE, 4)):
        assert L.slicegcn_embed_bwd(*args, None, 0, None) == B.EINVAL
    need = L.slicegcn_embed_bwd_workspace_bytes(5000, 4)
    assert L.slicegcn_embed_bwd(big, ONE, ONE, ONE, 4, ONE, 4, ONE, need - 1, None) == B.EWORKSPACE
    for change, status in BAD_EMBED + BAD_ROWS:
        assert L.slicegcn_embed_bwd(embed(**change), ONE, ONE, ONE, 4, ONE, 4, ONE, 1 << 30, None) == status


def test_embed_workspaces(L):  # noqa: F811
    sort, grad = L.slicegcn_embed_sort_workspace_bytes, L.slicegcn_embed_bwd_workspace_bytes
    assert sort(-1, 5) == sort(5, 0) == sort(2**31, 5) == sort(5, 2**31 - 1) == 0
    assert sort(1_000_000, 50_000) >= 16_000_000
    assert grad(-1, 4) == grad(100, 0) == grad(2**31, 4) == grad(0, 4) == grad(1, 4) == 0
    assert grad(100_000, 64) > 0


def resnorm(n=4, width=4, type=B.F32, post=B.NORM_RMS, pre=B.NORM_RMS, flags=0, residual=1.0, eps=1e-6):
    return B._RESNORM_DESC.pack(n, width, type, post, pre, flags, residual, eps)


def io(**kw):
    given = dict(dict(x=ONE, y=ONE, h=ONE, u=ONE, dh=ONE, du=ONE, stats=ONE), **kw)
    rows = lambda *names: [f for n in names for v in [given.get(n)] for f in (v if isinstance(v, tuple) else (v or 0, 4))]
    return B._RESNORM_IO.pack(*rows("x", "y", "gate", "h", "u"), given["stats"] or 0, *rows("dh", "du", "dx", "dy", "dgate"))


def params(**kw):
    return B._RESNORM_PARAMS.pack(*(kw.get(n, 0) for n in ("post_w", "post_b", "pre_w", "pre_b", "gate")))


BAD_RESNORM = [
    (dict(n=-1), {}, {}, B.EINVAL), (dict(width=0), {}, {}, B.EINVAL), (dict(width=16385), {}, {}, B.EUNSUPPORTED), (dict(type=3), {}, {}, B.EINVAL),
    (dict(post=3), {}, {}, B.EINVAL), (dict(pre=-1), {}, {}, B.EINVAL), (dict(flags=2), {}, {}, B.EINVAL), (dict(residual=float("nan")), {}, {}, B.EINVAL),
    (dict(eps=0.0), {}, {}, B.EINVAL), (dict(eps=-1e-6), {}, {}, B.EINVAL), (dict(eps=1e-60), {}, {}, B.EINVAL), (dict(eps=float("nan")), {}, {}, B.EINVAL),
    (dict(flags=1), {}, {}, B.EINVAL),                                   # sigmoid without gate
    ({}, dict(gate=ONE), dict(gate=ONE), B.EINVAL),                      # two gates
    (dict(post=0), dict(post_w=ONE), {}, B.EINVAL), (dict(pre=0), dict(pre_b=ONE), {}, B.EINVAL), ({}, dict(pre_w=ONE + 2), {}, B.EINVAL),
    ({}, {}, dict(x=None, y=None), B.EINVAL), ({}, {}, dict(y=None), B.EINVAL), (dict(post=0), dict(gate=ONE), dict(y=None), B.EINVAL),
    ({}, {}, dict(x=(ONE, 3)), B.EINVAL), ({}, {}, dict(y=ONE + 2), B.EINVAL), (dict(type=B.BF16), {}, dict(x=ONE + 1), B.EINVAL), ({}, {}, dict(stats=ONE + 8), B.EINVAL)]


@pytest.mark.parametrize("desc,p,rows,status", BAD_RESNORM)
def test_resnorm_refuses(L, desc, p, rows, status):  # noqa: F811
    d, q, r = resnorm(**desc), params(**p), io(**rows)
    assert L.slicegcn_resnorm_fwd(d, q, r, None) == status
    assert L.slicegcn_resnorm_bwd(d, q, r, None, None, 0, None) == status


def test_resnorm_directions_refuse(L):  # noqa: F811
    d, none = resnorm(), params()
    fwd = lambda **rows: L.slicegcn_resnorm_fwd(d, none, io(**rows), None)
    assert fwd(h=None, u=None) == fwd(u=None) == fwd(h=(ONE, 2)) == B.EINVAL
    assert L.slicegcn_resnorm_fwd(None, none, io(), None) == L.slicegcn_resnorm_fwd(d, None, io(), None) == B.EINVAL
    assert L.slicegcn_resnorm_fwd(d, none, None, None) == B.EINVAL

    def bwd(grads=None, p=None, ws=None, nbytes=0, **rows):
        return L.slicegcn_resnorm_bwd(d, params(**(p or {})), io(**rows), params(**(grads or {})), ws, nbytes, None)
    assert bwd(dh=None, du=None) == bwd(stats=None) == bwd(dx=ONE, x=None) == bwd(dgate=ONE) == bwd(dy=(ONE, 3)) == B.EINVAL
    assert bwd(grads=dict(pre_w=ONE)) == B.EINVAL                        # gradient of an absent parameter
    assert bwd(grads=dict(pre_w=ONE + 1), p=dict(pre_w=ONE)) == B.EINVAL
    need = L.slicegcn_resnorm_bwd_workspace_bytes(4, 4)
    assert bwd(grads=dict(pre_w=ONE), p=dict(pre_w=ONE)) == bwd(dict(pre_w=ONE), dict(pre_w=ONE), ONE, need - 1) == B.EWORKSPACE
    assert bwd(dict(pre_w=ONE), dict(pre_w=ONE), ONE + 4, need) == B.EINVAL
    ws = L.slicegcn_resnorm_bwd_workspace_bytes
    assert ws(-1, 4) == ws(4, 0) == ws(4, 16385) == 0 and ws(4, 4) > 0


def tensor_list(*entries):
    return (B._Tensor * max(len(entries), 1))(*[B._Tensor(*e) for e in entries])


@pytest.mark.parametrize("entries,count", [([(None, 4, 0, 0)], 1), ([(ONE, -1, 0, 0)], 1), ([(ONE, 4, 5, 0)], 1), ([(ONE + 2, 4, 0, 0)], 1), ([(ONE + 1, 4, 1, 0)], 1),
                                           ([], -1), ([(ONE, 1 << 48, 0, 0)], 1)])
def test_bad_tensors_are_refused(L, entries, count):  # noqa: F811
    a = tensor_list(*entries)
    assert L.slicegcn_global_norm_workspace_bytes(a, count) == 0
    assert L.slicegcn_global_norm(a, count, 0, 1.0, ONE, None, ONE, 1 << 20, None) == B.EINVAL
    assert L.slicegcn_clip(a, None, count, 0, 1.0, ONE, None, ONE, 1 << 20, None) == B.EINVAL
    assert L.slicegcn_clip(tensor_list((ONE, 4, 0, 0)), a, 1 if count == 1 else count, 0, 1.0, ONE, None, ONE, 1 << 20, None) == B.EINVAL


def test_norm_and_clip_refuse(L):  # noqa: F811
    a = tensor_list((ONE, 5_000_000, 0, 0), (None, 0, 1, 0))
    need = L.slicegcn_global_norm_workspace_bytes(a, 2)
    assert need > 0 and L.slicegcn_global_norm_workspace_bytes(tensor_list((ONE, 5000, 0, 0)), 1) == 0  # few elements: one launch, no workspace
    assert L.slicegcn_global_norm(a, 2, 0, 1.0, None, None, ONE, need, None) == B.EINVAL
    assert L.slicegcn_global_norm(a, 2, 2, 1.0, ONE, None, ONE, need, None) == B.EINVAL
    assert L.slicegcn_global_norm(a, 2, 0, -1.0, ONE, ONE, ONE, need, None) == B.EINVAL
    assert L.slicegcn_global_norm(a, 2, 0, float("nan"), ONE, ONE, ONE, need, None) == B.EINVAL
    assert L.slicegcn_global_norm(None, 2, 0, 1.0, ONE, None, ONE, need, None) == B.EINVAL
    assert L.slicegcn_global_norm(a, 2, 0, 1.0, ONE, None, ONE, need - 1, None) == B.EWORKSPACE
    assert L.slicegcn_global_norm(a, 2, 0, 1.0, ONE, None, None, 0, None) == B.EWORKSPACE
    assert L.slicegcn_global_norm(a, 2, 0, 1.0, ONE, None, ONE + 8, need, None) == B.EINVAL
    assert L.slicegcn_clip(a, tensor_list((ONE, 4_999_999, 0, 0), (None, 0, 1, 0)), 2, 0, 1.0, ONE, None, ONE, need, None) == B.EINVAL
    assert L.slicegcn_clip(a, tensor_list((ONE, 5_000_000, 1, 0), (None, 0, 1, 0)), 2, 0, 1.0, ONE, None, ONE, need, None) == B.EINVAL
    assert L.slicegcn_adam_step_scaled(ONE, ONE, None, ONE, ONE, 4, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, None) == B.EINVAL
    assert L.slicegcn_adam_step_scaled(ONE, ONE, ONE, ONE, ONE, 4, 1e-3, 0.9, 0.999, 1e-8, 0.0, 0, None) == B.EINVAL


def test_binding_refuses_what_is_no_device_tensor(L):  # noqa: F811
    t = torch.zeros(4, 4)
    with pytest.raises(TypeError):
        B.slicegcn_embed_fwd(torch.zeros(4, dtype=torch.int16), t, t)
    with pytest.raises(TypeError):
        B.slicegcn_embed_fwd(torch.zeros(4, dtype=torch.int64), t, t)
    with pytest.raises(TypeError):
        B.slicegcn_resnorm_fwd(t, None, t, None)
    with pytest.raises(ValueError):
        B.slicegcn_resnorm_fwd(None, None, t, None)
    with pytest.raises(TypeError):
        B.TensorList([t])


def test_new_tokens_go_into_the_embeddings_own_memory(L, monkeypatch):  # noqa: F811
    """A captured pass reads the tokens through their address, and a caller may use its own tensor again: set_tokens copies, and a refused
    call changes nothing."""
    from paper_2408_11500_amd import tokens
    sorted_ids = []
    monkeypatch.setattr(tokens.B, "slicegcn_embed_sort", lambda ids, *a, **k: sorted_ids.append((ids.data_ptr(), ids.tolist())))
    given = torch.tensor([3, 1, 2, 1])
    emb = tokens.Embedding(given, 5, 8)
    at = emb.ids.data_ptr()
    given.fill_(4)
    assert emb.ids.tolist() == [3, 1, 2, 1] and sorted_ids == [(at, [3, 1, 2, 1])]
    for dtype in (torch.int32, torch.int64):
        emb.set_tokens(torch.tensor([0, 4, -1, 9], dtype=dtype))
        assert emb.ids.data_ptr() == at and emb.ids.tolist() == [0, 4, -1, 9]
        emb.set_tokens(torch.tensor([[5, 0], [2, 0]], dtype=dtype)[:, 0].repeat(2))
        assert emb.ids.data_ptr() == at and emb.ids.tolist() == [5, 2, 5, 2]
    emb.set_tokens(torch.tensor([2**40, -2**40, 2**32 + 1, 0]))
    assert emb.ids.tolist() == [2**40, -2**40, 2**32 + 1, 0]
    calls = len(sorted_ids)
    for bad, error in ((torch.tensor([1, 2, 3]), ValueError), (torch.zeros(5, dtype=torch.int64), ValueError), (torch.zeros(4), TypeError),
                       (torch.zeros(4, dtype=torch.int16), TypeError), (torch.zeros(4, dtype=torch.int64, device="meta"), TypeError)):
        with pytest.raises(error):
            emb.set_tokens(bad)
    assert emb.ids.data_ptr() == at and emb.ids.tolist() == [2**40, -2**40, 2**32 + 1, 0] and len(sorted_ids) == calls
    with pytest.raises(TypeError):
        tokens.Embedding(torch.zeros(4), 5, 8)


@pytest.mark.parametrize("width", [2**31 - 1023, 2**31 - 512, 2**31 - 8, 2**31 - 1])
def test_rows_whose_columns_pass_32_bits_are_refused(L, width):  # noqa: F811
    """Lanes count columns in 32 bits, some of them past the end of a row."""
    d = embed(width=width)
    assert L.slicegcn_embed_bwd(d, ONE, ONE, ONE, width, ONE, width, None, 0, None) == B.ERANGE
    assert L.slicegcn_embed_fwd(d, ONE, ONE, width, ONE, width, None) == B.ERANGE
    assert L.slicegcn_embed_bwd_workspace_bytes(4, width) == 0
    assert L.slicegcn_embed_bwd_workspace_bytes(100_000, width) == 0


def test_a_norm_without_a_block_keeps_no_gradient_of_one(L):  # noqa: F811
    from paper_2408_11500_amd.tokens import BlockNorm
    first = BlockNorm(10, 8, post=B.NORM_NONE, gated=False, device="cpu", block=False)
    assert first.dy is None
    with pytest.raises(ValueError):
        first.forward(torch.zeros(10, 8), torch.zeros(10, 8))
    for kw in (dict(), dict(post=B.NORM_NONE, gated=False)):
        assert BlockNorm(10, 8, device="cpu", **kw).dy.shape == (10, 8)


def test_a_residual_without_norm_and_gate_is_handed_on(L, monkeypatch):  # noqa: F811
    """The next block's residual is x + y, whether or not a norm or a gate shapes y."""
    from paper_2408_11500_amd import tokens
    calls = []
    monkeypatch.setattr(tokens.B, "slicegcn_resnorm_fwd", lambda x, y, h, u, **k: calls.append(h))
    x, y = torch.zeros(10, 8), torch.zeros(10, 8)
    for post in (B.NORM_NONE, B.NORM_RMS):
        for gated in (False, True):
            h, u = tokens.BlockNorm(10, 8, post=post, gated=gated, device="cpu").forward(x, y)
            assert h is not None and h.shape == x.shape and calls[-1] is h, (post, gated)
    h, u = tokens.BlockNorm(10, 8, post=B.NORM_NONE, gated=False, device="cpu", block=False).forward(x, None)
    assert h is None and calls[-1] is None
    h, u = tokens.BlockNorm(10, 8, post=B.NORM_NONE, gated=False, device="cpu").forward(x, None)
    assert h is None and calls[-1] is None
