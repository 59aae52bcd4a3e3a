"""The norm over many tensors, clipping, and the optimiser step that takes the factor along, against 64-bit forms."""
import math

import pytest
import torch

import oracle
from gpu_util import dev
from paper_2408_11500_amd import binding as B
from train_util import F64, TYPES, U, assert_within

pytestmark = pytest.mark.gpu


def make(counts, types, seed=0, std=0.1, offset=0):
    gen = torch.Generator().manual_seed(seed)
    out = []
    for i, c in enumerate(counts):
        buf = (torch.randn(c + offset, generator=gen) * std).to(TYPES[types[i % len(types)]]).cuda()
        out.append(buf[offset:])
    return out


def want_norm(tensors, kind):
    if kind == B.NORM_MAX:
        return max([float(t.to(F64).abs().max()) for t in tensors if t.numel()], default=0.0)
    return math.sqrt(math.fsum(float((t.cpu().to(F64) ** 2).sum()) for t in tensors))


def ws_for(lst):
    return torch.empty(B.slicegcn_global_norm_workspace_bytes(lst), dtype=torch.uint8, device="cuda")


def scalars():
    return torch.full((1,), -1.0, device="cuda"), torch.full((1,), -1.0, device="cuda")


LISTS = [[1], [7], [0], [], [4096], [4097, 1, 0, 8191], [100_003], [5] * 143, [5] * 144, [64] * 145, [0] * 144 + [9], [3] * 300 + [70_001],
         [3_000_017, 12, 900_001]]


@pytest.mark.parametrize("types", [["f32"], ["bf16"], ["f16"], ["bf16", "f32", "f16"]])
@pytest.mark.parametrize("counts", LISTS, ids=lambda c: f"{len(c)}x{max(c, default=0)}")
@pytest.mark.parametrize("kind", [B.NORM_TWO, B.NORM_MAX])
@pytest.mark.parametrize("offset", [0, 1])
def test_norm_and_clip(types, counts, kind, offset):
    tensors = make(counts, types, seed=len(counts), offset=offset)
    lst = B.TensorList(tensors)
    want = want_norm(tensors, kind)
    norm, factor = scalars()
    for max_norm in (0.37, 1e6):
        B.slicegcn_global_norm(lst, norm, ws_for(lst), max_norm=max_norm, factor=factor, kind=kind)
        f = 1.0 if want <= max_norm else max_norm / want
        assert abs(float(norm) - want) <= (1 + 1e-6) * U * want, (float(norm), want)  # fp64 sums, one rounding
        assert abs(float(factor) - f) <= (1 + 1e-6) * U * f
        outs = [torch.full_like(t, 5.0) for t in tensors]
        n2, f2 = scalars()
        B.slicegcn_clip(lst, B.TensorList(outs), max_norm, n2, ws_for(lst), factor=f2, kind=kind)
        assert torch.equal(n2, norm) and torch.equal(f2, factor)
        for t, o in zip(tensors, outs):
            w = t.cpu().to(F64) * f
            assert_within(o, w, 3 * U * w.abs(), "clipped")  # the factor and the product
    copies = [t.clone() for t in tensors]
    B.slicegcn_clip(B.TensorList(copies), None, 0.37, None, ws_for(lst), kind=kind)  # in place, norm not wanted
    B.slicegcn_clip(lst, B.TensorList(outs), 0.37, n2, ws_for(lst), kind=kind)
    for c, o in zip(copies, outs):
        assert torch.equal(c, o)


@pytest.mark.parametrize("kind", [B.NORM_TWO, B.NORM_MAX])
def test_nothing_is_written_outside_or_where_nothing_is_clipped(kind):
    buf = torch.full((10_000,), 0.001, device="cuda")
    B.slicegcn_clip(B.TensorList([buf[3:9001]]), None, 1e-9, None, ws_for(B.TensorList([buf[3:9001]])), kind=kind)
    assert (buf[:3] == 0.001).all() and (buf[9001:] == 0.001).all() and not (buf[3:9001] == 0.001).any()
    t = torch.randn(5000, device="cuda")
    was = t.clone()
    B.slicegcn_clip(B.TensorList([t]), None, 1e9, None, ws_for(B.TensorList([t])), kind=kind)
    assert torch.equal(t, was)


@pytest.mark.parametrize("kind", [B.NORM_TWO, B.NORM_MAX])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("where", [0, 4099, 99_999])
def test_values_that_are_not_finite(kind, value, where):
    t = torch.randn(100_000, device="cuda")
    t[where] = value
    lst = B.TensorList([torch.randn(33, device="cuda"), t])
    norm, factor = scalars()
    B.slicegcn_global_norm(lst, norm, ws_for(lst), max_norm=1.0, factor=factor, kind=kind)
    if math.isnan(value):
        assert norm.isnan().all() and factor.isnan().all()
    else:
        assert norm.isinf().all() and (norm > 0).all() and (factor == 0).all()


def test_large_and_small_values_neither_overflow_nor_vanish():
    for scale in (1e30, 1e-30):
        t = torch.full((5000,), scale, device="cuda")
        norm, factor = scalars()
        lst = B.TensorList([t])
        B.slicegcn_global_norm(lst, norm, ws_for(lst), max_norm=1.0, factor=factor)
        want = math.sqrt(5000) * float(torch.tensor(scale))
        assert abs(float(norm) - want) <= 2 * U * want
    zero = B.TensorList([torch.zeros(100, device="cuda")])
    B.slicegcn_global_norm(zero, norm, ws_for(zero), max_norm=0.0, factor=factor)
    assert float(norm) == 0.0 and float(factor) == 1.0


def test_two_calls_give_the_same_bits_on_any_stream_and_in_graphs():
    tensors = make([900_001, 5, 77_777], ["f32", "bf16"])
    lst, outs = B.TensorList(tensors), [torch.empty_like(t) for t in tensors]
    to, ws = B.TensorList(outs), None
    ws = ws_for(lst)
    norm, factor = scalars()
    B.slicegcn_clip(lst, to, 1.0, norm, ws, factor=factor)
    first = [o.clone() for o in outs] + [norm.clone(), factor.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.slicegcn_clip(lst, to, 1.0, norm, ws, factor=factor)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, outs + [norm, factor]):
        assert torch.equal(a, b)
    from paper_2408_11500_amd.stack import GraphedStep
    graph = GraphedStep(lambda: B.slicegcn_clip(lst, to, 1.0, norm, ws, factor=factor))
    for i in range(4):
        tensors[0].normal_()
        B.slicegcn_clip(lst, to, 1.0, norm, ws, factor=factor)
        torch.cuda.synchronize()
        want = [o.clone() for o in outs] + [norm.clone(), factor.clone()]
        for t in outs + [norm, factor]:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, outs + [norm, factor]):
            assert torch.equal(a, b), i


@pytest.mark.parametrize("wd", [0.0, 0.01])
def test_scaled_adam_step(wd):
    gen = torch.Generator().manual_seed(3)
    count, factor = 10_007, torch.tensor([0.25], device="cuda")
    p = torch.randn(count, generator=gen)
    g = torch.randn(count, generator=gen)
    a = [p.cuda(), torch.zeros(count, device="cuda"), torch.zeros(count, device="cuda")]
    b = [t.clone() for t in a]
    for step in (1, 2, 3):
        B.slicegcn_adam_step_scaled(a[0], g.cuda(), factor, a[1], a[2], 1e-2, step, weight_decay=wd)
        B.slicegcn_adam_step(b[0], (0.25 * g).cuda(), b[1], b[2], 1e-2, step, weight_decay=wd)  # a power of two: the same product
    for s, t in zip(a, b):
        assert torch.equal(s, t)


def mixed(tiles, gen, empty=True):
    """Tensors of all types, sizes on, just below and just above whole tiles of 16 KB, empty ones among them; `tiles` of them in all, about."""
    types, out, k = ["f32", "bf16", "f16"], [], 0
    while tiles > 0:
        kind = types[k % 3]
        size = {"f32": 4096, "bf16": 8192, "f16": 8192}[kind]
        share = min(tiles, 1 + k * 37 % 211)
        out.append((torch.randn(share * size + (0, -1, 1, 7)[k % 4], generator=gen, device="cuda") * 0.1).to(TYPES[kind]))
        if empty and k % 5 == 2:
            out.append(torch.empty(0, dtype=TYPES[kind], device="cuda"))
        tiles -= share
        k += 1
    return out


@pytest.mark.parametrize("tiles", [2049, 2500, 5120, 9001])
@pytest.mark.parametrize("kind", [B.NORM_TWO, B.NORM_MAX])
def test_workgroups_that_take_tiles_in_turn(tiles, kind):
    """More tiles than a launch has workgroups: each goes over tensors of several types, forwards for the norm and back for the scaling."""
    gen = torch.Generator(device="cuda").manual_seed(tiles)
    tensors = mixed(tiles, gen)
    assert len(tensors) <= 144  # one launch
    lst = B.TensorList(tensors)
    if kind == B.NORM_TWO:
        want = math.sqrt(math.fsum(float((t.to(F64) ** 2).sum()) for t in tensors))
    else:
        want = max(float(t.to(F64).abs().max()) for t in tensors if t.numel())
    f = min(1.0, 0.37 / want)
    outs, copies = [torch.full_like(t, 5.0) for t in tensors], [t.clone() for t in tensors]
    norm, factor = scalars()
    B.slicegcn_clip(lst, B.TensorList(outs), 0.37, norm, ws_for(lst), factor=factor, kind=kind)
    assert abs(float(norm) - want) <= (1 + 1e-6) * U * want
    assert abs(float(factor) - f) <= (1 + 1e-6) * U * f
    n2, f2 = scalars()
    B.slicegcn_global_norm(lst, n2, ws_for(lst), max_norm=0.37, factor=f2, kind=kind)
    assert torch.equal(n2, norm) and torch.equal(f2, factor)
    B.slicegcn_clip(B.TensorList(copies), None, 0.37, None, ws_for(lst), kind=kind)
    for i, (t, o, c) in enumerate(zip(tensors, outs, copies)):
        assert torch.equal(o, (factor * t.float()).to(t.dtype)), i  # one fp32 product, rounded once
        assert torch.equal(c, o), i


def test_one_large_value_is_found_in_every_tile():
    """The largest absolute value in turn in the first and the last element of tensors that lie in any workgroup's share."""
    tensors = mixed(3000, torch.Generator(device="cuda").manual_seed(5))
    lst = B.TensorList(tensors)
    norm, _ = scalars()
    ws = ws_for(lst)
    for t in tensors:
        for place in (0, t.numel() // 2, t.numel() - 1) if t.numel() else ():
            was = t[place].clone()
            t[place] = -100.0
            B.slicegcn_global_norm(lst, norm, ws, kind=B.NORM_MAX)
            assert float(norm) == 100.0
            t[place] = was


@pytest.mark.parametrize("launches", [1, 2])
def test_lists_beyond_the_caches(launches):
    """256 MB and more: stored past the caches, in one launch and in two."""
    gen = torch.Generator(device="cuda").manual_seed(launches)
    if launches == 1:
        tensors = mixed(12_000, gen) + [torch.randn(20_000_003, generator=gen, device="cuda")]
        assert len(tensors) <= 144
    else:
        tensors = [(torch.randn(420_001 + 64 * i, generator=gen, device="cuda") * 0.1).to(TYPES[("f32", "bf16", "f16")[i % 3]]) for i in range(250)]
    assert sum(t.numel() * t.element_size() for t in tensors) > 256 << 20
    lst = B.TensorList(tensors)
    want = math.sqrt(math.fsum(float((t.to(F64) ** 2).sum()) for t in tensors))
    outs = [torch.full_like(t, 5.0) for t in tensors]
    norm, factor = scalars()
    B.slicegcn_clip(lst, B.TensorList(outs), 1.0, norm, ws_for(lst), factor=factor)
    assert abs(float(norm) - want) <= (1 + 1e-6) * U * want
    assert abs(float(factor) - 1 / want) <= (1 + 1e-6) * U / want
    scaled = [(factor * t.float()).to(t.dtype) for t in tensors]
    B.slicegcn_clip(lst, None, 1.0, None, ws_for(lst))
    for i, (w, o, t) in enumerate(zip(scaled, outs, tensors)):
        assert torch.equal(o, w) and torch.equal(t, w), i
