"""Token embeddings: lookup, sort and gradient against plain 64-bit forms, at sizes, types, strides and tokens where they can go wrong."""
import numpy as np
import pytest
import torch

from paper_2408_11500_amd import binding as B
from train_util import F64, TYPES, U, assert_within, embed_fwd, embed_grad, rows

pytestmark = pytest.mark.gpu

PAIRS = [("f32", "f32"), ("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f32", "f16")]
CHUNK = 64  # positions of a token that one lane group adds


def tokens(gen, n, vocab, kind):
    if kind == "even":
        return torch.randint(0, vocab, (n,), generator=gen)
    if kind == "hot":  # half of all positions hold one token
        ids = torch.randint(0, vocab, (n,), generator=gen)
        return torch.where(torch.rand(n, generator=gen) < 0.5, torch.tensor(vocab // 2), ids)
    if kind == "one":
        return torch.full((n,), vocab - 1)
    if kind == "skewed":
        return ((float(vocab) ** torch.rand(n, generator=gen, dtype=F64)).long() - 1).clamp_(0, vocab - 1)
    if kind == "bad":  # some outside the table, far and near
        ids = torch.randint(0, vocab, (n,), generator=gen)
        ids[::5] = -1
        ids[1::7] = vocab
        return ids
    raise ValueError(kind)


def sort(ids, vocab, pad=None):
    n = ids.numel()
    order = torch.full((n,), -7, dtype=torch.int32, device="cuda")
    starts = torch.full((vocab + 1,), -7, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.slicegcn_embed_sort_workspace_bytes(n, vocab), dtype=torch.uint8, device="cuda")
    B.slicegcn_embed_sort(ids, vocab, order, starts, ws, pad=pad)
    return order, starts


def grad_ws(n, width):
    return torch.empty(B.slicegcn_embed_bwd_workspace_bytes(n, width), dtype=torch.uint8, device="cuda")


# ---- lookup ---------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("table,out", PAIRS)
@pytest.mark.parametrize("n,vocab,width,ldt,ldo,offset", [
    (1, 1, 1, 1, 1, 0), (3, 7, 3, 3, 5, 1), (70, 10, 4, 4, 4, 0), (65, 9, 7, 9, 7, 3), (33, 50, 8, 8, 8, 0), (1000, 31, 64, 64, 64, 0),
    (517, 100, 100, 100, 128, 0), (129, 12, 257, 259, 261, 1), (40, 1000, 602, 602, 602, 0), (9, 5, 2049, 2051, 2049, 1), (5, 3, 8192, 8192, 8200, 0)])
def test_lookup(table, out, n, vocab, width, ldt, ldo, offset):
    gen = torch.Generator().manual_seed(n * 31 + width)
    tab, tab64 = rows(gen, vocab, width, TYPES[table], ldt, offset)
    ids = torch.randint(0, vocab, (n,), generator=gen)
    o, _ = rows(gen, n, width, TYPES[out], ldo, offset)
    B.slicegcn_embed_fwd(ids.cuda(), tab, o, scale=width ** 0.5)
    want = embed_fwd(ids, tab64, width ** 0.5, None)
    assert_within(o, want, 2 * U * want.abs(), "rows")  # the factor and the product are rounded to fp32


def test_lookup_leaves_the_padding_of_rows():
    buf = torch.full((50, 40), 7.0, device="cuda")
    B.slicegcn_embed_fwd(torch.arange(50, device="cuda"), torch.randn(50, 37, device="cuda"), buf[:, :37])
    assert (buf[:, 37:] == 7.0).all() and not (buf[:, :37] == 7.0).any()


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("pad", [None, 2, -1, -100])
def test_lookup_padding_and_tokens_outside(dtype, pad):
    vocab, width = 6, 20
    ids = torch.tensor([0, 2, 5, -1, 6, -100, 2, 1, 2**31 - 1] + ([2**40, -2**40, 2**32] if dtype == torch.int64 else []))
    tab, tab64 = rows(torch.Generator().manual_seed(1), vocab, width, torch.float32)
    out = torch.full((ids.numel(), width), 3.0, device="cuda")
    B.slicegcn_embed_fwd(ids.to(dtype).cuda(), tab, out, scale=1.0, pad=pad)
    want = embed_fwd(ids, tab64, 1.0, pad)
    assert torch.equal(out.cpu().isnan(), want.isnan())
    assert torch.equal(out.cpu().to(F64).nan_to_num(9.0), want.nan_to_num(9.0))


def test_lookup_carries_infinities_of_rows_that_are_looked_up_only():
    tab = torch.randn(4, 9, device="cuda")
    tab[1] = float("inf")
    tab[3] = float("nan")
    out = torch.empty(3, 9, device="cuda")
    B.slicegcn_embed_fwd(torch.tensor([0, 3, 2], device="cuda"), tab, out, pad=3)
    assert torch.equal(out, torch.stack([tab[0], torch.zeros(9, device="cuda"), tab[2]]))
    B.slicegcn_embed_fwd(torch.tensor([0, 1, 2], device="cuda"), tab, out)
    assert out[1].isinf().all() and out[0].isfinite().all() and out[2].isfinite().all()


def test_lookup_beyond_32_bit_offsets():
    """Rows whose elements lie past 2^31 in the table and in the output."""
    ld, vocab, width = 40_000, 60_000, 48
    tab = torch.empty((vocab, ld), dtype=torch.bfloat16, device="cuda")
    tab[:, :width] = torch.arange(vocab, device="cuda")[:, None] % 251
    out = torch.empty((vocab, ld), dtype=torch.bfloat16, device="cuda")
    ids = torch.arange(vocab - 1, -1, -1, device="cuda")
    B.slicegcn_embed_fwd(ids, tab[:, :width], out[:, :width])
    assert torch.equal(out[:, :width], tab[ids, :width])


# ---- sort -----------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("n", [0, 1, 2, 63, 64, 65, 1000, 4095, 4096, 4097, 8191, 20_011, 300_007])
@pytest.mark.parametrize("vocab", [1, 2, 3, 1000, 1023, 1024, 5000, 1_500_000])
def test_sort(n, vocab):
    gen = torch.Generator().manual_seed(n + vocab)
    for kind, dtype, pad in (("even", torch.int64, None), ("skewed", torch.int32, 0), ("bad", torch.int64, vocab // 2), ("one", torch.int32, None)):
        ids = tokens(gen, n, vocab, kind)
        order, starts = sort(ids.to(dtype).cuda(), vocab, pad)
        key = torch.where((ids < 0) | (ids >= vocab) | (ids == (-10**9 if pad is None else pad)), vocab, ids)
        want = torch.sort(key, stable=True)
        valid = int((key < vocab).sum())
        assert torch.equal(starts.cpu().long(), torch.searchsorted(want.values, torch.arange(vocab + 1))), (kind, "starts")
        assert int(starts[-1]) == valid
        assert torch.equal(order.cpu().long()[:valid], want.indices[:valid]), (kind, "order")


@pytest.mark.parametrize("n", [65_536, 65_537, 98_305, 196_608, 196_609, 524_288, 524_289, 1_100_003])
@pytest.mark.parametrize("vocab", [7, 40_000, 2_000_000])
def test_sort_of_many_tokens(n, vocab):
    """Both sides of every number of tokens at which the sort takes other tiles or another way to their prefix sums."""
    gen = torch.Generator().manual_seed(n + vocab)
    for kind, dtype, pad in (("skewed", torch.int64, None), ("hot", torch.int32, vocab // 2)):
        ids = tokens(gen, n, vocab, kind)
        order, starts = sort(ids.to(dtype).cuda(), vocab, pad)
        key = ids if pad is None else torch.where(ids == pad, vocab, ids)
        want = torch.sort(key, stable=True)
        valid = int((key < vocab).sum())
        assert torch.equal(starts.cpu().long(), torch.searchsorted(want.values, torch.arange(vocab + 1))), (kind, "starts")
        assert torch.equal(order.cpu().long()[:valid], want.indices[:valid]), (kind, "order")


# ---- gradient -------------------------------------------------------------------------------------------------------------

def check_grad(gen, ids, vocab, width, table, row, ldo, ldt, offset, scale, pad, accumulate, dtype=torch.int64):
    n = ids.numel()
    dout, dout64 = rows(gen, n, width, TYPES[row], ldo, offset, 0.5)
    dtab, old64 = rows(gen, vocab, width, TYPES[table], ldt, offset)
    order, starts = sort(ids.to(dtype).cuda(), vocab, pad)
    B.slicegcn_embed_bwd(order, starts, dout, dtab, grad_ws(n, width), scale=scale, accumulate=accumulate)
    want, size = embed_grad(ids, dout64, vocab, scale, pad)
    if accumulate:
        want, size = want + old64, size + old64.abs()
    # at most CHUNK additions in a row, 6 over lanes, the factor and its product, the old value
    assert_within(dtab, want, (CHUNK + 12) * U * size, "gradient")
    if not accumulate:
        empty = torch.ones(vocab, dtype=torch.bool)
        empty[ids[(ids >= 0) & (ids < vocab)]] = False
        assert (dtab.cpu()[empty] == 0).all()
    return order, starts, dout, dtab


@pytest.mark.parametrize("table,row", PAIRS)
@pytest.mark.parametrize("n,vocab,width,ldo,ldt,offset", [
    (1, 1, 1, 1, 1, 0), (1, 4, 5, 5, 5, 0), (64, 1, 3, 4, 5, 1), (65, 1, 8, 8, 8, 0), (200, 3, 7, 7, 7, 1), (1000, 40, 64, 64, 64, 0),
    (700, 5, 100, 128, 100, 0), (333, 2000, 257, 259, 263, 1), (5000, 7, 602, 602, 602, 0), (300, 2, 2050, 2050, 2051, 1)])
def test_gradient(table, row, n, vocab, width, ldo, ldt, offset):
    gen = torch.Generator().manual_seed(n + 7 * width)
    for kind, accumulate, pad in (("even", False, None), ("hot", True, None), ("bad", False, 0)):
        check_grad(gen, tokens(gen, n, vocab, kind), vocab, width, table, row, ldo, ldt, offset, 1.5, pad, accumulate)


@pytest.mark.parametrize("kind", ["one", "hot", "skewed", "even"])
@pytest.mark.parametrize("n,vocab,width", [(20_000, 1000, 40), (100_000, 77, 16), (30_000, 60_000, 130)])
def test_gradient_of_many_positions(kind, n, vocab, width):
    gen = torch.Generator().manual_seed(n)
    check_grad(gen, tokens(gen, n, vocab, kind), vocab, width, "f32", "f32", width, width, 0, 1.0, None, False, torch.int32)
    check_grad(gen, tokens(gen, n, vocab, kind), vocab, width, "bf16", "bf16", width, width, 0, 1.0, 0, True)


@pytest.mark.parametrize("run", [1, 63, 64, 65, 127, 128, 129, 191, 192, 193])
def test_gradient_of_runs_that_meet_chunk_boundaries(run):
    """Tokens with `run` positions each, whose places in the order start at every remainder of the chunk length sooner or later."""
    gen = torch.Generator().manual_seed(run)
    vocab = 2 * CHUNK + 3
    ids = torch.arange(vocab).repeat_interleave(run)[torch.randperm(vocab * run, generator=gen)]
    check_grad(gen, ids, vocab, 12, "f32", "f32", 12, 12, 0, 1.0, None, False)


def test_gradient_without_tokens_is_zero_or_untouched():
    for n, ids in ((0, torch.zeros(0, dtype=torch.int64)), (5, torch.full((5,), 3))):
        order, starts = sort(ids.cuda(), 4, pad=3)
        d = torch.full((4, 10), 2.0, device="cuda")
        B.slicegcn_embed_bwd(order, starts, torch.randn(n, 10, device="cuda"), d, None, accumulate=True)
        assert (d == 2.0).all()
        B.slicegcn_embed_bwd(order, starts, torch.randn(n, 10, device="cuda"), d, None)
        assert (d == 0.0).all()


def test_gradient_keeps_non_finite_rows_to_their_tokens():
    ids = torch.tensor([0, 1, 2, 1, 3] * 40)
    dout = torch.randn(200, 6, device="cuda")
    dout[ids.cuda() == 1] = float("nan")
    dout[ids.cuda() == 3] = float("inf")
    order, starts = sort(ids.cuda(), 4, pad=1)
    d = torch.empty(4, 6, device="cuda")
    B.slicegcn_embed_bwd(order, starts, dout, d, grad_ws(200, 6))
    assert (d[1] == 0).all() and d[3].isinf().all() and d[0].isfinite().all() and d[2].isfinite().all()


def test_gradient_leaves_the_padding_of_rows():
    buf = torch.full((3, 40), 7.0, device="cuda")
    ids = torch.randint(0, 3, (500,), device="cuda")
    order, starts = sort(ids, 3)
    B.slicegcn_embed_bwd(order, starts, torch.randn(500, 37, device="cuda"), buf[:, :37], grad_ws(500, 37))
    assert (buf[:, 37:] == 7.0).all() and not (buf[:, :37] == 7.0).any()


def test_gradient_beyond_32_bit_offsets():
    ld, n, width = 40_000, 60_000, 24
    dout = torch.empty((n, ld), dtype=torch.bfloat16, device="cuda")
    dout[:, :width] = torch.randint(-4, 5, (n, width), device="cuda").to(torch.bfloat16)
    ids = torch.randint(0, 50, (n,), device="cuda")
    order, starts = sort(ids, 50)
    d = torch.empty((50, width), device="cuda")
    B.slicegcn_embed_bwd(order, starts, dout[:, :width], d, grad_ws(n, width))
    want, _ = embed_grad(ids.cpu(), dout[:, :width].cpu().to(F64), 50, 1.0, None)
    assert torch.equal(d.cpu().to(F64), want)  # whole numbers below 2^24


def test_gradient_against_differences():
    """<gradient, direction> is the slope of <lookup, dout> along the direction (a linear map: up to rounding exactly)."""
    gen = torch.Generator().manual_seed(5)
    n, vocab, width, scale = 3000, 90, 33, 2.0
    ids = tokens(gen, n, vocab, "skewed")
    _, _, dout, dtab = check_grad(gen, ids, vocab, width, "f32", "f32", width, width, 0, scale, 4, False)
    way = torch.randn((vocab, width), generator=gen)
    up, down = (torch.empty((n, width), device="cuda") for _ in range(2))
    base = torch.randn((vocab, width), generator=gen)
    B.slicegcn_embed_fwd(ids.cuda(), (base + way).cuda(), up, scale=scale, pad=4)
    B.slicegcn_embed_fwd(ids.cuda(), (base - way).cuda(), down, scale=scale, pad=4)
    slope = float(((up - down).cpu().to(F64) / 2 * dout.cpu().to(F64)).sum())
    got = float((dtab.cpu().to(F64) * way.to(F64)).sum())
    size = float((up.cpu().to(F64).abs() + down.cpu().to(F64).abs()).mul(dout.cpu().to(F64).abs()).sum())
    assert abs(slope - got) <= (CHUNK + 20) * U * size


def test_two_calls_give_the_same_bits_and_other_streams_wait_for_nothing():
    gen = torch.Generator().manual_seed(8)
    ids = tokens(gen, 50_000, 300, "skewed").cuda()
    dout = torch.randn(50_000, 65, device="cuda")
    order, starts = sort(ids, 300)
    a, b = (torch.empty(300, 65, device="cuda") for _ in range(2))
    B.slicegcn_embed_bwd(order, starts, dout, a, grad_ws(50_000, 65))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        order2, starts2 = sort(ids, 300)
        B.slicegcn_embed_bwd(order2, starts2, dout, b, grad_ws(50_000, 65))
    side.synchronize()
    assert torch.equal(order, order2) and torch.equal(starts, starts2) and torch.equal(a, b)


def test_graph_replays_equal_the_eager_calls():
    n, vocab, width = 30_000, 500, 72
    ids, dout = torch.randint(0, vocab, (n,), device="cuda"), torch.randn(n, width, device="cuda")
    order, starts = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(vocab + 1, dtype=torch.int32, device="cuda")
    ws_sort = torch.empty(B.slicegcn_embed_sort_workspace_bytes(n, vocab), dtype=torch.uint8, device="cuda")
    ws, table = grad_ws(n, width), torch.randn(vocab, width, device="cuda")
    out, d = torch.empty(n, width, device="cuda"), torch.empty(vocab, width, device="cuda")

    def step():
        B.slicegcn_embed_fwd(ids, table, out, scale=3.0, pad=1)
        B.slicegcn_embed_sort(ids, vocab, order, starts, ws_sort, pad=1)
        B.slicegcn_embed_bwd(order, starts, dout, d, ws)
    from paper_2408_11500_amd.stack import GraphedStep
    graph = GraphedStep(step)
    for i in range(4):
        ids.copy_(torch.randint(0, vocab, (n,), device="cuda"))
        dout.normal_()
        step()
        torch.cuda.synchronize()
        want = out.clone(), order.clone(), starts.clone(), d.clone()
        for t in (out, order, starts, d):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip((out, order, starts, d), want):
            valid = int(want[2][-1]) if got is order else None
            assert torch.equal(got[:valid], w[:valid]), i


def test_orders_that_do_not_belong_touch_nothing_outside():
    """Entries outside [0, n), and starts that are no ascending positions, are skipped or clamped."""
    n, vocab, width = 200, 3, 16
    order = torch.arange(n, dtype=torch.int32, device="cuda")
    order[::2] = -5
    order[1::4] = 2**31 - 1
    starts = torch.tensor([0, 50, 120, 200], dtype=torch.int32, device="cuda")
    dout = torch.ones(n, width, device="cuda")
    d = torch.empty(vocab, width, device="cuda")
    B.slicegcn_embed_bwd(order, starts, dout, d, grad_ws(n, width))
    kept = ((order >= 0) & (order < n)).cpu()
    assert d[:, 0].cpu().tolist() == [int(kept[a:b].sum()) for a, b in ((0, 50), (50, 120), (120, 200))]


@pytest.mark.parametrize("n", [1, 5, 8, 9, 64, 200, 3000])
@pytest.mark.parametrize("kind", ["drop", "descend", "far", "end early"])
def test_starts_that_do_not_ascend_touch_nothing_outside(n, kind):
    """Also without a workspace, where few positions need none."""
    vocab, width = 4, 16
    starts = {"drop": [0, n, n // 2, n, n // 2], "descend": [n, n - 1, n // 2, 1, 0], "far": [-2**31, 2**31 - 1, -5, n + 7, 2**31 - 1],
              "end early": [0, 0, n + 1, 2**31 - 1, (n + 1) // 2]}[kind]
    order = torch.arange(n, dtype=torch.int32, device="cuda")
    need = B.slicegcn_embed_bwd_workspace_bytes(n, width)
    assert (need == 0) == (n <= 8)
    guarded = torch.full((vocab + 8, width), 7.0, device="cuda")
    ws = torch.full((need + 512,), 7, dtype=torch.uint8, device="cuda")
    B.slicegcn_embed_bwd(order, torch.tensor(starts, dtype=torch.int32, device="cuda"), torch.ones(n, width, device="cuda"), guarded[4:4 + vocab],
                         ws[:need] if need else None)
    torch.cuda.synchronize()
    assert (guarded[:4] == 7.0).all() and (guarded[4 + vocab:] == 7.0).all() and (ws[need:] == 7).all()


@pytest.mark.parametrize("table,row", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("kind", ["skewed", "hot"])
def test_gradient_beyond_the_caches(kind, table, row):
    """A table of 256 MB and more in whole lines: rows without tokens, with few and with many positions, stored past the caches."""
    vocab, width, n = (560_000, 128, 150_001) if table == "f32" else (560_000, 256, 150_001)
    gen = torch.Generator().manual_seed(n)
    ids = tokens(gen, n, vocab, kind)
    ids[: 50_000 : 2] = 77  # cut by every chunk
    ids = ids[torch.randperm(n, generator=gen)].cuda()
    order, starts = sort(ids, vocab, pad=3)
    dout = torch.randint(-2, 3, (n, width), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(TYPES[row])
    d = torch.full((vocab, width), 5.0, dtype=TYPES[table], device="cuda")
    assert d.numel() * d.element_size() >= 256 << 20 and d.data_ptr() % 128 == 0 and width * d.element_size() % 128 == 0
    B.slicegcn_embed_bwd(order, starts, dout, d, grad_ws(n, width))
    want = torch.zeros((vocab, width), dtype=F64, device="cuda")
    want.index_add_(0, ids, dout.to(F64))
    want[3] = 0
    # whole numbers below 2^24: sums are exact, and rounded once
    assert want.abs().max() < 2**24 and torch.equal(d, want.to(torch.float32).to(TYPES[table]))


def test_gradient_with_rows_not_in_whole_lines_beyond_the_caches():
    vocab, width, n = 700_000, 100, 20_000
    ids = torch.randint(0, vocab, (n,), device="cuda")
    order, starts = sort(ids, vocab)
    dout = torch.randint(-2, 3, (n, width), device="cuda").float()
    d = torch.full((vocab, width), 5.0, device="cuda")
    B.slicegcn_embed_bwd(order, starts, dout, d, grad_ws(n, width))
    want = torch.zeros((vocab, width), device="cuda")
    want.index_add_(0, ids, dout)
    assert torch.equal(d, want)


@pytest.mark.parametrize("n,vocab,width,table,out", [(1_050_003, 900, 260, "f32", "f32"), (540_001, 3000, 520, "bf16", "bf16"), (8_500_000, 50, 16, "f32", "f32")])
def test_lookups_of_more_rows_than_one_turn_of_the_workgroups(n, vocab, width, table, out):
    """More than 65 536 workgroups' rows, results of 256 MB and more, and tokens and rows in the last turn."""
    tab = torch.randn(vocab, width, device="cuda").to(TYPES[table])
    ids = torch.randint(0, vocab, (n,), device="cuda")
    ids[-1], ids[-2] = vocab - 1, -1
    o = torch.full((n, width), 5.0, dtype=TYPES[out], device="cuda")
    B.slicegcn_embed_fwd(ids, tab, o, scale=2.0, pad=-1)
    step = 1 << 20
    for r in range(0, n, step):
        i = ids[r:r + step]
        want = tab[i.clamp_min(0)] * 2
        want[i < 0] = 0
        assert torch.equal(o[r:r + step], want), r


def test_starts_of_more_rows_than_one_turn_of_the_workgroups():
    """A vocabulary of more than 65 536 workgroups' entries, behind a sort in tiles."""
    vocab, n = 17_000_000, 40_003
    gen = torch.Generator().manual_seed(4)
    ids = torch.randint(0, vocab, (n,), generator=gen)
    ids[:3] = torch.tensor([vocab - 1, 0, 65_536 * 256])
    order, starts = sort(ids.cuda(), vocab)
    want = torch.sort(ids, stable=True)
    assert torch.equal(starts.cpu().long(), torch.searchsorted(want.values, torch.arange(vocab + 1)))
    assert torch.equal(order.cpu().long(), want.indices)
