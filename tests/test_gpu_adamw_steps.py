"""AdamW with its steps counted on the device: updates that are left out do not count."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from paper_2408_11500_amd.stack import AdamW

pytestmark = pytest.mark.gpu


class Model:
    def __init__(self, seed=0):
        gen = torch.Generator().manual_seed(seed)
        self.w, self.g = (torch.randn((50, 33), generator=gen).cuda() for _ in range(2))

    def parameter_slots(self):
        return [(self, "w", self, "g")]


def as_bytes(t):
    return t.contiguous().view(torch.uint8)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("left_out", [(0,), (0, 1, 2), (2,), (1, 3)], ids=str)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_updates_after_one_that_was_left_out(left_out, bad, bits):
    """The weights, states and count of a run without the steps that were left out (the learning rate and the random bits go by the call)."""
    a, b = Model(), Model()
    opt = AdamW([a], lr_max=0.01, max_norm=1.0, state_bits=bits, weight_decay=0.1)
    plain = AdamW([b], lr_max=0.01, max_norm=1.0, state_bits=bits, weight_decay=0.1)
    for t in range(6):
        g = torch.randn(a.g.shape, generator=torch.Generator().manual_seed(100 + t)).cuda()
        a.g.copy_(g)
        if t in left_out:
            a.g[3, 4] = bad
        opt.step(t)
        plain._t += 1
        if t not in left_out:
            B.slicegcn_global_norm(B.TensorList([g]), plain.norm, plain.norm_ws, max_norm=1.0, factor=plain.factor)
            b.g.copy_(g)
            taken = t + 1 - sum(s <= t for s in left_out)
            lr = B.slicegcn_cosine_lr(0.01, 0.0, t, 1)
            B.slicegcn_adamw_step(plain.tensors, lr, taken, factor=plain.factor, seed=plain.seed + plain.t, **plain.hyper)
        assert torch.equal(a.w, b.w), t
        assert torch.equal(as_bytes(opt.m[0]), as_bytes(plain.m[0])) and torch.equal(as_bytes(opt.v[0]), as_bytes(plain.v[0])), t
        assert int(opt.steps) == t + 1 - sum(s <= t for s in left_out)


def test_first_update_after_one_that_was_left_out_has_its_size():
    """The first update of Adam moves every parameter by lr g / (|g| + eps), whatever was left out before it."""
    m = Model()
    m.g.fill_(1e-2)
    before = m.w.clone()
    opt = AdamW([m], lr_max=0.125, lr_min=0.125, max_norm=1.0, weight_decay=0.0)
    m.g[0, 0] = float("inf")
    opt.step(0)
    assert torch.equal(m.w, before)
    m.g[0, 0] = 1e-2
    opt.step(1)
    assert ((before - m.w).double() - 0.125).abs().max() < 0.125 * 1e-5 + 2.0 ** -22  # eps beside g (1e-6) and 16 roundings of the update; one of w, up to 4


@pytest.mark.parametrize("start", [0, 999, 2**31 - 2])
def test_the_count_goes_on_from_where_it_is_set_and_in_a_graph(start):
    p = [torch.ones(1000, device="cuda") for _ in range(2)]
    g = torch.randn(1000, generator=torch.Generator().manual_seed(1)).cuda()
    state = [[torch.zeros(1000, device="cuda") for _ in range(2)] for _ in range(2)]
    lists = [B.AdamList([p[i]], [g], [state[i][0]], [state[i][1]], decays=0.1) for i in range(2)]
    counter, factor = torch.tensor([start, 0, 0, 0], dtype=torch.int32, device="cuda"), torch.ones(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.slicegcn_adamw_step_counted(lists[0], 0.01, counter, factor=factor)
    taken = start
    for f in (1.0, 0.0, 0.5, float("nan"), 1.0, 1.0):
        factor.fill_(f)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        if f > 0:
            taken = min(taken + 1, 2**31 - 1)
            B.slicegcn_adamw_step(lists[1], 0.01, taken, factor=factor)
        assert int(counter[0]) == taken
        assert torch.equal(p[0], p[1]) and torch.equal(state[0][0], state[1][0]) and torch.equal(state[0][1], state[1][1]), f


def test_without_a_factor_every_step_counts():
    p, m, v, g = (torch.zeros(10, device="cuda") for _ in range(4))
    counter = torch.zeros(4, dtype=torch.int32, device="cuda")
    for i in range(3):
        B.slicegcn_adamw_step_counted(B.AdamList([p], [g], [m], [v]), 0.1, counter)
        assert int(counter[0]) == i + 1


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_without_a_bound_on_the_norm_updates_on_gradients_that_are_not_finite_are_left_out_too(bad):
    m, same = Model(), Model()
    opt, plain = AdamW([m], lr_max=0.1, max_norm=float("inf")), AdamW([same], lr_max=0.1)
    before, good = m.w.clone(), m.g.clone()
    m.g[3, 4] = bad
    opt.step(0)
    assert torch.equal(m.w, before) and int(opt.steps) == 0
    m.g.copy_(good)
    opt.step(0)
    plain.step(0)
    assert torch.equal(m.w, same.w) and int(opt.steps) == 1


@pytest.mark.parametrize("max_norm", [None, 1.0])
def test_going_on_with_the_states_of_an_earlier_run(max_norm):
    """With t set to the steps that they have seen, as one run."""
    a, b, grads = Model(), Model(), [torch.randn((50, 33), generator=torch.Generator().manual_seed(t)).cuda() for t in range(6)]
    make = lambda m: AdamW([m], lr_max=0.01, max_norm=max_norm)
    one, first = make(a), make(b)
    for t in range(6):
        a.g.copy_(grads[t])
        one.step(t)
    for t in range(3):
        b.g.copy_(grads[t])
        first.step(t)
    second = make(b)
    for name in ("m", "v"):
        for to, of in zip(getattr(second, name), getattr(first, name)):
            to.copy_(of)
    second.t = first.t
    for t in range(3, 6):
        b.g.copy_(grads[t])
        second.step(t)
    assert torch.equal(a.w, b.w) and second.t == 6
