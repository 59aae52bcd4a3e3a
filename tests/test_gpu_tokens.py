"""The operators of slicegcn_train.h together: a model that looks its inputs up, passes blocks with norms and gated residuals, and is
updated with clipped gradients.  All gradients of a small model against torch autograd in 64 bits, training runs, graph replay."""
import numpy as np
import pytest
import torch

import paper_2408_11500_amd as sg
import synth
from gpu_util import assert_close, dev, messy_edges
from paper_2408_11500_amd import binding as B
from paper_2408_11500_amd.stack import Optimizer
from paper_2408_11500_amd.tokens import TokenTrainer, seeded_trainer
from train_util import Resnorm, embed_grad

pytestmark = pytest.mark.gpu
F64 = torch.float64


def small_trainer(blocks, pad=None, n=300, vocab=40, k=2, hs=12, layers=2, classes=5, **kw):
    rng = np.random.default_rng(3)
    src, dst = messy_edges(n, 900, rng)
    g = sg.slicegcn_build_norm_csr(dev(src, torch.int64), dev(dst, torch.int64), n)
    gen = torch.Generator().manual_seed(1)
    ids = torch.randint(0, vocab, (n,), generator=gen)
    labels = torch.randint(0, classes, (n,), generator=gen)
    tr = TokenTrainer(g, ids.cuda(), vocab, labels.cuda(), k, hs, layers, 16, classes, blocks=blocks, pad=pad, **kw)
    normal = lambda *shape: (torch.randn(shape, generator=gen) * 0.3).cuda()
    tr.emb.table.copy_(normal(vocab, k * hs))
    for ff, stack in zip(tr.ffs, tr.stacks):
        ff.set_params(normal(k * hs, k * hs), normal(k * hs), normal(k * hs, hs), normal(hs))
        for i in range(k):
            for layer, (wi, wo) in enumerate(stack.widths):
                stack.set_params(i, layer, normal(wi, wo), normal(wo), normal(wi, wo), normal(wo))
        stack.E.copy_(normal(k, hs))
    for norm in tr.norms:
        for p in norm.params.values():
            p += normal(k * hs)
    tr.cls.set_params(normal(k * hs, 16), normal(16), normal(16, classes), normal(classes))
    return g, tr, ids, labels


def plain_loss(tr, A, ids, labels, pad):
    """Loss of the model in 64 bits, and its parameters as leaves in the order of the trainer's slots."""
    get = lambda o, key: o[key] if isinstance(o, dict) else getattr(o, key)
    leaves = {(id(o), key): get(o, key).detach().cpu().to(F64).requires_grad_() for m in tr.models() for o, key, _, _ in m.parameter_slots()}
    P = lambda o, key: leaves[id(o), key]
    x = P(tr.emb, "table")[ids] * tr.emb.scale
    if pad is not None:
        x = x * (ids != pad).to(F64)[:, None]

    def norm(v):
        return v / torch.sqrt((v * v).mean(1, True) + 1e-6)
    u = norm(x) * P(tr.norms[0].params, "pre_w")
    for ff, stack, nb in zip(tr.ffs, tr.stacks, tr.norms[1:]):
        fused = torch.relu(u @ P(ff, "W1") + P(ff, "b1")) @ P(ff, "W2") + P(ff, "b2")
        outs = []
        for i in range(stack.k):
            h = fused
            for layer in range(stack.L):
                q = stack.params[i][layer]
                h = torch.relu(A @ h @ P(q, "W_agg") + P(q, "b")) + h @ P(q, "W_self") + P(q, "b_self")
            outs.append(h + P(stack, "E")[i])
        x = x + P(nb.params, "gate") * norm(torch.cat(outs, 1)) * P(nb.params, "post_w")
        u = norm(x) * P(nb.params, "pre_w")
    logits = torch.relu(u @ P(tr.cls, "W1") + P(tr.cls, "b1")) @ P(tr.cls, "W2") + P(tr.cls, "b2")
    return torch.nn.functional.cross_entropy(logits, labels), leaves


@pytest.mark.parametrize("blocks,pad", [(1, None), (2, 3)])
def test_all_gradients_of_a_small_model(blocks, pad):
    g, tr, ids, labels = small_trainer(blocks, pad)
    h = g.to_host()
    A = torch.zeros((h["n"], h["n"]), dtype=F64)
    rows = np.repeat(np.arange(h["n"]), np.diff(h["rowptr"]))
    deg = torch.as_tensor(h["deg"].astype(np.float64))
    A[rows, h["colidx"]] = (1 / torch.sqrt(deg[rows] * deg[h["colidx"]]))
    tr.forward_backward()
    loss, leaves = plain_loss(tr, A, ids, labels, pad)
    loss.backward()
    assert abs(float(tr.cls.loss) - loss.item()) < 1e-5
    get = lambda o, key: o[key] if isinstance(o, dict) else getattr(o, key)
    for m in tr.models():
        for po, pk, go, gk in m.parameter_slots():
            assert_close(get(go, gk).cpu().numpy(), leaves[id(po), pk].grad.numpy(), f"{type(m).__name__}.{gk}")
    g.destroy()


@pytest.mark.parametrize("blocks", [1, 2])
def test_training_reduces_the_loss(blocks):
    g, tr = seeded_trainer(synth.WORKLOADS["cfg1"], 200, blocks)
    tr.start(1e-2, 1e-4, 60)
    losses, norms = [], []
    for t in range(60):
        losses.append(tr.epoch(t).item())
        norms.append(tr.opt.norm.item())
        want = float((tr.opt.G.to(F64) ** 2).sum().sqrt())
        assert abs(norms[-1] - want) <= 1e-6 * want
    assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0], losses[::10]
    g.destroy()


def test_training_with_graph_replay_equals_eager():
    w = synth.WORKLOADS["cfg1"]
    (g1, eager), (g2, replay) = seeded_trainer(w, 300, 2), seeded_trainer(w, 300, 2, graph_replay=True)
    for tr in (eager, replay):
        tr.start(1e-2, 1e-4, 60, max_norm=0.5)
    for t in range(6):
        a, b = eager.epoch(t), replay.epoch(t)
        torch.cuda.synchronize()
        assert torch.equal(a, b) and torch.equal(eager.opt.P, replay.opt.P) and torch.equal(eager.opt.norm, replay.opt.norm), t
    g1.destroy()
    g2.destroy()


class _Slots:
    def __init__(self, *params):
        self.p, self.g = dict(enumerate(params)), {i: torch.zeros_like(p) for i, p in enumerate(params)}

    def parameter_slots(self):
        return [(self.p, i, self.g, i) for i in self.p]


@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_clipped_updates_are_updates_on_clipped_gradients(max_norm):
    gen = torch.Generator().manual_seed(2)
    start = [torch.randn(s, generator=gen).cuda() for s in ((30, 7), (7,), (100,))]
    a, b = _Slots(*[p.clone() for p in start]), _Slots(*[p.clone() for p in start])
    clipped, plain = Optimizer([a], lr_max=1e-2, max_norm=max_norm), Optimizer([b], lr_max=1e-2)
    for step in range(3):
        for i in a.g:
            v = torch.randn(a.g[i].shape, generator=gen).cuda()
            a.g[i].copy_(v)
            b.g[i].copy_(v)
        lst = B.TensorList([plain.G])
        ws = torch.empty(B.slicegcn_global_norm_workspace_bytes(lst), dtype=torch.uint8, device="cuda")
        B.slicegcn_clip(lst, None, max_norm, None, ws)
        clipped.step(step)
        plain.step(step)
        assert torch.equal(clipped.P, plain.P) and torch.equal(clipped.V, plain.V)


def test_new_tokens_take_effect():
    g, tr, ids, labels = small_trainer(1)
    tr.emb.forward()
    new = (ids + 1) % 40
    tr.emb.set_tokens(new.cuda())
    X = tr.emb.forward().cpu()
    assert torch.allclose(X, tr.emb.table.cpu()[new] * tr.emb.scale, rtol=1e-6, atol=0.0)
    dX = torch.randn(X.shape, device="cuda")
    tr.emb.backward(dX)
    want, _ = embed_grad(new, dX.cpu().to(F64), 40, tr.emb.scale, None)
    assert_close(tr.emb.dtable.cpu().numpy(), want.numpy(), "table", tol=1e-6)
    g.destroy()


@pytest.mark.parametrize("dtype", [torch.int64, torch.int32])
def test_new_tokens_reach_a_replayed_graph(dtype):
    """set_tokens between replayed epochs, from a tensor that is overwritten afterwards: the same bits as eager epochs on those tokens."""
    w, vocab = synth.WORKLOADS["cfg1"], 300
    (g1, eager), (g2, replay) = seeded_trainer(w, vocab, 2), seeded_trainer(w, vocab, 2, graph_replay=True)
    for tr in (eager, replay):
        tr.start(1e-2, 1e-4, 60, max_norm=0.5)
    for t in range(5):
        if t:
            ids = torch.randint(0, vocab, (w.n_nodes,), generator=torch.Generator().manual_seed(t)).to(dtype).cuda()
            eager.emb.set_tokens(ids.clone())
            replay.emb.set_tokens(ids)
            ids.fill_(-5)
        a, b = eager.epoch(t), replay.epoch(t)
        torch.cuda.synchronize()
        assert a.isfinite().all() and torch.equal(a, b), t
        assert torch.equal(eager.emb.X, replay.emb.X) and torch.equal(eager.emb.dtable, replay.emb.dtable) and torch.equal(eager.opt.P, replay.opt.P), t
    g1.destroy()
    g2.destroy()


def test_a_plain_residual_between_blocks():
    """Neither norm nor gate after the block: h = x + y, and its gradient reaches both."""
    from paper_2408_11500_amd.tokens import BlockNorm
    n, width = 50, 24
    norm = BlockNorm(n, width, post=B.NORM_NONE, gated=False)
    x, y, dh, du = (torch.randn(n, width, device="cuda") for _ in range(4))
    h, u = norm.forward(x, y)
    assert torch.equal(h, x + y)
    dx, dy = norm.backward(x, y, dh, du)
    want = Resnorm(x.cpu().to(F64), y.cpu().to(F64), pre=B.NORM_RMS)
    g, size = want.backward(dh.cpu().to(F64), du.cpu().to(F64))
    assert_close(u.cpu().numpy(), want.u.numpy(), "u", tol=1e-5)
    for got, name in ((dx, "dx"), (dy, "dy")):
        assert_close(got.cpu().numpy(), g[name].numpy(), name, tol=1e-5)
