"""Feed-forward blocks and AdamW as a model uses them: behind the slice stacks of a token model, and by themselves on 16-bit rows."""
import numpy as np
import pytest
import torch

import synth
from gpu_util import assert_close
from paper_2408_11500_amd import binding as B
from paper_2408_11500_amd.stack import AdamW, GraphedStep
from paper_2408_11500_amd.tokens import GatedFeedForward, seeded_trainer
from product_util import gated_fwd
from test_gpu_tokens import small_trainer
from train_util import F64, TYPES

pytestmark = pytest.mark.gpu


def get(o, key):
    return o[key] if isinstance(o, dict) else getattr(o, key)


@pytest.mark.parametrize("blocks", [1, 2])
def test_all_gradients_of_a_small_model(blocks):
    """Embedding, stacks, norms, feed-forward blocks and classifier against torch autograd in 64 bits."""
    g, tr, ids, labels = small_trainer(blocks, feed_forward=34)
    n, gen = ids.numel(), torch.Generator().manual_seed(5)
    for ff in tr.gated:
        ff.set_params(*(torch.randn(t.shape, generator=gen) * 0.3 for t in (ff.Wg, ff.Wu, ff.Wd)))
    for norm in tr.gated_norms:
        norm.params["pre_w"] += (torch.randn(norm.params["pre_w"].shape, generator=gen) * 0.3).cuda()
    tr.forward_backward()

    h = g.to_host()
    A = torch.zeros((n, n), dtype=F64)
    at = np.repeat(np.arange(n), np.diff(h["rowptr"]))
    deg = torch.as_tensor(h["deg"].astype(np.float64))
    A[at, h["colidx"]] = 1 / torch.sqrt(deg[at] * deg[h["colidx"]])
    leaves = {(id(o), key): get(o, key).detach().cpu().to(F64).requires_grad_() for m in tr.models() for o, key, _, _ in m.parameter_slots()}
    P = lambda o, key: leaves[id(o), key]
    norm = lambda v: v / torch.sqrt((v * v).mean(1, True) + 1e-6)
    x = P(tr.emb, "table")[ids] * tr.emb.scale
    u = norm(x) * P(tr.norms[0].params, "pre_w")
    for ff, stack, nb, gated, gn in zip(tr.ffs, tr.stacks, tr.norms[1:], tr.gated, tr.gated_norms):
        fused = torch.relu(u @ P(ff, "W1") + P(ff, "b1")) @ P(ff, "W2") + P(ff, "b2")
        outs = []
        for i in range(stack.k):
            t = fused
            for layer in range(stack.L):
                q = stack.params[i][layer]
                t = torch.relu(A @ t @ P(q, "W_agg") + P(q, "b")) + t @ P(q, "W_self") + P(q, "b_self")
            outs.append(t + P(stack, "E")[i])
        x = x + P(nb.params, "gate") * norm(torch.cat(outs, 1)) * P(nb.params, "post_w")
        u = norm(x) * P(nb.params, "pre_w")
        a = u @ P(gated, "Wg")
        x = x + (a * torch.sigmoid(a) * (u @ P(gated, "Wu"))) @ P(gated, "Wd")
        u = norm(x) * P(gn.params, "pre_w")
    logits = torch.relu(u @ P(tr.cls, "W1") + P(tr.cls, "b1")) @ P(tr.cls, "W2") + P(tr.cls, "b2")
    loss = torch.nn.functional.cross_entropy(logits, labels)
    loss.backward()
    assert abs(float(tr.cls.loss) - loss.item()) < 1e-5
    for m in tr.models():
        for po, pk, go, gk in m.parameter_slots():
            assert_close(get(go, gk).cpu().numpy(), leaves[id(po), pk].grad.numpy(), f"{type(m).__name__}.{gk}")
    g.destroy()


@pytest.mark.parametrize("bits", [8, 32])
def test_training_runs(bits):
    g, tr = seeded_trainer(synth.WORKLOADS["cfg1"], 200, 2, feed_forward=176)
    tr.start(1e-2, 1e-4, 20, weight_decay=0.01, state_bits=bits)
    losses = [tr.epoch(t).item() for t in range(20)]
    assert np.isfinite(losses).all() and len(set(losses)) > 1
    assert all(torch.isfinite(p).all() for p in tr.opt.params)
    g.destroy()


@pytest.mark.parametrize("bits", [8, 32])
def test_training_with_graph_replay_equals_eager(bits):
    w = synth.WORKLOADS["cfg1"]
    (g1, eager), (g2, replay) = seeded_trainer(w, 300, 1, feed_forward=96), seeded_trainer(w, 300, 1, graph_replay=True, feed_forward=96)
    for tr in (eager, replay):
        tr.start(1e-2, 1e-4, 60, max_norm=0.5, state_bits=bits)
    for t in range(5):
        a, b = eager.epoch(t), replay.epoch(t)
        torch.cuda.synchronize()
        assert torch.equal(a, b) and torch.equal(eager.opt.norm, replay.opt.norm), t
        assert all(torch.equal(p, q) for p, q in zip(eager.opt.params, replay.opt.params)), t
    g1.destroy()
    g2.destroy()


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,width,inner", [(1, 64, 176), (24, 128, 344), (300, 72, 200)])
def test_a_block_by_itself(kind, n, width, inner):
    """x + FF(norm x) on rows of each type against 64 bits, eagerly and from a graph: every value within the roundings on its way (H's, of 2^-8 in bf16, each of the inner
    products sees by itself; u's enters both projections)."""
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(4)
    x = torch.randn((n, width), generator=gen).to(dtype).cuda()
    ws = [(torch.randn(s, generator=gen) / s[0] ** 0.5).to(dtype) for s in ((width, inner), (width, inner), (inner, width))]
    ff = GatedFeedForward(n, width, inner, dtype=dtype)
    ff.set_params(*(w.cuda() for w in ws))
    u = torch.empty_like(x)

    def run():
        B.slicegcn_resnorm_fwd(x, None, None, u, pre=B.NORM_RMS)
        return ff.forward(x, u)
    graphed = GraphedStep(run)
    for seed in range(3):
        x.copy_(torch.randn((n, width), generator=torch.Generator().manual_seed(seed)).to(dtype))
        eager = run().clone()
        ff.x.zero_()
        graphed.replay()
        torch.cuda.synchronize()
        assert torch.equal(ff.x, eager)
        x64, (wg, wu, wd) = x.cpu().to(F64), (w.to(F64) for w in ws)
        u64 = u.cpu().to(F64)
        h = gated_fwd(u64, wg, wu, None, None, "silu", dtype)["H"][0]
        want = x64 + h @ wd
        eps = torch.finfo(dtype).eps / 2
        bound = 1.1 * eps * (want.abs() + h.abs() @ wd.abs()) + 1e-5 * (h.abs() @ wd.abs() + 1)
        assert ((eager.cpu().to(F64) - want).abs() <= bound).all()


def test_weights_of_16_bits_keep_their_masters():
    """Updates far below a step of bf16 add up in the masters."""
    class Model:
        def __init__(self):
            self.w, self.g = torch.ones((40, 33), dtype=torch.bfloat16, device="cuda"), torch.ones((40, 33), dtype=torch.bfloat16, device="cuda")

        def parameter_slots(self):
            return [(self, "w", self, "g")]
    m = Model()
    opt = AdamW([m], lr_max=1e-4, lr_min=1e-4, weight_decay=0.0)
    for t in range(100):
        opt.step(t)
    # a constant gradient moves each parameter by lr a step (up to eps and 2^-24 a step)
    assert (opt.masters[0] - 0.99).abs().max() < 1e-5 and torch.equal(m.w, opt.masters[0].to(torch.bfloat16))


def test_norm_that_is_not_finite_leaves_an_update_out():
    class Model:
        def __init__(self):
            self.w, self.g = torch.ones((5, 7), device="cuda"), torch.ones((5, 7), device="cuda")

        def parameter_slots(self):
            return [(self, "w", self, "g")]
    m = Model()
    opt = AdamW([m], lr_max=0.1, max_norm=1.0, state_bits=8)
    m.g[2, 3] = float("inf")
    opt.step(0)
    assert (m.w == 1).all() and (opt.m[0].float() == 0).all()
    m.g[2, 3] = 1.0
    opt.step(0)
    assert (m.w < 1).all()


def test_states_of_other_widths_are_refused():
    with pytest.raises(ValueError):
        AdamW([], lr_max=0.1, state_bits=4)
