"""Training on graphs whose nodes carry tokens (categories, item ids) instead of feature vectors: a learned embedding feeds slice
stacks put one after another, with a norm before and after each, a gated residual round it, and clipped updates.

    x_0 = scale * table[token];  u_0 = pre(x_0)
    y_b = stack_b(MLP_FF_b(u_b));  x_{b+1} = x_b + gate_b * post_b(y_b);  u_{b+1} = pre_{b+1}(x_{b+1})
    loss = cross-entropy(MLP_CLS(u_blocks))

and with a feed-forward block behind each stack, x_{b+1} += (silu(u_{b+1} Wg) * (u_{b+1} Wu)) Wd before the next block, normed again.

This module orders library calls and owns buffers; every arithmetic step of an epoch is a kernel of the library.  Run
``python -m paper_2408_11500_amd.tokens --workload cfg1 --epochs 60`` for a seeded synthetic run (a node's label is a function of its
token, so that there is something to learn).
"""
from __future__ import annotations

import argparse
import math
import os
import sys
import time

import torch

from . import binding as B
from .stack import AdamW, Classifier, FeatureFusion, GraphedStep, Optimizer, SliceStack


class Embedding:
    """Rows of a learned table, looked up by the nodes' tokens.  The tokens stay the same in every epoch, so they are sorted once;
    call ``set_tokens`` for new ones.  The embedding keeps its own copy of them, in memory that stays where it is: a captured pass
    finds new tokens there, as it finds their order."""

    def __init__(self, ids: torch.Tensor, vocab: int, width: int, scale: float | None = None, pad: int | None = None):
        self.vocab, self.pad = vocab, pad
        self.scale = math.sqrt(width) if scale is None else scale
        f32 = dict(dtype=torch.float32, device=ids.device)
        n = ids.numel()
        self.table, self.dtable = (torch.zeros((vocab, width), **f32) for _ in range(2))
        self.X = torch.empty((n, width), **f32)
        self.ids = torch.empty(n, dtype=torch.int64, device=ids.device)  # 64 bits hold any token of either type
        self.order = torch.empty(n, dtype=torch.int32, device=ids.device)
        self.starts = torch.empty(vocab + 1, dtype=torch.int32, device=ids.device)
        self.ws = torch.empty(max(B.slicegcn_embed_sort_workspace_bytes(n, vocab), B.slicegcn_embed_bwd_workspace_bytes(n, width)),
                              dtype=torch.uint8, device=ids.device)
        self.set_tokens(ids)

    def set_tokens(self, ids: torch.Tensor):
        """As many tokens as before, int32 or int64."""
        if ids.dtype not in (torch.int32, torch.int64) or ids.device != self.ids.device:
            raise TypeError(f"ids: expected int32 or int64 on {self.ids.device}, not {ids.dtype} on {ids.device}")
        if ids.numel() != self.ids.numel():
            raise ValueError(f"expected {self.ids.numel()} tokens, not {ids.numel()}")
        self.ids.copy_(ids.reshape(-1))
        B.slicegcn_embed_sort(self.ids, self.vocab, self.order, self.starts, self.ws, pad=self.pad)

    def forward(self) -> torch.Tensor:
        return B.slicegcn_embed_fwd(self.ids, self.table, self.X, scale=self.scale, pad=self.pad)

    def backward(self, dX: torch.Tensor):
        B.slicegcn_embed_bwd(self.order, self.starts, dX, self.dtable, self.ws, scale=self.scale)

    def parameter_slots(self):
        return [(self, "table", self, "dtable")]


class BlockNorm:
    """What lies between two blocks: the norm after one, its gate (a learned value per column) and residual, the norm before the
    next.  ``block`` = False with ``post`` = NORM_NONE and no gate: the norm before the first block, which takes no block output."""

    def __init__(self, n: int, width: int, post: int = B.NORM_RMS, pre: int = B.NORM_RMS, gated: bool = True, device="cuda",
                 block: bool = True):
        f32 = dict(dtype=torch.float32, device=device)
        self.post, self.pre = post, pre
        names = (["post_w"] if post != B.NORM_NONE else []) + (["pre_w"] if pre != B.NORM_NONE else []) + (["gate"] if gated else [])
        self.params = {name: torch.ones(width, **f32) for name in names}
        self.grads = {"d" + name: torch.zeros(width, **f32) for name in names}
        self.u, self.dx = (torch.empty((n, width), **f32) for _ in range(2))
        self.h, self.dy = (torch.empty((n, width), **f32) if block else None for _ in range(2))
        self.stats = torch.empty((n, 4), **f32)
        self.ws = torch.empty(B.slicegcn_resnorm_bwd_workspace_bytes(n, width), dtype=torch.uint8, device=device)

    def forward(self, x: torch.Tensor, y: torch.Tensor | None):
        if y is not None and self.dy is None:
            raise ValueError("a norm before the first block takes no block output")
        h = self.h if y is not None else None  # without a block h is x itself
        B.slicegcn_resnorm_fwd(x, y, h, self.u, post=self.post, pre=self.pre, stats=self.stats, **self.params)
        return h, self.u

    def backward(self, x: torch.Tensor, y: torch.Tensor | None, dh: torch.Tensor | None, du: torch.Tensor):
        B.slicegcn_resnorm_bwd(x, y, self.stats, dh, du, self.dx, self.dy if y is not None else None, self.ws, post=self.post,
                               pre=self.pre, **self.params, **self.grads)
        return self.dx, self.dy

    def parameter_slots(self):
        return [(self.params, name, self.grads, "d" + name) for name in self.params]


class GatedFeedForward:
    """x' = x + (act(u Wg) * (u Wu)) Wd on rows of fp32, bf16 or fp16: gated projections to ``inner`` columns and the way back with the
    residual in its epilogue.  ``u``: x behind the norm before the block.  ``two_terms``: gradients before the activation are kept in two terms of a
    16-bit type.  Without ``training`` nothing is kept for a backward pass and there are no gradients."""

    def __init__(self, n: int, width: int, inner: int, act: int = B.ACT_SILU, dtype: torch.dtype = torch.float32, device="cuda",
                 two_terms: bool = False, training: bool = True):
        self.act, self.two_terms, self.training = act, two_terms, training
        like = dict(dtype=dtype, device=device)
        self.Wg, self.Wu = (torch.zeros((width, inner), **like) for _ in range(2))
        self.Wd = torch.zeros((inner, width), **like)
        self.H, self.x = torch.empty((n, inner), **like), torch.empty((n, width), **like)
        self.G = self.U = None
        sizes = [B.slicegcn_gated_fwd_workspace_bytes(n, width, inner, dtype), B.slicegcn_product_fwd_workspace_bytes(n, inner, width, dtype)]
        if training:
            self.dWg, self.dWu, self.dWd = (torch.zeros_like(w) for w in (self.Wg, self.Wu, self.Wd))
            self.G, self.U, self.dH = (torch.empty((n, inner), **like) for _ in range(3))
            self.du = torch.empty((n, width), **like)
            sizes += [B.slicegcn_gated_bwd_workspace_bytes(n, width, inner, dtype, two_terms), B.slicegcn_product_bwd_workspace_bytes(n, inner, width, dtype)]
        self.ws = torch.empty(max(sizes), dtype=torch.uint8, device=device)

    def set_params(self, Wg, Wu, Wd):
        for dst, src in ((self.Wg, Wg), (self.Wu, Wu), (self.Wd, Wd)):
            dst.copy_(src)

    def forward(self, x: torch.Tensor, u: torch.Tensor) -> torch.Tensor:
        B.slicegcn_gated_fwd(u, self.Wg, self.Wu, self.H, self.ws, G=self.G, U=self.U, act=self.act)
        return B.slicegcn_product_fwd(self.H, self.Wd, self.x, self.ws, R=x)

    def backward(self, u: torch.Tensor, dx: torch.Tensor) -> torch.Tensor:
        """Gradient of u from that of x'; the gradient of x is that of x' (and what reaches it through u)."""
        if not self.training:
            raise RuntimeError("a feed-forward block without training keeps nothing for a backward pass")
        B.slicegcn_product_bwd(self.H, self.Wd, None, dx, self.ws, dX=self.dH, dW=self.dWd)
        B.slicegcn_gated_bwd(u, self.Wg, self.Wu, self.G, self.U, self.dH, self.ws, dX=self.du, dWg=self.dWg, dWu=self.dWu, act=self.act,
                             two_terms=self.two_terms)
        return self.du

    def parameter_slots(self):
        return [(self, w, self, "d" + w) for w in ("Wg", "Wu", "Wd")] if self.training else []


class TokenTrainer:
    def __init__(self, graph: B.Graph, ids: torch.Tensor, vocab: int, labels: torch.Tensor, k: int, slice_hidden: int, layers: int,
                 hidden: int, classes: int, blocks: int = 1, pad: int | None = None, graph_replay: bool = False,
                 feed_forward: int = 0):
        """``blocks`` slice stacks of k slice models with ``layers`` layers each.  ``feed_forward``: columns inside the gated feed-forward
        block behind each stack (0: none).  ``graph_replay``: forward, loss and backward of an
        epoch are captured into a HIP graph at the first epoch and replayed afterwards."""
        n, width = ids.numel(), k * slice_hidden
        dev = ids.device
        self.labels = labels.to(torch.int32)
        self.emb = Embedding(ids, vocab, width, pad=pad)
        self.norms = [BlockNorm(n, width, post=B.NORM_NONE, gated=False, device=dev, block=False)]
        self.norms += [BlockNorm(n, width, device=dev) for _ in range(blocks)]
        self.ffs = [FeatureFusion(n, width, slice_hidden, device=dev) for _ in range(blocks)]
        self.stacks = [SliceStack(graph, n, k, slice_hidden, slice_hidden, layers, device=dev, shared_input=ff.Xff) for ff in self.ffs]
        self.gated = [GatedFeedForward(n, width, feed_forward, device=dev) for _ in range(blocks if feed_forward else 0)]
        self.gated_norms = [BlockNorm(n, width, post=B.NORM_NONE, gated=False, device=dev, block=False) for _ in self.gated]
        self.cls = Classifier(n, width, hidden, classes, device=dev)
        self.du = torch.empty((n, width), dtype=torch.float32, device=dev)
        self.opt = None
        self.graph_replay, self._graph = graph_replay, None

    def models(self):
        return [self.emb, *self.norms, *self.ffs, *self.stacks, *self.gated, *self.gated_norms, self.cls]

    def start(self, lr_max: float, lr_min: float, epochs: int, weight_decay: float = 0.0, max_norm: float | None = 1.0,
              state_bits: int | None = None):
        """Call once after the parameters of all models are set.  ``state_bits`` (8 or 32): AdamW with such states instead of Adam."""
        args = dict(lr_max=lr_max, lr_min=lr_min, t_max=epochs, weight_decay=weight_decay, max_norm=max_norm)
        self.opt = Optimizer(self.models(), **args) if state_bits is None else AdamW(self.models(), state_bits=state_bits, **args)

    def forward_backward(self):
        """Forward, loss and backward of one epoch (no update)."""
        xs = [self.emb.forward()]
        _, u = self.norms[0].forward(xs[0], None)
        us, ys = [u], []
        inner = []  # what enters the feed-forward blocks
        for b, (ff, stack, norm) in enumerate(zip(self.ffs, self.stacks, self.norms[1:])):
            ff.forward(us[-1])
            ys.append(stack.forward())
            x, u = norm.forward(xs[-1], ys[-1])
            if self.gated:
                inner.append(u)
                x = self.gated[b].forward(x, u)
                _, u = self.gated_norms[b].forward(x, None)
            xs.append(x)
            us.append(u)
        self.cls.forward_backward(us[-1], self.labels, self.du)
        dx = None
        for b in reversed(range(len(self.stacks))):
            du = self.du
            if self.gated:
                dx, _ = self.gated_norms[b].backward(xs[b + 1], None, dx, du)
                du = self.gated[b].backward(inner[b], dx)
            dx, dy = self.norms[b + 1].backward(xs[b], ys[b], dx, du)
            self.stacks[b].backward(dy)
            self.ffs[b].backward(us[b], self.stacks[b].dXin[:, :self.ffs[b].s], self.du)
        dx, _ = self.norms[0].backward(xs[0], None, dx, self.du)
        self.emb.backward(dx)

    def epoch(self, t: int) -> torch.Tensor:
        """One epoch: forward, loss, backward, clipped update.  Returns the loss (device scalar, before the update)."""
        if self.graph_replay:
            if self._graph is None:
                self._graph = GraphedStep(self.forward_backward)
            self._graph.replay()
        else:
            self.forward_backward()
        self.opt.step(t)
        return self.cls.loss


def seeded_trainer(w, vocab: int, blocks: int = 1, graph_replay: bool = False, device="cuda:0", feed_forward: int = 0):
    """(graph, trainer) for a workload of ``synth.configs`` with seeded tokens, labels and parameters."""
    from synth import configs, model, rng
    src, dst = configs.edges(w, device=device)
    g = B.slicegcn_build_norm_csr(src, dst, w.n_nodes)
    u = rng.uniform(w.seed, STREAM_TOKENS, rng.arange64(w.n_nodes, device))
    ids = (float(vocab) ** u).long().clamp_(1, vocab) - 1  # a token's frequency falls with its rank
    tr = TokenTrainer(g, ids, vocab, ids % w.classes, w.k, w.slice_hidden, w.layers, w.hidden, w.classes, blocks=blocks,
                      graph_replay=graph_replay, feed_forward=feed_forward)
    width = w.k * w.slice_hidden
    tr.emb.table.copy_(configs.normal_matrix(w.seed, STREAM_TABLE, vocab, width, device=device, std=1 / tr.emb.scale))
    for b, (ff, stack) in enumerate(zip(tr.ffs, tr.stacks)):
        tag = 1000 * (b + 1)
        ff.set_params(configs.glorot(w.seed, tag, width, width, device), torch.zeros(width, device=device),
                      configs.glorot(w.seed, tag + 1, width, ff.s, device), torch.zeros(ff.s, device=device))
        for i in range(w.k):
            for layer, (wi, wo) in enumerate(stack.widths):
                stack.set_params(i, layer, *model.slice_layer_params(w, i, layer, wi, wo, device=device))
    for b, ff in enumerate(tr.gated):
        tag = TAG_GATED + 10 * b
        ff.set_params(*(configs.glorot(w.seed, tag + i, *shape, device) for i, shape in enumerate(2 * [(width, feed_forward)] + [(feed_forward, width)])))
    tr.cls.set_params(*model.classifier_params(w, width, device=device))
    return g, tr


STREAM_TOKENS, STREAM_TABLE = 20, 21  # of the seeded generator
TAG_GATED = (1 << 20) + 1000  # behind those of the classifier


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--workload", default="cfg1")
    ap.add_argument("--vocab", type=int, default=500)
    ap.add_argument("--blocks", type=int, default=1, help="slice stacks one after another")
    ap.add_argument("--epochs", type=int, default=60)
    ap.add_argument("--lr", type=float, default=1e-2)
    ap.add_argument("--max-norm", type=float, default=1.0, help="gradients are clipped to this norm")
    ap.add_argument("--feed-forward", type=int, default=0, help="columns inside a gated feed-forward block behind each stack (0: none)")
    ap.add_argument("--state-bits", type=int, choices=(8, 32), default=None, help="AdamW with states of so many bits instead of Adam")
    ap.add_argument("--weight-decay", type=float, default=0.0)
    ap.add_argument("--graph", action="store_true", help="replay forward + loss + backward as one HIP graph")
    args = ap.parse_args(argv)
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    import synth
    g, tr = seeded_trainer(synth.WORKLOADS[args.workload], args.vocab, args.blocks, args.graph, feed_forward=args.feed_forward)
    tr.start(args.lr, args.lr * 1e-2, args.epochs, weight_decay=args.weight_decay, max_norm=args.max_norm, state_bits=args.state_bits)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for t in range(args.epochs):
        loss = tr.epoch(t)
        if t % max(1, args.epochs // 10) == 0 or t == args.epochs - 1:
            print(f"epoch {t:4d}  loss {loss.item():.4f}  gradient norm {tr.opt.norm.item():.4f}", flush=True)
    torch.cuda.synchronize()
    print(f"{args.epochs / (time.perf_counter() - t0):.2f} epochs/s")
    g.destroy()


if __name__ == "__main__":
    main()
