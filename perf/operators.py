"""Operators for models that learn their inputs and are built from blocks, as cases that can be timed: token embeddings with
their gradient, norms around a block with its gate and residual, and the global gradient norm with clipping.

``run`` computes an operator in its plain form, from elementary torch operations, or with this package's kernels (``own``).
Sizes are those of the benchmark workloads of ``synth.configs`` (cfg1 to cfg5) or generic ones; ``draw`` spreads over the ranges
between them.  A case names its operator and its sizes:

  embed        rows of a table looked up by token and scaled
  embed_grad   the table's gradient: tokens sorted, the rows of equal tokens added
  resnorm      p = post-norm(y);  h = residual * x + gate * p;  u = pre-norm(h)
  resnorm_grad its backward pass, from dh and du, with the gradients of the norms' weights and of the gate
  clip         the norm over all gradients of a model, and the gradients scaled to at most a given norm
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5


def listed():
    return [
        # Every node of a small graph (cfg1) looks up its token: latency is all there is.
        dict(name="embed_small", op="embed", n=2048, vocab=1000, width=64, table="f32", rows="f32", ids="i32", ld=64, pad=-1),
        # The items of a co-purchase graph (cfg4): 100-wide rows padded to whole cache lines from a table kept in 16 bits.
        dict(name="embed_items", op="embed", n=2_449_029, vocab=500_000, width=100, table="bf16", rows="f32", ids="i64", ld=128,
             pad=-1),
        # The gradient of the first case: a few rows, many of them of the same tokens.
        dict(name="embed_grad_small", op="embed_grad", n=2048, vocab=1000, width=64, table="f32", rows="f32", ids="i32", ld=64,
             pad=-1),
        # A citation graph (cfg2) whose nodes carry one token each, some padded; the ordinary training step.
        dict(name="embed_grad_citation", op="embed_grad", n=169_343, vocab=50_000, width=128, table="f32", rows="f32", ids="i64",
             ld=128, pad=0),
        # A wide table in 16 bits trained on long batches of text: most of its rows get no gradient.
        dict(name="embed_grad_wide", op="embed_grad", n=65_536, vocab=128_000, width=2048, table="bf16", rows="bf16", ids="i64",
             ld=2048, pad=-1),
        # One new row passes between two blocks, as when a model answers one request.
        dict(name="resnorm_single", op="resnorm", n=1, width=1024, type="bf16", post="rms", pre="rms", gate="column", sigmoid=False,
             residual=1.0, ld=1024),
        # Between two slice stacks over a citation graph (cfg2, hidden 256).
        dict(name="resnorm_citation", op="resnorm", n=169_343, width=256, type="f32", post="rms", pre="rms", gate="column",
             sigmoid=False, residual=1.0, ld=256),
        # Backward between two stacks of a small graph (cfg1).
        dict(name="resnorm_grad_small", op="resnorm_grad", n=2048, width=64, type="f32", post="layer", pre="layer", gate="column",
             sigmoid=False, residual=1.0, ld=64),
        # A social graph's 602 features (cfg3): rows that fill no tile, a gate of the same size through a sigmoid.
        dict(name="resnorm_grad_social", op="resnorm_grad", n=232_965, width=602, type="f32", post="layer", pre="layer",
             gate="matrix", sigmoid=True, residual=0.5, ld=602),
        # A wide model in 16 bits.
        dict(name="resnorm_grad_wide", op="resnorm_grad", n=16_384, width=4096, type="bf16", post="rms", pre="rms", gate="column",
             sigmoid=False, residual=1.0, ld=4096),
        # The gradients of a small model (cfg1): two slice models of two layers, encoding and classifier.
        dict(name="clip_small", op="clip", model="slices", k=2, layers=2, width=64, hidden=64, classes=8, type="f32", kind="two",
             max_norm=1.0),
        # The gradients of a large model: 48 blocks of matrices in 16 bits, with norms and biases in 32.
        dict(name="clip_large", op="clip", model="blocks", layers=48, width=1000, type="bf16", kind="two", max_norm=1.0),
    ]


# ---- drawn cases ------------------------------------------------------------------------------------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_ld(rng, width):
    kind = rng.choice(["dense", "dense", "lines", "odd"])
    return width if kind == "dense" else (width + 31) // 32 * 32 if kind == "lines" else width + rng.randrange(1, 8)


def _draw(rng):
    op = rng.choice(["embed", "embed_grad", "resnorm", "resnorm_grad", "clip"])
    if op in ("embed", "embed_grad"):
        table, rows = rng.choice([("f32", "f32"), ("bf16", "f32"), ("f16", "f32"), ("bf16", "bf16"), ("f16", "f16")])
        width = _log(rng, 8, 4096)
        return dict(op=op, n=_log(rng, 1, 2_500_000), vocab=_log(rng, 2, 1_000_000), width=width, table=table, rows=rows,
                    ids=rng.choice(["i32", "i64"]), ld=_draw_ld(rng, width), pad=rng.choice([-1, -1, 0, 1]))
    if op in ("resnorm", "resnorm_grad"):
        width = _log(rng, 16, 8192)
        gate = rng.choice(["none", "column", "matrix"])
        return dict(op=op, n=_log(rng, 1, 1_000_000), width=width, type=rng.choice(["f32", "bf16", "f16"]),
                    post=rng.choice(["none", "rms", "rms", "layer"]), pre=rng.choice(["rms", "rms", "layer"]), gate=gate,
                    sigmoid=gate != "none" and rng.random() < 0.5, residual=rng.choice([1.0, 1.0, 0.5, 1.25]),
                    ld=_draw_ld(rng, width))
    kind, max_norm = rng.choice(["two", "two", "two", "max"]), rng.choice([0.1, 1.0, 1e4])
    if rng.random() < 0.5:
        return dict(op=op, model="slices", k=rng.choice([1, 2, 4, 8]), layers=rng.choice([1, 2, 3]), width=_log(rng, 8, 320),
                    hidden=8 * _log(rng, 4, 64), classes=_log(rng, 2, 64), type="f32", kind=kind, max_norm=max_norm)
    return dict(op=op, model="blocks", layers=_log(rng, 1, 64), width=_log(rng, 16, 1100),
                type=rng.choice(["f32", "bf16", "f16"]), kind=kind, max_norm=max_norm)


def draw(rng):
    """One more case of the same ranges: sizes log-uniform, none costs more than the largest listed one."""
    limit = 2_000_000_000
    while True:
        case = _draw(rng)
        if work(case)["bytes"] <= limit and case.get("n", 1) * case.get("ld", 1) <= 250_000_000:
            return case


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _rows(gen, n, width, ld, kind, std=1.0):
    """n rows of normal values as a view of rows that lie ``ld`` elements apart."""
    return (torch.randn((n, ld), generator=gen, device="cuda") * std).to(TYPES[kind])[:, :width]


def _like(case, kind, n=None):
    return torch.empty((case["n"] if n is None else n, case["ld"]), dtype=TYPES[kind], device="cuda")[:, :case["width"]]


def _tokens(gen, case):
    """Token frequencies fall with their rank, as words' and items' do: the first few make up a tenth of all."""
    n, vocab = case["n"], case["vocab"]
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = (float(vocab) ** u).long().clamp_(1, vocab) - 1
    ids = torch.randperm(vocab, generator=gen, device="cuda")[rank]
    return ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)


def _parameters(case):
    """Shapes and types of a model's parameters, in the order in which it lists them."""
    shapes = []
    if case["model"] == "slices":
        hs = case["hidden"] // case["k"]
        for _ in range(case["k"]):
            for layer in range(case["layers"]):
                wi = case["width"] if layer == 0 else hs
                shapes += [(wi, hs), (hs,), (wi, hs), (hs,)]
        shapes += [(case["k"], hs), (case["k"] * hs, case["hidden"]), (case["hidden"],), (case["hidden"], case["classes"]),
                   (case["classes"],)]
    else:
        w = case["width"]
        for _ in range(case["layers"]):
            shapes += [(w,), (w, 3 * w), (w, w), (w,), (w, 4 * w), (4 * w, w)]
    return [(shape, "f32" if len(shape) == 1 else case["type"]) for shape in shapes]


def _laid_out(parameters):
    """A zeroed buffer per type, and a view into it for every parameter, on 256-byte boundaries as an optimiser keeps them."""
    sizes, places = {}, []
    for shape, kind in parameters:
        start = sizes.get(kind, 0)
        places.append((kind, start, math.prod(shape), shape))
        sizes[kind] = start + -(-math.prod(shape) // 128) * 128
    flat = {kind: torch.zeros(size, dtype=TYPES[kind], device="cuda") for kind, size in sizes.items()}
    return flat, [flat[kind][start:start + count].view(shape) for kind, start, count, shape in places]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case=case, **globals()["_prepare_" + case["op"]](case, gen))
    if own:
        globals()["_buffers_" + case["op"]](case, state)
    return state


def _prepare_embed(case, gen):
    return dict(ids=_tokens(gen, case), table=_rows(gen, case["vocab"], case["width"], case["width"], case["table"], 0.02))


def _prepare_embed_grad(case, gen):
    return dict(ids=_tokens(gen, case), dout=_rows(gen, case["n"], case["width"], case["ld"], case["rows"], 0.01))


def _prepare_resnorm(case, gen):
    n, w, ld, kind = case["n"], case["width"], case["ld"], case["type"]
    s = dict(x=_rows(gen, n, w, ld, kind), y=_rows(gen, n, w, ld, kind, 2.0))
    for name, norm in (("post", case["post"]), ("pre", case["pre"])):
        s[name + "_w"] = 1 + 0.1 * torch.randn(w, generator=gen, device="cuda") if norm != "none" else None
        s[name + "_b"] = 0.1 * torch.randn(w, generator=gen, device="cuda") if norm == "layer" else None
    s["gate"] = (None if case["gate"] == "none" else 0.5 * torch.randn(w, generator=gen, device="cuda") + 0.5
                 if case["gate"] == "column" else _rows(gen, n, w, ld, kind))
    return s


def _prepare_resnorm_grad(case, gen):
    s = _prepare_resnorm(case, gen)
    s["dh"] = _rows(gen, case["n"], case["width"], case["ld"], case["type"])
    s["du"] = _rows(gen, case["n"], case["width"], case["ld"], case["type"])
    return s


def _prepare_clip(case, gen):
    flat, grads = _laid_out(_parameters(case))
    for g in grads:
        g.copy_(torch.randn(g.shape, generator=gen, device="cuda") * 0.01)
    flat_out, outs = _laid_out(_parameters(case))
    return dict(flat=flat, grads=grads, flat_out=flat_out, outs=outs)


# ---- buffers and workspaces of the package's own calls, kept from pass to pass ----------------------------------------

def _bytes(count):
    return torch.empty(count, dtype=torch.uint8, device="cuda")


def _buffers_embed(case, s):
    s["out"] = _like(case, case["rows"])


def _buffers_embed_grad(case, s):
    from paper_2408_11500_amd import binding as B
    s["order"] = torch.empty(case["n"], dtype=torch.int32, device="cuda")
    s["starts"] = torch.empty(case["vocab"] + 1, dtype=torch.int32, device="cuda")
    s["ws_sort"] = _bytes(B.slicegcn_embed_sort_workspace_bytes(case["n"], case["vocab"]))
    s["ws"] = _bytes(B.slicegcn_embed_bwd_workspace_bytes(case["n"], case["width"]))
    s["dtable"] = torch.empty((case["vocab"], case["width"]), dtype=TYPES[case["table"]], device="cuda")


def _buffers_resnorm(case, s):
    s["h"], s["u"] = _like(case, case["type"]), _like(case, case["type"])


def _resnorm_args(case, s):
    from paper_2408_11500_amd import binding as B
    norms = {"none": B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}
    return dict(post=norms[case["post"]], pre=norms[case["pre"]], post_w=s["post_w"], post_b=s["post_b"], pre_w=s["pre_w"],
                pre_b=s["pre_b"], gate=s["gate"], sigmoid=case["sigmoid"], residual=case["residual"], eps=EPS)


def _buffers_resnorm_grad(case, s):
    from paper_2408_11500_amd import binding as B
    # what the forward pass leaves for the backward pass
    s["stats"] = torch.empty((case["n"], 4), dtype=torch.float32, device="cuda")
    h, u = _like(case, case["type"]), _like(case, case["type"])
    B.slicegcn_resnorm_fwd(s["x"], s["y"], h, u, stats=s["stats"], **_resnorm_args(case, s))
    s["ws"] = _bytes(B.slicegcn_resnorm_bwd_workspace_bytes(case["n"], case["width"]))
    s["dx"], s["dy"] = h, u  # buffers of the same shape
    for name in ("post_w", "post_b", "pre_w", "pre_b", "gate"):
        p = s[name]
        s["d" + name] = (None if p is None else torch.empty_like(p) if p.dim() == 1 else _like(case, case["type"]))


def _buffers_clip(case, s):
    from paper_2408_11500_amd import binding as B
    s["norm"] = torch.empty(1, dtype=torch.float32, device="cuda")
    s["from"], s["to"] = B.TensorList(s["grads"]), B.TensorList(s["outs"])
    s["ws"] = _bytes(B.slicegcn_global_norm_workspace_bytes(s["from"]))


# ---- one pass ---------------------------------------------------------------------------------------------------------

def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state["case"], state)


def _pad(case):
    return None if case["pad"] < 0 else case["pad"]


def _scale(case):
    return math.sqrt(case["width"])


def _own_embed(case, s):
    from paper_2408_11500_amd import binding as B
    return B.slicegcn_embed_fwd(s["ids"], s["table"], s["out"], scale=_scale(case), pad=_pad(case))


def _own_embed_grad(case, s):
    from paper_2408_11500_amd import binding as B
    B.slicegcn_embed_sort(s["ids"], case["vocab"], s["order"], s["starts"], s["ws_sort"], pad=_pad(case))
    return B.slicegcn_embed_bwd(s["order"], s["starts"], s["dout"], s["dtable"], s["ws"], scale=_scale(case))


def _own_resnorm(case, s):
    from paper_2408_11500_amd import binding as B
    B.slicegcn_resnorm_fwd(s["x"], s["y"], s["h"], s["u"], **_resnorm_args(case, s))
    return dict(h=s["h"], u=s["u"])


def _own_resnorm_grad(case, s):
    from paper_2408_11500_amd import binding as B
    B.slicegcn_resnorm_bwd(s["x"], s["y"], s["stats"], s["dh"], s["du"], s["dx"], s["dy"], s["ws"], dpost_w=s["dpost_w"],
                           dpost_b=s["dpost_b"], dpre_w=s["dpre_w"], dpre_b=s["dpre_b"], dgate=s["dgate"], **_resnorm_args(case, s))
    out = dict(dx=s["dx"], dy=s["dy"])
    out.update({k: s[k] for k in ("dpost_w", "dpost_b", "dpre_w", "dpre_b", "dgate") if s[k] is not None})
    return out


def _own_clip(case, s):
    from paper_2408_11500_amd import binding as B
    B.slicegcn_clip(s["from"], s["to"], case["max_norm"], s["norm"], s["ws"], kind=B.NORM_MAX if case["kind"] == "max" else B.NORM_TWO)
    return dict(norm=s["norm"], **s["flat_out"])


# The plain forms: elementary operations in 32 bits, long sums in 64, one rounding at the end.

def _plain_embed(case, s):
    out = s["table"][s["ids"].long()].float() * _scale(case)
    if case["pad"] >= 0:
        out = out * (s["ids"] != case["pad"]).float()[:, None]
    return out.to(TYPES[case["rows"]])


def _plain_embed_grad(case, s):
    rows = s["dout"].double()
    if case["pad"] >= 0:
        rows = rows * (s["ids"] != case["pad"]).double()[:, None]
    total = torch.zeros((case["vocab"], case["width"]), dtype=torch.float64, device="cuda")
    total.index_add_(0, s["ids"].long(), rows)
    return (total * _scale(case)).to(TYPES[case["table"]])


def _normed(v, norm):
    """Normalised rows, and the factor they were multiplied by."""
    if norm == "none":
        return v, None
    if norm == "layer":
        v = v - v.mean(dim=1, keepdim=True)
    r = torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS)
    return v * r, r


def _affine(v, w, b):
    if w is not None:
        v = v * w
    return v if b is None else v + b


def _gate(case, s):
    if s["gate"] is None:
        return None
    g = s["gate"].float()
    return torch.sigmoid(g) if case["sigmoid"] else g


def _plain_resnorm(case, s):
    p = _affine(_normed(s["y"].float(), case["post"])[0], s["post_w"], s["post_b"])
    g = _gate(case, s)
    h = case["residual"] * s["x"].float() + (p if g is None else g * p)
    u = _affine(_normed(h, case["pre"])[0], s["pre_w"], s["pre_b"])
    return dict(h=h.to(TYPES[case["type"]]), u=u.to(TYPES[case["type"]]))


def _through_norm(d, v, r, norm):
    """Gradient of the rows from the gradient of the normalised rows v."""
    if norm == "none":
        return d
    out = d - v * (d * v).mean(dim=1, keepdim=True)
    if norm == "layer":
        out = out - d.mean(dim=1, keepdim=True)
    return r * out


def _columns(m):
    return m.sum(dim=0, dtype=torch.float64).float()


def _plain_resnorm_grad(case, s):
    kind = TYPES[case["type"]]
    yn, ry = _normed(s["y"].float(), case["post"])
    p = _affine(yn, s["post_w"], s["post_b"])
    g = _gate(case, s)
    hn, rh = _normed(case["residual"] * s["x"].float() + (p if g is None else g * p), case["pre"])
    du = s["du"].float()
    dh = s["dh"].float() + _through_norm(_affine(du, s["pre_w"], None), hn, rh, case["pre"])
    dp = dh if g is None else dh * g
    dy = _through_norm(_affine(dp, s["post_w"], None), yn, ry, case["post"])
    out = dict(dx=(case["residual"] * dh).to(kind), dy=dy.to(kind))
    for name, value in (("post_w", lambda: dp * yn), ("post_b", lambda: dp), ("pre_w", lambda: du * hn), ("pre_b", lambda: du)):
        if s[name] is not None:
            out["d" + name] = _columns(value())
    if g is not None:
        dg = dh * p * (g * (1 - g)) if case["sigmoid"] else dh * p
        out["dgate"] = _columns(dg) if case["gate"] == "column" else dg.to(kind)
    return out


def _plain_clip(case, s):
    grads = s["grads"]
    if case["kind"] == "max":
        norm = torch.stack([g.float().abs().max() for g in grads]).max().double()
    else:
        norm = torch.stack([(g.float() * g.float()).sum(dtype=torch.float64) for g in grads]).sum().sqrt()
    factor = (case["max_norm"] / norm).clamp(max=1.0).float()
    for g, out in zip(grads, s["outs"]):
        out.copy_(g.float() * factor)
    return dict(norm=norm.float().reshape(1), **s["flat_out"])


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = globals()["_prepare_" + case["op"]](case, gen)
    return globals()["_exact_" + case["op"]](case, s)


def _exact_embed(case, s):
    out = torch.index_select(s["table"].double(), 0, s["ids"].long()).mul_(math.sqrt(case["width"]))
    if case["pad"] >= 0:
        out.masked_fill_((s["ids"] == case["pad"])[:, None], 0.0)
    return out


def _exact_embed_grad(case, s):
    """Rows put in the order of their tokens; a token's sum is the difference of the running sums at its ends."""
    ids, where = torch.sort(s["ids"].long(), stable=True)
    bounds = torch.searchsorted(ids, torch.arange(case["vocab"] + 1, device="cuda"))
    out = torch.empty((case["vocab"], case["width"]), dtype=torch.float64, device="cuda")
    step = max(1, 100_000_000 // max(case["n"], case["vocab"]))
    for c in range(0, case["width"], step):
        run_sum = torch.zeros((case["n"] + 1, min(step, case["width"] - c)), dtype=torch.float64, device="cuda")
        torch.cumsum(s["dout"][:, c:c + step].double()[where], dim=0, out=run_sum[1:])
        out[:, c:c + step] = (run_sum[bounds[1:]] - run_sum[bounds[:-1]]) * math.sqrt(case["width"])
    if case["pad"] >= 0:
        out[case["pad"]] = 0.0
    return out


def _exact_block(case, x, y, post_w, post_b, pre_w, pre_b, gate):
    def norm(v, kind, w, b):
        if kind == "none":
            return v
        mean = v.mean(1, True) if kind == "layer" else 0.0
        v = (v - mean) / torch.sqrt(((v - mean) ** 2).mean(1, True) + EPS)
        return v * w + (0.0 if b is None else b)
    g = 1.0 if gate is None else 1 / (1 + torch.exp(-gate)) if case["sigmoid"] else gate
    h = case["residual"] * x + g * norm(y, case["post"], post_w, post_b)
    return h, norm(h, case["pre"], pre_w, pre_b)


_BLOCK = ("x", "y", "post_w", "post_b", "pre_w", "pre_b", "gate")


def _exact_resnorm(case, s):
    h, u = _exact_block(case, *(None if s[k] is None else s[k].double() for k in _BLOCK))
    return dict(h=h, u=u)


def _exact_resnorm_grad(case, s):
    """The definition differentiated by torch, rows in parts; gradients of weights add up over the parts."""
    whole = ("post_w", "post_b", "pre_w", "pre_b") + (("gate",) if case["gate"] == "column" else ())
    sums, parts = {}, {}
    step = max(1, 50_000_000 // case["width"])
    for r in range(0, case["n"], step):
        leaves = {k: None if s[k] is None else (s[k] if k in whole else s[k][r:r + step]).double().requires_grad_() for k in _BLOCK}
        h, u = _exact_block(case, *(leaves[k] for k in _BLOCK))
        torch.autograd.backward([h, u], [s["dh"][r:r + step].double(), s["du"][r:r + step].double()])
        for k, v in leaves.items():
            if v is not None and k in whole:
                sums[k] = sums.get(k, 0) + v.grad
            elif v is not None:
                parts.setdefault(k, []).append(v.grad)
    grads = {**{k: torch.cat(v) for k, v in parts.items()}, **sums}
    return {"d" + k: grads[k] for k in ("x", "y", "post_w", "post_b", "pre_w", "pre_b", "gate") if k in grads}


def _exact_clip(case, s):
    if case["kind"] == "max":
        norm = max(float(g.double().abs().amax()) for g in s["grads"])
    else:
        norm = math.sqrt(math.fsum(float(torch.dot(g.double().flatten(), g.double().flatten())) for g in s["grads"]))
    factor = min(1.0, case["max_norm"] / norm)
    return dict(norm=torch.tensor([norm], dtype=torch.float64, device="cuda"), **{k: v.double() * factor for k, v in s["flat"].items()})


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def _model_sizes(case):
    """(elements of matrices, elements of vectors) of a clip case."""
    if case["model"] == "slices":
        k, hs, w, h, c = case["k"], case["hidden"] // case["k"], case["width"], case["hidden"], case["classes"]
        m = k * sum(2 * (w if layer == 0 else hs) * hs for layer in range(case["layers"])) + k * hs + k * hs * h + h * c
        return m, 2 * k * case["layers"] * hs + h + c
    w = case["width"]
    return case["layers"] * 12 * w * w, case["layers"] * 2 * w


def work(case):
    op = case["op"]
    if op == "clip":
        m, v = _model_sizes(case)
        return {"bytes": 2 * (m * SIZE[case["type"]] + 4 * v), "flops": 3 * (m + v)}
    n, w = case["n"], case["width"]
    if op in ("embed", "embed_grad"):
        ids = n * (4 if case["ids"] == "i32" else 8)
        table = w * SIZE[case["table"]]
        rows = n * w * SIZE[case["rows"]]
        if op == "embed":  # of a table longer than the batch no more than a row per token is read
            return {"bytes": ids + min(n, case["vocab"]) * table + rows, "flops": n * w}
        return {"bytes": ids + rows + case["vocab"] * table, "flops": n * w + case["vocab"] * w}
    e = SIZE[case["type"]]
    rows = n * w * e
    gate = rows if case["gate"] == "matrix" else 0
    vectors = 4 * w * ((case["post"] != "none") + (case["post"] == "layer") + 1 + (case["pre"] == "layer") + (case["gate"] == "column"))
    if op == "resnorm":
        return {"bytes": 4 * rows + gate + vectors, "flops": 12 * n * w}
    return {"bytes": 6 * rows + 2 * gate + 2 * vectors, "flops": 30 * n * w}
