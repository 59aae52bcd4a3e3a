"""The feed-forward block of a model and the update of its weights, as cases that can be timed: gated projections, products with
their epilogue, and an AdamW step over many tensors.

``run`` computes an operator in its plain form, from elementary torch operations, or with this package's kernels (``own``).
Sizes are those of the benchmark workloads of ``synth.configs`` (cfg1 to cfg4) or generic ones; ``draw`` spreads over the ranges
between them.  A case names its operator and its sizes (n rows, w_in -> w_out columns):

  gated         G = X Wg + bg;  U = X Wu + bu;  H = act(G) * U, with G and U where a backward pass follows (``save``)
  gated_grad    its backward pass, from dH: gradients of X, of both weights and biases
  product       Y = residual * R + act(X W + b), with P = X W + b where a backward pass follows
  product_grad  its backward pass, from dY: gradients of X, W and b
  adamw         m, v and the parameters of a whole model after one step, states in 32 bits or in 8 with scales per block
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
BLOCK = 128  # elements that share a scale of the states in 8 bits
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.1


def listed():
    return [
        # One new row passes a feed-forward block, as when a model answers one request: both weights are read for it.
        dict(name="gated_single", op="gated", n=1, w_in=1024, w_out=2816, type="bf16", act="silu", bias=False, save=False, ld="dense"),
        # Every node of a citation graph (cfg2, hidden 256) through the block of a model in 32 bits, in training.
        dict(name="gated_citation", op="gated", n=169_343, w_in=256, w_out=680, type="f32", act="silu", bias=False, save=True,
             ld="dense"),
        # A wide model in 16 bits on a long batch of tokens.
        dict(name="gated_wide", op="gated", n=8192, w_in=4096, w_out=10240, type="bf16", act="silu", bias=False, save=False, ld="dense"),
        # Backward on a small graph (cfg1), in 32 bits with biases: latency counts, and columns that fill no tile.
        dict(name="gated_grad_small", op="gated_grad", n=2048, w_in=64, w_out=170, type="f32", act="gelu", bias=True, ld="dense"),
        # Backward of the wide model.
        dict(name="gated_grad_wide", op="gated_grad", n=8192, w_in=4096, w_out=10240, type="bf16", act="silu", bias=False, ld="dense"),
        # A few requests at a time on their way back from a block's inner width: the weights are all there is to read.
        dict(name="product_requests", op="product", n=24, w_in=10240, w_out=4096, type="f16", act="none", bias=False, residual=1.0,
             save=False, ld="dense"),
        # A social graph's 602 features (cfg3) projected to its hidden width in 32 bits, in training.
        dict(name="product_social", op="product", n=232_965, w_in=602, w_out=256, type="f32", act="gelu", bias=True, residual=0.0,
             save=True, ld="dense"),
        # The wide model's way back to its width, with the bias and the residual.
        dict(name="product_wide", op="product", n=8192, w_in=10240, w_out=4096, type="bf16", act="none", bias=True, residual=1.0,
             save=False, ld="dense"),
        # Backward of a co-purchase graph's 100 features (cfg4) in 16 bits: 2.4 M rows that fill no tile.
        dict(name="product_grad_items", op="product_grad", n=2_449_029, w_in=100, w_out=256, type="bf16", act="gelu", bias=True,
             residual=0.0, ld="dense"),
        # Backward of the wide model's way back.
        dict(name="product_grad_wide", op="product_grad", n=8192, w_in=10240, w_out=4096, type="bf16", act="none", bias=True,
             residual=1.0, ld="dense"),
        # One step on a small model (cfg1): two slice models of two layers, encoding and classifier.
        dict(name="adamw_small", op="adamw", model="slices", k=2, layers=2, width=64, hidden=64, classes=8, type="f32", bits=32,
             master=False),
        # One step on a large model: 48 blocks of matrices in 16 bits with masters in 32, norms and biases in 32, states in 8.
        dict(name="adamw_large", op="adamw", model="blocks", layers=48, width=1000, type="bf16", bits=8, master=True),
    ]


# ---- drawn cases ------------------------------------------------------------------------------------------------------

def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    op = rng.choice(["gated", "gated", "gated_grad", "gated_grad", "product", "product", "product_grad", "product_grad", "adamw"])
    if op == "adamw":
        kind = rng.choice(["f32", "bf16", "bf16", "f16"])
        c = dict(op=op, type=kind, bits=rng.choice([8, 32]), master=kind != "f32" and rng.random() < 0.6)
        if rng.random() < 0.4:
            return dict(c, model="slices", k=rng.choice([1, 2, 4, 8]), layers=rng.choice([1, 2, 3]), width=_log(rng, 8, 320),
                        hidden=8 * _log(rng, 4, 64), classes=_log(rng, 2, 64))
        return dict(c, model="blocks", layers=_log(rng, 1, 48), width=_log(rng, 16, 1000))
    c = dict(op=op, n=_log(rng, 1, 250_000), w_in=_log(rng, 8, 10240), w_out=_log(rng, 8, 10240), type=rng.choice(["f32", "bf16", "f16"]),
             act=rng.choice(["silu", "silu", "gelu", "relu", "none"]), bias=rng.random() < 0.5, ld=rng.choice(["dense", "dense", "lines", "odd"]))
    if op in ("gated", "product"):
        c["save"] = rng.random() < 0.5 and (op == "gated" or c["act"] != "none")
    if op in ("product", "product_grad"):
        c["residual"] = rng.choice([0.0, 1.0, 1.0, 0.5])
    return c


def draw(rng):
    """One more case of the same ranges: sizes log-uniform, none costs more than the largest listed one."""
    while True:
        case = _draw(rng)
        w = work(case)
        if w["flops"] <= (2.7e12 if case.get("type") != "f32" or case["op"] == "adamw" else 0.5e12) and w["bytes"] <= 5e9:
            return case


# ---- inputs -----------------------------------------------------------------------------------------------------------

def _ld(case, width):
    """Leading dimension of rows: contiguous, on whole cache lines, or neither."""
    return width if case["ld"] == "dense" else (width + 63) // 64 * 64 if case["ld"] == "lines" else width + 1 + width % 5


def _rows(gen, case, width, std=1.0):
    """n rows of normal values as a view of rows that lie a leading dimension apart."""
    m = torch.randn((case["n"], _ld(case, width)), generator=gen, device="cuda").mul_(std)
    return m.to(TYPES[case["type"]])[:, :width]


def _weights(gen, case):
    std = 1 / math.sqrt(case["w_in"])
    return (torch.randn((case["w_in"], case["w_out"]), generator=gen, device="cuda") * std).to(TYPES[case["type"]])


def _bias(gen, case):
    return 0.1 * torch.randn(case["w_out"], generator=gen, device="cuda") if case["bias"] else None


def _projected(case, x, w, b):
    p = x.float() @ w.float()
    out = torch.empty((case["n"], _ld(case, case["w_out"])), dtype=TYPES[case["type"]], device="cuda")[:, :case["w_out"]]
    return out.copy_(p if b is None else p + b)


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


def _spread(shapes):
    """Where each tensor starts in a buffer that holds them on boundaries of whole blocks, and the buffer's length."""
    starts, total = [], 0
    for shape in shapes:
        starts.append(total)
        total += -(-math.prod(shape) // BLOCK) * BLOCK
    return starts, total


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    state = dict(case=case, **globals()["_prepare_" + case["op"]](case, gen))
    if own:
        globals()["_buffers_" + case["op"]](case, state)
    return state


def _prepare_gated(case, gen):
    return dict(x=_rows(gen, case, case["w_in"]), wg=_weights(gen, case), wu=_weights(gen, case), bg=_bias(gen, case),
                bu=_bias(gen, case))


def _prepare_gated_grad(case, gen):
    s = _prepare_gated(case, gen)
    # what the forward pass kept
    s["g"], s["u"] = _projected(case, s["x"], s["wg"], s["bg"]), _projected(case, s["x"], s["wu"], s["bu"])
    s["dh"] = _rows(gen, case, case["w_out"], 0.1)
    return s


def _prepare_product(case, gen):
    return dict(x=_rows(gen, case, case["w_in"]), w=_weights(gen, case), b=_bias(gen, case),
                r=_rows(gen, case, case["w_out"]) if case["residual"] else None)


def _prepare_product_grad(case, gen):
    s = dict(x=_rows(gen, case, case["w_in"]), w=_weights(gen, case), b=_bias(gen, case))
    s["p"] = _projected(case, s["x"], s["w"], s["b"]) if case["act"] != "none" else None
    s["dy"] = _rows(gen, case, case["w_out"], 0.1)
    return s


def _prepare_adamw(case, gen):
    """Parameters, gradients and states of a model in the middle of its training, each kind in one buffer."""
    parameters = _parameters(case)
    shapes = [shape for shape, _ in parameters]
    starts, total = _spread(shapes)
    f32 = dict(dtype=torch.float32, device="cuda")
    flat, tensors = {}, []
    by_kind = {kind: _spread([s for s, k in parameters if k == kind]) for kind in {k for _, k in parameters}}
    for kind, (_, size) in by_kind.items():
        for what in ("param", "grad") + (("master",) if case["master"] and kind != "f32" else ()):
            flat[what + "_" + kind] = torch.zeros(size, dtype=torch.float32 if what == "master" else TYPES[kind], device="cuda")
    m, v = (torch.zeros(total, **f32) for _ in range(2))
    nexts = {kind: iter(s) for kind, (s, _) in by_kind.items()}
    for (shape, kind), at in zip(parameters, starts):
        count, of_kind = math.prod(shape), next(nexts[kind])
        t = {what: flat[what + "_" + kind][of_kind:of_kind + count].view(shape)
             for what in ("param", "grad", "master") if what + "_" + kind in flat}
        values = torch.randn(shape, generator=gen, device="cuda") * (0.02 if len(shape) > 1 else 0.1)
        t["param"].copy_(values)
        if "master" in t:
            t["master"].copy_(values)
        t["grad"].copy_(torch.randn(shape, generator=gen, device="cuda") * 1e-2)
        m[at:at + count].normal_(generator=gen).mul_(3e-3)
        v[at:at + count].normal_(generator=gen).square_().mul_(1e-4).add_(1e-6)
        t.update(at=at, count=count, decay=DECAY if len(shape) > 1 else 0.0)
        tensors.append(t)
    if case["bits"] == 8:
        flat["m"], flat["v"] = (torch.zeros(total, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
        flat["scales"] = torch.empty((total // BLOCK, 2), dtype=torch.float8_e8m0fnu, device="cuda")
        for i, (codes, values) in enumerate((("m", m), ("v", v))):
            blocks = values.view(-1, BLOCK)
            byte = ((blocks.abs().amax(1).view(torch.int32) >> 23) - 7).clamp(min=1)
            flat[codes].copy_((blocks * _power(127 - byte)[:, None]).view(-1))
            flat["scales"].view(torch.uint8)[:, i] = byte.to(torch.uint8)
    else:
        flat["m"], flat["v"] = m, v
    for t in tensors:
        t["m"], t["v"] = (flat[k][t["at"]:t["at"] + t["count"]] for k in ("m", "v"))
        t["scales"] = flat["scales"][t["at"] // BLOCK:-(-(t["at"] + t["count"]) // BLOCK)] if case["bits"] == 8 else None
    factor = torch.rand(1, generator=gen, device="cuda") * 0.5 + 0.5  # of the clipping, where the norm over all gradients put it
    return dict(flat=flat, tensors=tensors, factor=factor, step=1000, seed=1000)


# ---- buffers and workspaces of the package's own calls, kept from pass to pass ----------------------------------------

def _like(case, width):
    return torch.empty((case["n"], _ld(case, width)), dtype=TYPES[case["type"]], device="cuda")[:, :width]


def _bytes(count):
    return torch.empty(count, dtype=torch.uint8, device="cuda")


def _act(case):
    from paper_2408_11500_amd import binding as B
    return {"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU}[case["act"]]


def _buffers_gated(case, s):
    from paper_2408_11500_amd import binding as B
    s["h"] = _like(case, case["w_out"])
    s["g"], s["u"] = (_like(case, case["w_out"]) if case["save"] else None for _ in range(2))
    s["ws"] = _bytes(B.slicegcn_gated_fwd_workspace_bytes(case["n"], case["w_in"], case["w_out"], TYPES[case["type"]]))


def _buffers_gated_grad(case, s):
    from paper_2408_11500_amd import binding as B
    s["dx"] = _like(case, case["w_in"])
    s["dwg"], s["dwu"] = torch.empty_like(s["wg"]), torch.empty_like(s["wu"])
    s["dbg"], s["dbu"] = (torch.empty_like(s[k]) if case["bias"] else None for k in ("bg", "bu"))
    s["ws"] = _bytes(B.slicegcn_gated_bwd_workspace_bytes(case["n"], case["w_in"], case["w_out"], TYPES[case["type"]]))


def _buffers_product(case, s):
    from paper_2408_11500_amd import binding as B
    s["y"] = _like(case, case["w_out"])
    s["p"] = _like(case, case["w_out"]) if case["save"] else None
    s["ws"] = _bytes(B.slicegcn_product_fwd_workspace_bytes(case["n"], case["w_in"], case["w_out"], TYPES[case["type"]]))


def _buffers_product_grad(case, s):
    from paper_2408_11500_amd import binding as B
    s["dx"], s["dw"] = _like(case, case["w_in"]), torch.empty_like(s["w"])
    s["db"] = torch.empty_like(s["b"]) if case["bias"] else None
    s["ws"] = _bytes(B.slicegcn_product_bwd_workspace_bytes(case["n"], case["w_in"], case["w_out"], TYPES[case["type"]]))


def _buffers_adamw(case, s):
    from paper_2408_11500_amd import binding as B
    ts = s["tensors"]
    s["list"] = B.AdamList([t["param"] for t in ts], [t["grad"] for t in ts], [t["m"] for t in ts], [t["v"] for t in ts],
                           scales=[t["scales"] for t in ts], masters=[t.get("master") for t in ts], decays=[t["decay"] for t in ts])


# ---- one pass ---------------------------------------------------------------------------------------------------------

def run(state):
    return globals()[("_own_" if own else "_plain_") + state["case"]["op"]](state["case"], state)


def _present(**outputs):
    return {k: v for k, v in outputs.items() if v is not None}


def _updated(s):
    return {k: v for k, v in s["flat"].items() if not k.startswith("grad")}


def _own_gated(case, s):
    from paper_2408_11500_amd import binding as B
    B.slicegcn_gated_fwd(s["x"], s["wg"], s["wu"], s["h"], s["ws"], bg=s["bg"], bu=s["bu"], G=s["g"], U=s["u"], act=_act(case))
    return _present(h=s["h"], g=s["g"], u=s["u"])


def _own_gated_grad(case, s):
    from paper_2408_11500_amd import binding as B
    B.slicegcn_gated_bwd(s["x"], s["wg"], s["wu"], s["g"], s["u"], s["dh"], s["ws"], dX=s["dx"], dWg=s["dwg"], dWu=s["dwu"],
                         dbg=s["dbg"], dbu=s["dbu"], act=_act(case))
    return _present(dx=s["dx"], dwg=s["dwg"], dwu=s["dwu"], dbg=s["dbg"], dbu=s["dbu"])


def _own_product(case, s):
    from paper_2408_11500_amd import binding as B
    B.slicegcn_product_fwd(s["x"], s["w"], s["y"], s["ws"], b=s["b"], R=s["r"], P=s["p"], act=_act(case), residual=case["residual"])
    return _present(y=s["y"], p=s["p"])


def _own_product_grad(case, s):
    from paper_2408_11500_amd import binding as B
    B.slicegcn_product_bwd(s["x"], s["w"], s["p"], s["dy"], s["ws"], dX=s["dx"], dW=s["dw"], db=s["db"], act=_act(case))
    return _present(dx=s["dx"], dw=s["dw"], db=s["db"])


def _own_adamw(case, s):
    from paper_2408_11500_amd import binding as B
    B.slicegcn_adamw_step(s["list"], LR, s["step"], beta1=BETA1, beta2=BETA2, eps=EPS, factor=s["factor"], seed=s["seed"])
    return _updated(s)


# The plain forms: elementary operations in 32 bits, long sums in 64, one rounding at the end.

def _activated(case, v):
    act = case["act"]
    if act == "none":
        return v
    if act == "relu":
        return v.clamp(min=0)
    return v * torch.sigmoid(v) if act == "silu" else v * 0.5 * (1 + torch.erf(v * math.sqrt(0.5)))


def _slope(case, v):
    act = case["act"]
    if act == "none":
        return torch.ones_like(v)
    if act == "relu":
        return (v > 0).float()
    if act == "silu":
        s = torch.sigmoid(v)
        return s * (1 + v * (1 - s))
    return 0.5 * (1 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1 / math.sqrt(2 * math.pi))


def _affine(x, w, b):
    p = x.float() @ w.float()
    return p if b is None else p + b


def _columns(m):
    return m.sum(dim=0, dtype=torch.float64).float()


def _plain_gated(case, s):
    kind = TYPES[case["type"]]
    g, u = _affine(s["x"], s["wg"], s["bg"]), _affine(s["x"], s["wu"], s["bu"])
    h = (_activated(case, g) * u).to(kind)
    return dict(h=h, g=g.to(kind), u=u.to(kind)) if case["save"] else dict(h=h)


def _plain_gated_grad(case, s):
    kind = TYPES[case["type"]]
    x, g, dh = s["x"].float(), s["g"].float(), s["dh"].float()
    dg, du = dh * s["u"].float() * _slope(case, g), dh * _activated(case, g)
    out = dict(dx=(dg @ s["wg"].float().t() + du @ s["wu"].float().t()).to(kind), dwg=(x.t() @ dg).to(kind), dwu=(x.t() @ du).to(kind))
    return dict(out, dbg=_columns(dg), dbu=_columns(du)) if case["bias"] else out


def _plain_product(case, s):
    kind = TYPES[case["type"]]
    p = _affine(s["x"], s["w"], s["b"])
    y = _activated(case, p)
    if s["r"] is not None:
        y = case["residual"] * s["r"].float() + y
    return dict(y=y.to(kind), p=p.to(kind)) if case["save"] else dict(y=y.to(kind))


def _plain_product_grad(case, s):
    kind = TYPES[case["type"]]
    dp = s["dy"].float()
    if s["p"] is not None:
        dp = dp * _slope(case, s["p"].float())
    out = dict(dx=(dp @ s["w"].float().t()).to(kind), dw=(s["x"].float().t() @ dp).to(kind))
    return dict(out, db=_columns(dp)) if case["bias"] else out


def _noise(seed, tensor, count):
    """32 bits for every element of a tensor of the list: the upper half for m, the lower one for v."""
    low = 0xFFFFFFFF
    key = ((seed & low) * 0x6A09E667 + (seed >> 32) * 0xBB67AE85 + tensor * 0x3C6EF373) & low
    x = (torch.arange(count, device="cuda") * 0x9E3779B9 + key) & low
    x = x ^ (x >> 15)
    x = (x * 0xA54FF53B) & low
    return x ^ (x >> 16)


def _power(exponent):
    """2^exponent in 32 bits, for exponents of normal numbers."""
    return ((exponent + 127) << 23).to(torch.int32).view(torch.float32)


def _blocks(values):
    """Rows of a block each; the last one filled up with zeros."""
    return torch.nn.functional.pad(values, (0, -values.numel() % BLOCK)).view(-1, BLOCK)


def _decoded(codes, scales, which):
    power = _power(scales.view(torch.uint8)[:, which].int() - 127)
    return (_blocks(codes.float()) * power[:, None]).view(-1)[:codes.numel()]


def _store_8(values, noise, codes, scales, which):
    """values as e4m3 numbers times a power of two per block, rounded up or down by chance (16 bits), without bias."""
    blocks = _blocks(values)
    byte = ((blocks.abs().amax(1).view(torch.int32) >> 23) - 7).clamp(min=1)
    t = blocks.abs() * _power(127 - byte)[:, None]
    lift = (t < 2.0 ** -6).float() * 2.0 ** -6  # below the smallest normal number the grid is that of the binade above it
    bits = (t + lift).view(torch.int32) + (_blocks(noise) << 4).to(torch.int32)
    t = (bits & -(1 << 20)).view(torch.float32) - lift
    if which == 1:
        t = torch.where((blocks > 0) & (t == 0), 2.0 ** -9, t)
    codes.copy_(torch.copysign(t, blocks).view(-1)[:codes.numel()])
    scales.view(torch.uint8)[:, which] = byte.to(torch.uint8)


def _plain_adamw(case, s):
    """In place, as the step is.  Every operation that a state in 8 bits depends on is rounded by itself."""
    c1, c2 = 1 - BETA1 ** s["step"], 1 - BETA2 ** s["step"]
    for i, t in enumerate(s["tensors"]):
        p = t.get("master", t["param"]).float()
        g = t["grad"].float() * s["factor"]
        m, v = t["m"], t["v"]
        if case["bits"] == 8:
            m, v = _decoded(m, t["scales"], 0), _decoded(v, t["scales"], 1)
        m = m * BETA1 + g.view(-1) * (1 - BETA1)
        v = v * BETA2 + (g * g).view(-1) * (1 - BETA2)
        update = (m * (1 / c1)) / ((v * (1 / c2)).sqrt() + EPS)
        p = p - (LR * t["decay"]) * p - LR * update.view(p.shape)
        if "master" in t:
            t["master"].copy_(p)
        t["param"].copy_(p)
        if case["bits"] == 8:
            noise = _noise(s["seed"], i, t["count"])
            _store_8(m, noise >> 16, t["m"], t["scales"], 0)
            _store_8(v, noise & 0xFFFF, t["v"], t["scales"], 1)
        else:
            t["m"].copy_(m)
            t["v"].copy_(v)
    return _updated(s)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = globals()["_prepare_" + case["op"]](case, gen)
    return globals()["_exact_" + case["op"]](case, s)


def _exact_act(case, v):
    return {"none": lambda: v, "relu": lambda: torch.where(v > 0, v, 0.0), "silu": lambda: v / (1 + torch.exp(-v)),
            "gelu": lambda: v * 0.5 * torch.special.erfc(-v / math.sqrt(2.0))}[case["act"]]()


def _with_slope(case, v):
    """act(v) and its derivative, by differentiation."""
    v = v.clone().requires_grad_()
    y = _exact_act(case, v)
    return y.detach(), torch.autograd.grad(y.sum(), v)[0]


def _parts(case, width):
    step = max(1, 200_000_000 // width)
    return [slice(r, min(r + step, case["n"])) for r in range(0, case["n"], step)]


def _exact_gated(case, s):
    wg, wu = s["wg"].double(), s["wu"].double()
    g, u = (torch.cat([torch.mm(s["x"][r].double(), w) for r in _parts(case, case["w_in"])]) for w in (wg, wu))
    if case["bias"]:
        g, u = g + s["bg"], u + s["bu"]
    out = dict(h=_exact_act(case, g) * u)
    return dict(out, g=g, u=u) if case["save"] else out


def _exact_gated_grad(case, s):
    wg, wu = s["wg"].double(), s["wu"].double()
    dx, dwg, dwu, dbg, dbu = [], 0.0, 0.0, 0.0, 0.0
    for r in _parts(case, case["w_in"] + 4 * case["w_out"]):
        x, dh = s["x"][r].double(), s["dh"][r].double()
        y, slope = _with_slope(case, s["g"][r].double())
        dg, du = slope * s["u"][r] * dh, y * dh
        dx.append(torch.mm(du, wu.t()) + torch.mm(dg, wg.t()))
        dwg, dwu = dwg + torch.mm(x.t(), dg), dwu + torch.mm(x.t(), du)
        dbg, dbu = dbg + dg.sum(0), dbu + du.sum(0)
    out = dict(dx=torch.cat(dx), dwg=dwg, dwu=dwu)
    return dict(out, dbg=dbg, dbu=dbu) if case["bias"] else out


def _exact_product(case, s):
    w = s["w"].double()
    p = torch.cat([torch.mm(s["x"][r].double(), w) for r in _parts(case, case["w_in"])])
    if case["bias"]:
        p = p + s["b"]
    y = _exact_act(case, p)
    if case["residual"]:
        y = y + case["residual"] * s["r"]
    return dict(y=y, p=p) if case["save"] else dict(y=y)


def _exact_product_grad(case, s):
    w = s["w"].double()
    dx, dw, db = [], 0.0, 0.0
    for r in _parts(case, case["w_in"] + 4 * case["w_out"]):
        dp = s["dy"][r].double()
        if s["p"] is not None:
            dp = dp * _with_slope(case, s["p"][r].double())[1]
        dx.append(torch.mm(dp, w.t()))
        dw, db = dw + torch.mm(s["x"][r].double().t(), dp), db + dp.sum(0)
    out = dict(dx=torch.cat(dx), dw=dw)
    return dict(out, db=db) if case["bias"] else out


def _exact_8(values, chance, floor):
    """(numbers on the e4m3 grid, scale per block): each value goes to the grid point below it or to the next, by ``chance``."""
    pad = -values.numel() % BLOCK
    blocks = torch.cat([values, values.new_zeros(pad)]).view(-1, BLOCK)
    chance = torch.cat([chance, chance.new_zeros(pad)]).view(-1, BLOCK)
    def power(e):
        return ((e.long() + 1023) << 52).view(torch.float64)
    largest = blocks.abs().amax(1)
    exponent = torch.frexp(largest)[1] - 1  # 2^exponent <= largest
    scale = power(torch.where(largest > 0, (exponent - 7).clamp(min=-126), -126))
    t = blocks.abs() / scale[:, None]
    quantum = power(torch.where(t > 0, torch.frexp(t)[1] - 4, -9).clamp(min=-9))
    t = torch.floor(t / quantum + chance) * quantum
    if floor:
        t = torch.where(blocks > 0, t.clamp(min=2.0 ** -9), t)
    return (t * blocks.sign()).view(-1)[:values.numel()], scale


def _exact_adamw(case, s):
    out = {k: torch.zeros(v.shape, dtype=torch.float64, device="cuda") for k, v in _updated(s).items()}
    if case["bits"] == 8:
        out["scales"].fill_(1.0)
    places = {k: 0 for k in out}
    for i, t in enumerate(s["tensors"]):
        kind = next(k for k, v in TYPES.items() if v is t["param"].dtype)
        blocks = slice(t["at"] // BLOCK, t["at"] // BLOCK + -(-t["count"] // BLOCK))
        here = slice(t["at"], t["at"] + t["count"])
        m, v = t["m"].double(), t["v"].double()
        if case["bits"] == 8:
            scale = t["scales"].double().repeat_interleave(BLOCK, dim=0)[:t["count"]]
            m, v = m * scale[:, 0], v * scale[:, 1]
        g = t["grad"].double().flatten() * s["factor"].double()
        m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g ** 2
        p = t.get("master", t["param"]).double().flatten()
        p = p - LR * (t["decay"] * p + m / (1 - BETA1 ** s["step"]) / (torch.sqrt(v / (1 - BETA2 ** s["step"])) + EPS))
        for what in ("param", "master"):
            if what in t:
                at = places[what + "_" + kind]
                out[what + "_" + kind][at:at + t["count"]] = p
                places[what + "_" + kind] = at + -(-t["count"] // BLOCK) * BLOCK
        if case["bits"] == 8:
            noise = _noise(s["seed"], i, t["count"])
            for which, (name, values, chance) in enumerate((("m", m, noise >> 16), ("v", v, noise & 0xFFFF))):
                out[name][here], out["scales"][blocks, which] = _exact_8(values, chance.double() / 65536, which == 1)
        else:
            out["m"][here], out["v"][here] = m, v
    return out


# ---- what a pass cannot do without ------------------------------------------------------------------------------------

def work(case):
    op, e = case["op"], SIZE[case["type"]]
    if op == "adamw":
        total = {"bytes": 0, "flops": 0}
        for shape, kind in _parameters(case):
            count = math.prod(shape)
            state = 16 if case["bits"] == 32 else 4 + 4 / BLOCK  # both read and written
            master = 8 + SIZE[kind] if case["master"] and kind != "f32" else 2 * SIZE[kind]
            total["bytes"] += int(count * (state + master + SIZE[kind]))
            total["flops"] += 16 * count
        return total
    n, wi, wo = case["n"], case["w_in"], case["w_out"]
    x, y, w, b = n * wi * e, n * wo * e, wi * wo * e, 4 * wo * case["bias"]
    if op == "gated":
        return {"bytes": x + 2 * w + 2 * b + y * (3 if case["save"] else 1), "flops": 4 * n * wi * wo + 6 * n * wo}
    if op == "gated_grad":
        return {"bytes": 2 * x + 4 * w + 2 * b + 3 * y, "flops": 8 * n * wi * wo + 12 * n * wo}
    if op == "product":
        return {"bytes": x + w + b + y * (1 + bool(case["residual"]) + case["save"]), "flops": 2 * n * wi * wo + 4 * n * wo}
    return {"bytes": 2 * x + 2 * w + b + y * (1 + (case["act"] != "none")), "flops": 4 * n * wi * wo + 6 * n * wo}
