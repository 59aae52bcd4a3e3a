"""Plain 64-bit forms of products and gated projections with bounds on what the kernels may be off by (see train_util for U and half_step).

A sum of K products goes through the matrix cores 32 terms at a time, so that a term passes at most 32 additions inside an instruction and one for every
instruction after it: K / 32 of them, six times as many for fp32 operands, which are split in three.  Additions may truncate (2 U each).  The
products themselves are exact for 16-bit operands; for fp32 ones what the split leaves out is below 4 U of a product.  Parts of k are joined in fp64."""
import torch

from train_util import F64, U, half_step

ACTS = ("none", "relu", "silu", "gelu")


def depth(k, dtype):
    """Relative error of a sum of k products, in terms of the sum of their absolute values."""
    return U * (2 * (34 + (6 if dtype == torch.float32 else 1) * -(-k // 32)) + 4)


def act(v, name):
    """act(v) and its derivative."""
    if name == "none":
        return v, torch.ones_like(v)
    if name == "relu":
        return v.clamp(min=0), (v > 0).to(F64)
    if name == "silu":
        s = torch.sigmoid(v)
        return v * s, s * (1 + v * (1 - s))
    p = 0.5 * torch.special.erfc(-v / 2 ** 0.5)
    return v * p, p + v * torch.exp(-v * v / 2) / (2 * torch.pi) ** 0.5


# |act'| <= 1.13 for all of them; what act(v) itself is off by is some rounding errors of its steps, each relative to at most |v| (the arguments of exp and erfc are
# rounded too: by U |v| of an exponent of at most v^2 / 2, where the value has fallen faster than that grows)
SLOPE, STEPS = 1.13, 16


def projection(x, w, b, dtype):
    """X W + b and its bound."""
    size = x.abs() @ w.abs()
    p = x @ w
    if b is not None:
        p, size = p + b, size + b.abs()
    return p, (depth(x.shape[1], dtype) + U) * size


def product_fwd(x, w, b, r, residual, name, dtype):
    """{output: (value, bound)}."""
    p, ep = projection(x, w, b, dtype)
    y, _ = act(p, name)
    ey = SLOPE * ep + (STEPS * U * p.abs() if name != "none" else 0)
    if r is not None:
        y = residual * r + y
        ey = ey + U * (abs(residual) * r.abs() * 2 + y.abs())
    return dict(P=(p, ep), Y=(y, ey))


def gated_fwd(x, wg, wu, bg, bu, name, dtype):
    (g, eg), (u, eu) = projection(x, wg, bg, dtype), projection(x, wu, bu, dtype)
    a, _ = act(g, name)
    ea = SLOPE * eg + STEPS * U * g.abs()
    return dict(G=(g, eg), U=(u, eu), H=(a * u, ea * (u.abs() + eu) + a.abs() * eu + 2 * U * (a * u).abs()))


def _products(x, pairs, dtype, terms):
    """Gradients of X and of the weights from [(dP, bound of dP, W)]: dP is rounded to the rows' type before the products, or is the sum of two terms that are."""
    dx = ex = 0
    out = []
    for dp, ep, w in pairs:
        ep = ep + (half_step(dp, dtype) if terms == 1 else half_step(half_step(dp, dtype), dtype))
        k = w.shape[1] * len(pairs)
        dx, ex = dx + dp @ w.t(), ex + (ep + depth(k, dtype) * (dp.abs() + ep)) @ w.abs().t()
        n = dp.shape[0]
        out.append((x.t() @ dp, x.abs().t() @ (ep + depth(n, dtype) * (dp.abs() + ep))))
    return (dx, ex), out


def _columns(dp, ep):
    """Column sums of unrounded gradients: 32 rows at a time in fp32, then fp64."""
    return dp.sum(0), (ep + 34 * U * dp.abs()).sum(0)


def product_bwd(x, w, p, dy, residual, name, dtype, terms=1):
    if name == "none":
        dp, ep = dy, torch.zeros_like(dy)
    else:
        _, slope = act(p, name)
        dp, ep = dy * slope, dy.abs() * U * (STEPS * (1 + p.abs()) + 2)
    dx, (dw,) = _products(x, [(dp, ep, w)], dtype, terms)
    return dict(dX=dx, dW=dw, db=_columns(dp, ep), dR=(residual * dy, U * (residual * dy).abs()))


def gated_bwd(x, wg, wu, g, u, dh, name, dtype, terms=1):
    y, slope = act(g, name)
    dg, du = dh * u * slope, dh * y
    eg, eu = dh.abs() * u.abs() * U * (STEPS * (1 + g.abs()) + 2), dh.abs() * U * (STEPS + 2) * g.abs()
    dx, (dwg, dwu) = _products(x, [(dg, eg, wg), (du, eu, wu)], dtype, terms)
    return dict(dX=dx, dWg=dwg, dWu=dwu, dbg=_columns(dg, eg), dbu=_columns(du, eu))
