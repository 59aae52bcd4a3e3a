"""Plain 64-bit forms of the operators of slicegcn_train.h (torch on the CPU), with bounds on what fp32 arithmetic may be off by.

U = 2^-24 is the relative error of one fp32 operation.  A result is compared within C * U times the size of everything that was added up to
form it (the formula evaluated with absolute values) plus half a step of its own type."""
import torch

U = 2.0 ** -24
F64 = torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def half_step(want, dtype):
    """Largest rounding error of a result of this type: half a step of a normal number, of the smallest one below those."""
    f = torch.finfo(dtype)
    return want.abs() * (f.eps / 2) + f.tiny * f.eps


def assert_within(got, want, bound, what):
    got = got.detach().cpu()
    assert got.shape == want.shape, what
    tol = bound + half_step(want, got.dtype)
    err = (got.to(F64) - want).abs()
    bad = ~(err <= tol)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, the first at {tuple(bad.nonzero()[0].tolist())}: "
                           f"{float(got[tuple(bad.nonzero()[0])])} for {float(want[tuple(bad.nonzero()[0])])}, {float((err / tol.clamp_min(1e-300)).max()):.2f} of the bound")


def rows(gen, n, width, dtype, ld=None, offset=0, std=1.0, device="cuda"):
    """Normal values as a view with leading dimension ld that starts `offset` elements into its buffer; (device view, 64-bit copy)."""
    ld = width if ld is None else ld
    buf = torch.full((n * ld + offset,), float("nan"), dtype=dtype)
    view = buf[offset:].view(n, ld)[:, :width]
    view.copy_((torch.randn((n, width), generator=gen) * std).to(dtype))
    dev = buf.to(device)
    return dev[offset:].view(n, ld)[:, :width], view.to(F64)


# ---- embedding ------------------------------------------------------------------------------------------------------------

def embed_fwd(ids, table, scale, pad):
    ok = (ids >= 0) & (ids < table.shape[0])
    out = table[torch.where(ok, ids, 0)] * scale
    out[~ok] = float("nan")
    if pad is not None:
        out[ids == pad] = 0.0
    return out


def embed_grad(ids, dout, vocab, scale, pad):
    """The gradient, and the same sum of absolute values."""
    ok = (ids >= 0) & (ids < vocab)
    if pad is not None:
        ok &= ids != pad
    total, size = (torch.zeros((vocab, dout.shape[1]), dtype=F64) for _ in range(2))
    total.index_add_(0, ids[ok], dout[ok])
    size.index_add_(0, ids[ok], dout[ok].abs())
    return total * scale, size * abs(scale)


# ---- residual norm --------------------------------------------------------------------------------------------------------

NONE, RMS, LAYER = 0, 1, 2


def norm(v, kind, eps):
    """Normalised rows, the factor, and the size of what they were formed from."""
    if kind == NONE:
        return v, torch.ones_like(v[:, :1]), v.abs()
    mean = v.mean(1, True) if kind == LAYER else torch.zeros_like(v[:, :1])
    r = 1 / torch.sqrt(((v - mean) ** 2).mean(1, True) + eps)
    return (v - mean) * r, r, r * (v.abs() + (v.abs().mean(1, True) if kind == LAYER else 0))


def _or(t, default):
    return torch.tensor(default, dtype=F64) if t is None else t


class Resnorm:
    """One call in 64 bits.  Arguments are 64-bit tensors or None; names as in the binding."""

    def __init__(self, x, y, post=NONE, pre=NONE, post_w=None, post_b=None, pre_w=None, pre_b=None, gate=None, sigmoid=False,
                 residual=1.0, eps=1e-6):
        self.__dict__.update(locals())
        zero = torch.zeros_like(x if x is not None else y)
        self.s = torch.ones(1, dtype=F64) if gate is None else torch.sigmoid(gate) if sigmoid else gate
        if y is None:
            self.yn = self.yn_size = self.p = self.p_size = zero
            self.ry = zero[:, :1] + 1
        else:
            self.yn, self.ry, self.yn_size = norm(y, post, eps)
            self.p = self.yn * _or(post_w, 1.0) + _or(post_b, 0.0)
            self.p_size = self.yn_size * _or(post_w, 1.0).abs() + _or(post_b, 0.0).abs()
        xr = zero if x is None else residual * x
        self.h = xr + self.s * self.p
        self.h_size = xr.abs() + self.s.abs() * self.p_size
        self.hn, self.rh, _ = norm(self.h, pre, eps)
        self.hn_size = self.h_size if pre == NONE else self.rh * (self.h_size + (self.h_size.mean(1, True) if pre == LAYER else 0))
        self.hn_size = torch.maximum(self.hn_size, self.hn.abs() * self.rh * self.h_size.amax(1, True)) if pre != NONE else self.hn_size
        self.u = self.hn * _or(pre_w, 1.0) + _or(pre_b, 0.0)
        self.u_size = self.hn_size * _or(pre_w, 1.0).abs() + _or(pre_b, 0.0).abs()

    def backward(self, dh, du):
        """Gradients by the formulas, and their sizes: two dicts."""
        zero = torch.zeros_like(self.h)
        dh, du = _or(dh, 0.0) + zero, (_or(du, 0.0) + zero)
        g, z = {}, {}

        def through(d, dsize, v, vsize, r, kind):
            if kind == NONE:
                return d, dsize
            out = d - v * (d * v).mean(1, True) - (d.mean(1, True) if kind == LAYER else 0)
            size = dsize + vsize * (dsize * vsize).mean(1, True) + (dsize.mean(1, True) if kind == LAYER else 0)
            return r * out, r * size
        dun = du * _or(self.pre_w, 1.0)
        a, asize = through(dun, dun.abs(), self.hn, self.hn_size, self.rh, self.pre)
        dH, dHs = dh + a, dh.abs() + asize
        g["dx"], z["dx"] = self.residual * dH, abs(self.residual) * dHs
        g["dpre_w"], z["dpre_w"] = (du * self.hn).sum(0), (du.abs() * self.hn_size).sum(0)
        g["dpre_b"], z["dpre_b"] = du.sum(0), du.abs().sum(0)
        slope = self.s * (1 - self.s) if self.sigmoid else torch.ones(1, dtype=F64)
        g["dgate"], z["dgate"] = dH * self.p * slope, dHs * self.p_size * (1.0 if not self.sigmoid else 0.25 + self.s.abs())
        if self.gate is None or self.gate.dim() == 1:
            g["dgate"], z["dgate"] = g["dgate"].sum(0), z["dgate"].sum(0)
        dp, dps = dH * self.s, dHs * self.s.abs()
        g["dpost_w"], z["dpost_w"] = (dp * self.yn).sum(0), (dps * self.yn_size).sum(0)
        g["dpost_b"], z["dpost_b"] = dp.sum(0) + torch.zeros(self.h.shape[1], dtype=F64), dps.sum(0) + torch.zeros(self.h.shape[1], dtype=F64)
        w = _or(self.post_w, 1.0)
        g["dy"], z["dy"] = through(dp * w, dps * w.abs(), self.yn, self.yn_size, self.ry, self.post)
        return g, z
