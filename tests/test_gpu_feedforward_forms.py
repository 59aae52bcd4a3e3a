"""Feed-forward blocks that only answer, and such that keep their gradients before the activation in two terms."""
import pytest
import torch

from paper_2408_11500_amd.tokens import GatedFeedForward
from train_util import F64, TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("n,width,inner", [(1, 64, 176), (300, 72, 200)])
def test_without_training(n, width, inner, kind):
    dtype = TYPES[kind]
    gen = torch.Generator().manual_seed(4)
    ws = [(torch.randn(s, generator=gen) / s[0] ** 0.5).to(dtype).cuda() for s in ((width, inner), (width, inner), (inner, width))]
    x, u, dx = (torch.randn((n, width), generator=gen).to(dtype).cuda() for _ in range(3))
    learns, answers = GatedFeedForward(n, width, inner, dtype=dtype), GatedFeedForward(n, width, inner, dtype=dtype, training=False)
    for ff in (learns, answers):
        ff.set_params(*ws)
    assert torch.equal(learns.forward(x, u), answers.forward(x, u))
    size = lambda ff: sum(t.numel() for t in vars(ff).values() if torch.is_tensor(t) and t.dtype == dtype)
    assert size(answers) == 3 * width * inner + n * (inner + width) and size(learns) == 6 * width * inner + n * (4 * inner + 2 * width)
    assert answers.parameter_slots() == [] and len(learns.parameter_slots()) == 3
    learns.backward(u, dx)
    with pytest.raises(RuntimeError):
        answers.backward(u, dx)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_two_terms(kind):
    """Gradients of the gated projections against 64 bits from what the block holds: closer to them than with gradients that are rounded once."""
    dtype = TYPES[kind]
    n, width, inner = 1000, 136, 344
    gen = torch.Generator().manual_seed(5)
    ws = [(torch.randn(s, generator=gen) / s[0] ** 0.5).to(dtype).cuda() for s in ((width, inner), (width, inner), (inner, width))]
    x, u, dx = (torch.randn((n, width), generator=gen).to(dtype).cuda() for _ in range(3))
    errors = []
    for two in (False, True):
        ff = GatedFeedForward(n, width, inner, dtype=dtype, two_terms=two)
        ff.set_params(*ws)
        ff.forward(x, u)
        ff.backward(u, dx)
        g, up, dh, u64, wg, wu = (t.to(F64) for t in (ff.G, ff.U, ff.dH, u, ff.Wg, ff.Wu))
        s = torch.sigmoid(g)
        dg, du = dh * up * s * (1 + g * (1 - s)), dh * g * s
        want = dict(du=dg @ wg.t() + du @ wu.t(), dWg=u64.t() @ dg, dWu=u64.t() @ du)
        errors.append({k: float(torch.linalg.vector_norm(getattr(ff, k).to(F64) - w) / torch.linalg.vector_norm(w)) for k, w in want.items()})
    half = torch.finfo(dtype).eps / 2
    # one rounding of a result is at most half a step of each, so of the norm too; another one of what it is formed from is not left
    assert all(e < half for e in errors[1].values()) and all(errors[1][k] < errors[0][k] for k in errors[1]), errors
