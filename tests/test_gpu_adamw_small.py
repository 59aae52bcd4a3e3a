"""AdamW on gradients whose squares are subnormal numbers."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from train_util import F64, U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beta1,beta2,step", [(0.0, 0.0, 1), (0.9, 0.999, 1), (0.5, 0.5, 3)])
@pytest.mark.parametrize("eps", [1e-30, 1e-21, 1e-15, 1e-8])
def test_step(eps, beta1, beta2, step):
    gen = torch.Generator().manual_seed(1)
    n = 4000
    g = torch.randn(n, generator=gen) * 10.0 ** (torch.rand(n, generator=gen) * 10 - 25)  # 1e-25 to 1e-15: squares of 0, subnormal and normal
    g[::50] = 0.0
    p, m, v = (torch.zeros(n, device="cuda") for _ in range(3))
    B.slicegcn_adamw_step(B.AdamList([p], [g.cuda()], [m], [v]), 1.0, step, beta1=beta1, beta2=beta2, eps=eps)
    o1, o2 = (torch.tensor(1 - b, dtype=torch.float32) for b in (beta1, beta2))
    m32, v32 = g * o1, (g * g) * o2
    assert torch.equal(m.cpu(), m32) and torch.equal(v.cpu(), v32)
    # from the states: t = v / c2, which is rounded to a multiple of 2^-149 where it is subnormal
    t = v32.to(F64) / (1 - beta2 ** step)
    update = lambda t: (m32.to(F64) / (1 - beta1 ** step)) / (torch.sqrt(t) + eps)
    want, ends = update(t), [update((t + d).clamp(min=0)) for d in (-2.0 ** -149, 2.0 ** -149)]
    # 16 roundings as for other numbers (square root and reciprocal are good to one place, eps and the corrections are rounded)
    tol = 16 * U * torch.stack([e.abs() for e in (want, *ends)]).amax(0) + (torch.stack([(e - want).abs() for e in ends]).amax(0) if step > 1 or beta2 else 0)
    assert ((-p.cpu().to(F64) - want).abs() <= tol + 2.0 ** -149).all()


def test_zeros_stay_with_the_smallest_eps():
    p, g, m, v = (torch.zeros(100, device="cuda") for _ in range(4))
    g[1] = 1.0
    B.slicegcn_adamw_step(B.AdamList([p], [g], [m], [v]), 1.0, 1, eps=2.0 ** -126)
    assert p[0] == 0 and abs(float(p[1]) + 1) < 16 * U and (p[2:] == 0).all()
