"""AdamW with its steps counted on the device, without a GPU: refusals before any device work."""
import pytest
import torch

from paper_2408_11500_amd import binding as B
from test_abi_host import L  # noqa: F401  (a fixture)
from test_block_host import ONE, adam


def test_refusals(L):  # noqa: F811
    ok = dict(t=adam(count=0), count=1, states=32, lr=0.1, b1=0.9, b2=0.999, eps=1e-8, counter=ONE)
    run = lambda **kw: L.slicegcn_adamw_step_counted(*{**ok, **kw}.values(), None, 0, None)
    for kw in (dict(counter=None), dict(counter=ONE + 2), dict(t=None), dict(count=-1), dict(states=16), dict(lr=float("nan")), dict(b1=1.0), dict(b2=-1.0), dict(eps=0.0),
               dict(t=adam(param=None)), dict(t=adam(m=ONE + 2))):
        assert run(**kw) == B.EINVAL, kw


def test_the_binding_refuses_counters_that_do_not_fit():
    tensors = B.AdamList([], [], [], [])
    with pytest.raises(ValueError):
        B.slicegcn_adamw_step_counted(tensors, 0.1, torch.zeros(1, dtype=torch.int32))
    with pytest.raises(TypeError):
        B.slicegcn_adamw_step_counted(tensors, 0.1, torch.zeros(4, dtype=torch.int32))  # on the host


def test_eps_that_has_no_reciprocal_in_fp32_is_refused(L):  # noqa: F811
    for eps in (1e-40, 1e-38, 2.0 ** -127):
        assert L.slicegcn_adamw_step(adam(count=0), 1, 32, 0.1, 0.9, 0.999, eps, 1, None, 0, None) == B.EINVAL
        assert L.slicegcn_adamw_step_counted(adam(count=0), 1, 32, 0.1, 0.9, 0.999, eps, ONE, None, 0, None) == B.EINVAL
    assert L.slicegcn_adamw_step(adam(count=0), 1, 32, 0.1, 0.9, 0.999, 2.0 ** -126, 1, None, 0, None) == 0
