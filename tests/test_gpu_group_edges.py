"""Groups of tensors: arguments that are not what they should be, infinite norms, tensors that are let go while the device still
works on them."""
import math

import pytest
import torch

from paper_2501_02379_amd import group, tgrad as T

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_scaling_needs_an_earlier_result():
    """None is no factor, and a result whose two numbers do not lie side by side is none; nothing is written."""
    g = [torch.randn(5000, device=DEV), torch.randn(70, device=DEV)]
    was = [t.clone() for t in g]
    grp = group.Group(g)
    apart = torch.ones(6, device=DEV)[2::2]
    assert apart.shape == (2,) and apart.storage_offset() == 2
    for bad in (lambda: grp.tgrad_group_scale(None), lambda: grp.tgrad_group_scale(apart), lambda: grp.tgrad_group_grad_norm(1.0, into=apart),
                lambda: grp.tgrad_group_clip(1.0, into=apart), lambda: grp.tgrad_group_clip(1.0, into=torch.ones(2, device=DEV))):
        with pytest.raises(T.TgradError):
            bad()
    assert all(torch.equal(a, b) for a, b in zip(g, was))
    grp.tgrad_group_scale(grp.tgrad_group_grad_norm(1.0))
    assert not torch.equal(g[0], was[0])
