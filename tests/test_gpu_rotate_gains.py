"""Gradients of gains that a rotation without norms does not use are zero: added to what is there, or written."""
import pytest
import torch

import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("N", [0, 5])
def test_gains_without_norms(N):
    D = 24
    x = lambda h: torch.ones(N, h, D, device=DEV)
    args = (torch.ones(N, 1, device=DEV), torch.ones(4, device=DEV), x(2), x(1), torch.ones(D, device=DEV), torch.ones(D, device=DEV))
    for flags, left in ((cngp.ZERO_GRADS, 0.0), (0, 7.0)):
        into = [torch.full((D,), 7.0, device=DEV) for _ in range(2)]
        got = cngp.rotate_bwd(cngp.RotateConfig(2, 1, D, (4,), flags=flags), None, None, *args, dgamma_q=into[0], dgamma_k=into[1])
        for given, out in zip(into, got[2:]):
            assert out is given and bool((out == left).all())
