"""Orthogonalised updates of matrices whose norm lies outside fp32, or whose norm's inverse does: entries at both ends of fp32's range.

Tolerance: against the same matrix of a middle size.  A power of two apart, its normalised entries are the same numbers but for the rounding of one
product each (2^-24 of an entry); that noise is lifted as any other error of the input, by 3.4445 a step (test_gpu_ortho.py), and norms bound entries:
the normalised matrix has norm 1."""
import numpy as np
import pytest
import torch

import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("m,n", [(1, 1), (32, 64), (100, 64), (64, 128), (200, 130), (300, 700)])
@pytest.mark.parametrize("power", [-146, -130, 100, 122])
@pytest.mark.parametrize("steps", [0, 1, 5])
def test_entries_at_the_ends_of_the_range(m, n, power, steps):
    g = np.random.default_rng(m + n)
    # whole numbers up to 8 in magnitude: exact at every power, the smallest of them subnormal numbers
    whole = g.integers(-8, 9, size=(2, m, n)).astype(np.float64)
    whole[0, 0, 0] = whole[1, 0, 0] = 8
    cfg = cngp.OrthoConfig(m, n, 2, steps=steps, eps=0.0)
    run = lambda p: cngp.orthogonalise(cfg, torch.from_numpy((whole * 2.0 ** p).astype(np.float32)).to(DEV)).double().cpu()
    got, want = run(power), run(0)
    assert bool(torch.isfinite(got).all())
    assert float((got - want).abs().max()) <= 2 * 2.0 ** -24 * 3.4445 ** steps


@pytest.mark.parametrize("m,n", [(32, 64), (200, 130)])
def test_optimiser_step_of_gradients_at_the_ends_of_the_range(m, n):
    g = np.random.default_rng(m)
    whole = torch.from_numpy(g.integers(-8, 9, size=(m, n)).astype(np.float32)).to(DEV)
    cfg, opt = cngp.OrthoConfig(m, n, eps=0.0), cngp.Muon(1.0, 0.0, nesterov=False)
    moved = []
    for power in (0, -146, 122):
        w, mom, grad = torch.zeros_like(whole), torch.zeros_like(whole), (whole.double() * 2.0 ** power).float()
        cngp.muon_step(cfg, opt, w, None, mom, grad)
        moved.append(w.double().cpu())
    for w in moved[1:]:
        assert bool(torch.isfinite(w).all()) and float((w - moved[0]).abs().max()) <= 2 * 2.0 ** -24 * 3.4445 ** 5
