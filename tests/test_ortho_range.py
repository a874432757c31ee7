"""The range into which five steps with the default coefficients bring singular values, as include/cngp.h states it: from 0.0016 of the norm on 0.68 .. 1.21,
0.001 to 0.47.  On the host from the polynomial, on the GPU from matrices of known singular values."""
import numpy as np
import pytest
import torch

import paper_2312_17241_amd as cngp


def after(s, steps=5):
    a, b, c = cngp.OrthoConfig(1, 1).coefficients
    for _ in range(steps):
        s = a * s + b * s ** 3 + c * s ** 5
    return s


def test_range_of_the_polynomial():
    s = after(np.concatenate([np.geomspace(0.0016, 1.0, 400001), np.linspace(0.0016, 1.0, 400001)]))
    assert 0.68 < s.min() < 0.69 and 1.20 < s.max() < 1.21
    assert abs(after(0.001) - 0.47) < 0.005 and after(0.0015) < 0.68


@pytest.mark.gpu
@pytest.mark.parametrize("m,n", [(60, 100), (200, 130)])
def test_range_on_the_gpu(m, n):
    """Singular values by the polynomial, to the 2e-3 that five steps may make of 2^-19 (each lifts an error by 3.4445 at most)."""
    r = np.random.default_rng(m)
    small = min(m, n)
    s = np.geomspace(0.0016, 1.0, small)
    s[-1] = np.sqrt(1.0 - (s[:-1] ** 2).sum()) if (s[:-1] ** 2).sum() < 1 else s[-1]
    s = s / np.linalg.norm(s)
    u, v = np.linalg.qr(r.normal(size=(m, small)))[0], np.linalg.qr(r.normal(size=(n, small)))[0]
    out = cngp.orthogonalise(cngp.OrthoConfig(m, n, eps=0.0), torch.from_numpy((u * s @ v.T)[None].astype(np.float32)).cuda())[0].double().cpu().numpy()
    got = (u.T @ out @ v).diagonal()
    assert np.abs(got - after(s)).max() < 2e-3
    assert (got[s >= 0.0016] > 0.68 - 2e-3).all() and got.max() < 1.21
