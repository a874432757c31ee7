"""Orthogonalised updates of small matrices beside fp32 arithmetic: their sums are short, so that there is little rounding for that of the operands' parts to hide in.

Yardstick: the same five steps in fp32 on the host, their error against 64 bits over 48 matrices.  An operand in two parts is off by 2^-23 at most, twice a rounding of
fp32, one to a factor where fp32 rounds products and sums as often as there are terms, at least eight here: evaluated on the host with parts (ortho_parts.py's
with all four products, sums of low ones apart) the errors are 0.8 to 1.0 of the yardstick, with all products in one set of sums that cuts off 1.2 to 1.5.  1.4 allows for the
order of sums and for 48 matrices standing for all."""
import numpy as np
import pytest
import torch

import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
A, B, C = (float(np.float32(v)) for v in cngp.OrthoConfig(1, 1).coefficients)


def steps(x, dtype):
    wide = x.shape[1] <= x.shape[2]
    x = x.astype(np.float64) / np.linalg.norm(x.astype(np.float64), axis=(1, 2), keepdims=True)
    x = (x if wide else x.transpose(0, 2, 1)).astype(dtype)
    a, b, c = (dtype(v) for v in (A, B, C))
    for _ in range(5):
        gram = x @ x.transpose(0, 2, 1)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return (x if wide else x.transpose(0, 2, 1)).astype(np.float64)


@pytest.mark.parametrize("m,n", [(14, 84), (475, 9), (17, 58), (14, 178), (24, 61), (9, 331)])
def test_small_matrices_beside_fp32(m, n):
    r = np.random.default_rng(m)
    rank = max(1, min(m, n) // 8)
    g = ((r.normal(size=(48, m, rank)) @ r.normal(size=(48, rank, n)) / np.sqrt(rank) * 0.5 + r.normal(size=(48, m, n))) * 1e-2).astype(np.float32)
    want = steps(g, np.float64)
    off = lambda x: float(np.sqrt(((x - want) ** 2).mean()))
    got = cngp.orthogonalise(cngp.OrthoConfig(m, n, 48, eps=0.0), torch.from_numpy(g).cuda()).double().cpu().numpy()
    assert off(got) <= 1.4 * off(steps(g, np.float32)), (off(got), off(steps(g, np.float32)))
