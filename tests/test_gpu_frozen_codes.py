"""Codes that do not train collect no gradient, whatever they are added to."""
import pytest
import torch

import paper_2312_17241_amd as cngp
from paper_2312_17241_amd.module import Codes

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_frozen_codes_added_to_encodings_that_train():
    codes = Codes(5, 6, scale=2.0)
    ids = torch.tensor([4, 0, 4, 7, -2, 4], device=DEV)
    base = torch.randn(6, 6, device=DEV, requires_grad=True)
    codes.requires_grad_(False)
    y = codes(ids, base)
    y.sum().backward()
    assert bool((base.grad == 1).all()) and bool((codes.grad_table == 0).all())
    codes.requires_grad_(True)
    codes(ids, base).sum().backward()
    want = torch.zeros(5, 6)
    want[4], want[0] = 6.0, 2.0
    assert torch.equal(codes.grad_table.cpu(), want) and bool((base.grad == 2).all())
    # frozen between forward and backward: what the forward pass recorded counts, as with any parameter
    y = codes(ids, base)
    codes.requires_grad_(False)
    y.sum().backward()
    assert torch.equal(codes.grad_table.cpu(), 2 * want)
    table = codes.table.clone()
    codes.grad_table.zero_()
    codes(ids, base).sum().backward()
    codes.step(cngp.Adam(lr=1e-2))
    assert torch.equal(codes.table, table)


def test_only_the_codes_train():
    codes = Codes(5, 6)
    ids = torch.tensor([1, 1, 3], device=DEV)
    base = torch.randn(3, 6, device=DEV)
    codes(ids, base).sum().backward()
    want = torch.zeros(5, 6)
    want[1], want[3] = 2.0, 1.0
    assert torch.equal(codes.grad_table.cpu(), want) and base.grad is None
