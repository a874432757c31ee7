"""Orthogonalised updates on the GPU to what operands of 22 bits allow, on matrices that show every part of every product (ortho_parts.py); test_ortho_bounds.py
shows on the host that a part left out is far outside."""
import pytest
import torch

import ortho_parts as O
import paper_2312_17241_amd as cngp
from test_ortho_bounds import SHAPES

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("batch,m,n", SHAPES)
@pytest.mark.parametrize("steps", [1, 2])
def test_all_parts_of_all_products(batch, m, n, steps):
    G = O.matrices(batch, m, n, 5)
    out = cngp.orthogonalise(cngp.OrthoConfig(m, n, batch, steps=steps, eps=0.0), torch.from_numpy(G).to(DEV)).cpu().numpy()
    for i in {0, batch // 2, batch - 1}:
        assert O.off_by(O.wide(out[i]), O.exact(O.wide(G[i]), steps)) <= O.tolerance_of(m, n, steps), i
