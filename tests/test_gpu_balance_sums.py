"""The loss of levels of very many rows: the sums of the softmax weights do not drift with their number.

Tolerance, u = 2^-24: N_p + 6 for a softmax weight, at most 64 + 6 + 4 + 24 additions of 32 bits on the way to a level's sum whatever the
number of rows, N_p + 4 for the loss: below 140 of them for N_p <= 16."""
import pytest
import torch

import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("N_p,top_k,log_rows", [(8, 5, 27), (16, 11, 26), (4, 3, 24), (4, 3, 17), (2, 0, 28)])
def test_equal_rows(N_p, top_k, log_rows):
    cfg = cngp.Config(d=3, L=1, F=2, N_f=2**10, N_c=2**log_rows, N_p=N_p, N_min=4, N_max=64, top_k=top_k)
    row = torch.zeros(N_p) if top_k else torch.tensor([0.0, -1.25])
    v = row.to(DEV).expand(1, 2**log_rows, N_p).contiguous()
    loss, counts, _ = cngp.probe_balance(cfg, v, grad_Dhat_c=None)
    assert counts[0].tolist() == [2**log_rows] + [0] * (N_p - 1)
    kept = row.double()[: top_k or N_p]
    want = N_p * float(kept.softmax(0)[0])                             # every row's winner is the first
    assert abs(float(loss[0]) - want) <= 140 * 2.0 ** -24 * want
