"""Calls of more values than one launch has work-items for (2^32 lanes)."""
import pytest
import torch

import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(autouse=True)
def give_back():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def parts(n, each=1 << 15):
    return [slice(i, min(i + each, n)) for i in range(0, n, each)]


def test_one_row_each_of_more_than_2_to_34_values():
    N, C = 2**20 + 3, 2**14
    cfg = cngp.RecurConfig(C, 1, cngp.F16, cngp.F16)
    gate = torch.rand((N, 1), device=DEV).half()
    x = torch.empty((N, C), dtype=torch.float16, device=DEV)
    columns = torch.arange(C, device=DEV) % 97
    for p in parts(N):
        x[p] = (torch.arange(p.start, p.stop, device=DEV)[:, None] % 1009 + columns).half()
    y, _ = cngp.recur_fwd(cfg, gate, x, sequences=N, last=False)
    for p in parts(N):
        assert torch.equal(y[p], x[p]), p


def test_lookup_of_more_than_2_to_24_wide_rows():
    N, dim = 2**24 + 5, 2052
    cfg = cngp.EmbedConfig(7, dim, cngp.F32, cngp.F16, cngp.I32)
    table = torch.arange(7, device=DEV)[:, None] * 100.0 + torch.arange(dim, device=DEV) % 89
    ids = (torch.arange(N, device=DEV) % 9 - 1).int()                # two of nine are padding
    y = cngp.embed_fwd(cfg, ids, table)
    half = torch.cat([table, torch.zeros(2, dim, device=DEV)]).half()
    rows = torch.where((ids >= 0) & (ids < 7), ids, 7).long()
    for p in parts(N, 1 << 20):
        assert torch.equal(y[p], half[rows[p]]), p
    assert cngp.embed_fwd(cfg, ids, table, base=y, y=y) is y
    for p in parts(N, 1 << 20):
        assert torch.equal(y[p], 2 * half[rows[p]]), p


def test_states_without_rows_of_more_than_2_to_32_values():
    S, C = 2**21 + 1, 2049
    cfg = cngp.RecurConfig(C, C)
    none = torch.empty((0, C), device=DEV)
    last = torch.full((S, C), 7.0, device=DEV)
    cngp.recur_fwd(cfg, none, none, sequences=S, y=False, last=last)
    assert all(bool((last[p] == 0).all()) for p in parts(S, 1 << 18))
    for p in parts(S, 1 << 18):
        last[p] = torch.arange(p.start, p.stop, device=DEV)[:, None].float()
    _, _, dh0 = cngp.recur_bwd(cfg, none, none, dlast=last, sequences=S, dh0=True)
    assert all(torch.equal(dh0[p], last[p]) for p in parts(S, 1 << 18))
