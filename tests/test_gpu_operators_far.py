"""Arrays of more than 2^31 entries, and batches whose sequences are nearly all empty: the operators at the far ends of their ranges."""
import numpy as np
import pytest
import torch

import paper_2312_17241_amd as cngp
import recur_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


def host(t):
    return t.cpu().numpy().astype(np.float64)


@pytest.mark.parametrize("C,reverse", [(64, False), (3, True)])
def test_recurrence_over_more_than_2_to_31_entries(C, reverse):
    """One gate per row; a shut gate shortly before each end makes what follows it independent of the rest."""
    N = (2**31) // C + 1001
    flags = cngp.RECUR_REVERSE if reverse else 0
    cfg = cngp.RecurConfig(C, 1, cngp.F16, cngp.F16, 0, flags)
    g = torch.Generator(device=DEV).manual_seed(1)
    gate = torch.rand((N, 1), generator=g, device=DEV).half()
    x = torch.empty((N, C), dtype=torch.float16, device=DEV)
    for part in x.split(1 << 22):
        part.copy_(torch.randn(part.shape, generator=g, device=DEV))
    lo, hi = 700, N - 700
    gate[lo] = gate[hi] = 0
    y, last = cngp.recur_fwd(cfg, gate, x)
    dy_last = torch.randn((1, C), generator=g, device=DEV)
    dgate, dx, _ = cngp.recur_bwd(cfg, gate, x, dlast=dy_last, y=y)
    for rows, start in ((slice(0, lo + 1), lo), (slice(hi, N), hi)):
        ours = slice(0, lo + 1) if reverse else slice(hi, N)
        if rows != ours:
            continue
        a, v = host(gate[rows]), host(x[rows])
        ref = R.backward(a, v, [(0, a.shape[0])], None, None, host(dy_last), reverse, False, False, 2.0 ** -11)
        R.within("y", host(y[rows]), ref["y"], ref["Ey"], np.float16)
        R.within("last", host(last), ref["last"], ref["El"])
        inner = slice(0, lo) if reverse else slice(1, None)       # the shut gate's own gradient needs the row outside
        R.within("dx", host(dx[rows]), ref["dx"], ref["Ex"], np.float16)
        R.within("dgate", host(dgate[rows])[inner], ref["dgate"][inner], ref["Eg"][inner], np.float16)
    far = slice(hi, N) if reverse else slice(0, lo + 1)           # the other end gets no gradient through the shut gates
    assert bool((dx[far] == 0).all())


def test_lookup_in_a_table_of_more_than_2_to_31_entries():
    rows, dim = 2**25 + 3, 80
    cfg = cngp.EmbedConfig(rows, dim, cngp.F16, cngp.F32, cngp.I64, 2.0, cngp.ZERO_GRADS)
    table = torch.zeros((rows, dim), dtype=torch.float16, device=DEV)
    ids = torch.tensor([rows - 1, 5, rows - 2, rows - 1, 2**25, rows, -1, 2**31, 2**33 + 5], device=DEV)
    for i in (rows - 1, 5, rows - 2, 2**25):
        table[i] = torch.randn(dim, device=DEV)
    y = cngp.embed_fwd(cfg, ids, table)
    assert torch.equal(y[:5], 2.0 * table[ids[:5]].float()) and bool((y[5:] == 0).all())
    dy = torch.randn((9, dim), device=DEV)
    grad = cngp.embed_bwd(cfg, ids, dy)
    assert torch.equal(grad[rows - 1], 2.0 * (dy[0] + dy[3])) and torch.equal(grad[2**25], 2.0 * dy[4]) and torch.equal(grad[5], 2.0 * dy[1])
    assert int((grad != 0).any(1).sum()) == 4
    y = cngp.embed_fwd(cngp.EmbedConfig(7, 2**15, cngp.F16, cngp.F16, cngp.I32), torch.arange(70000, device=DEV, dtype=torch.int32) % 7,
                       torch.arange(7, device=DEV).half()[:, None].expand(7, 2**15).contiguous())
    assert bool((y[:, 17] == torch.arange(70000, device=DEV) % 7).all()) and bool((y[-1] == 69999 % 7).all())


def test_balance_of_more_than_2_to_31_logits():
    cfg = cngp.Config(d=3, L=9, F=2, N_f=2**10, N_c=2**24, N_p=16, N_min=4, N_max=64, flags=cngp.ZERO_GRADS)
    v = torch.empty((9, 2**24, 16), device=DEV)
    v.fill_(-1.0)
    v[8, :, 3] = 1.0
    v[8, ::2, 5] = 2.0
    loss, counts, grad = cngp.probe_balance(cfg, v, 1.0)
    assert counts[0].tolist() == [2**24] + [0] * 15 and counts[8].tolist() == [0, 0, 0, 2**23, 0, 2**23] + [0] * 10
    row = host(v[8, :2]).copy()
    sigma = np.exp(row) / np.exp(row).sum(1, keepdims=True)
    f = np.zeros(16)
    f[[3, 5]] = 0.5
    want = 16 / 2**24 * sigma * (f - (sigma * f).sum(1, keepdims=True))
    # every term is a softmax weight of one rounding of 16 sums: 32 u relative to its magnitude
    assert np.abs(host(grad[8, :2]) - want).max() <= 64 * 2.0 ** -24 * 16 / 2**24
    assert torch.equal(grad[8, 0], grad[8, -2]) and torch.equal(grad[8, 1], grad[8, -1])


@pytest.mark.parametrize("C,shared", [(3, True), (2, False), (12, True), (40, False)])
@pytest.mark.parametrize("spread", ["between", "in front", "behind", "all"])
def test_thousands_of_empty_sequences(C, shared, spread):
    g = np.random.default_rng(3)
    full = [0] if spread == "all" else [70, 3, 500, 1, 1, 260]
    empty = [0] * 3000
    lengths = {"between": sum(([n] + empty for n in full), []), "in front": empty + full, "behind": full + empty, "all": empty}[spread]
    S, N, G = len(lengths), sum(lengths), 1 if shared else C
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    gate, x = g.random((N, G)).astype(np.float32), g.normal(size=(N, C)).astype(np.float32)
    h0, dlast = g.normal(size=(S, C)).astype(np.float32), g.normal(size=(S, C)).astype(np.float32)
    dev = lambda a: torch.from_numpy(a).to(DEV)
    cfg = cngp.RecurConfig(C, G)
    where = dict(h0=dev(h0), offsets=dev(off))
    y, last = cngp.recur_fwd(cfg, dev(gate), dev(x), **where)
    dgate, dx, dh0 = cngp.recur_bwd(cfg, dev(gate), dev(x), dlast=dev(dlast), y=y if N else None, **where)
    ref = R.backward(gate.astype(np.float64), x.astype(np.float64), R.spans(N, S, off), h0, None, dlast.astype(np.float64), False, False, False)
    R.within("last", host(last), ref["last"], ref["El"])
    R.within("dh0", host(dh0), ref["dh0"], ref["E0"])
    if N:
        R.within("y", host(y), ref["y"], ref["Ey"])
        R.within("dx", host(dx), ref["dx"], ref["Ex"])
        R.within("dgate", host(dgate), ref["dgate"], ref["Eg"])
