"""Recurrences over more than 2^30 rows, in sequences that are cut into windows: gates of one and inputs of zero but for a few
rows of whole numbers, so that every state is a small whole number, which has to arrive through every cut unchanged, forward and backward."""
import pytest
import torch

import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"
MOST = 2**31 - 2**16


def pieces(lo, hi):
    return [slice(i, min(i + (1 << 28), hi)) for i in range(lo, hi, 1 << 28)]


@pytest.mark.parametrize("N,S,reverse,ragged", [(1_200_000_000, 1, False, False), (1_600_000_000, 2, False, False), (1_500_000_000, 3, True, False),
                                                (MOST, 1, True, False), (MOST, 2, False, False), (MOST, 2, True, True)])
def test_states_and_gradients_arrive(N, S, reverse, ragged):
    each = N // S
    offsets = torch.arange(S + 1, device=DEV, dtype=torch.int32) * each if ragged else None
    cfg = cngp.RecurConfig(1, 1, cngp.F16, cngp.F16, 0, cngp.RECUR_REVERSE if reverse else 0)
    gate, x = torch.ones((N, 1), dtype=torch.float16, device=DEV), torch.zeros((N, 1), dtype=torch.float16, device=DEV)
    steps = [each // 3, each // 2 + 5, each - 70_001]          # rows of each sequence, in the order of the memory, that add 1, 2 and 4
    for s in range(S):
        for i, r in enumerate(steps):
            x[s * each + r] = 2 ** i
    h0, dlast = torch.arange(1, S + 1, device=DEV).float()[:, None] * 8, torch.arange(1, S + 1, device=DEV).float()[:, None] * 0.5
    y, last = cngp.recur_fwd(cfg, gate, x, h0=h0, offsets=offsets, sequences=S)
    assert torch.equal(last, h0 + 7)
    dgate, dx, dh0 = cngp.recur_bwd(cfg, gate, x, dlast=dlast, h0=h0, y=y, offsets=offsets, sequences=S)
    assert torch.equal(dh0, dlast)
    for s in range(S):
        state, edges = float(h0[s]), [0] + steps + [each]
        order = range(3, -1, -1) if reverse else range(4)      # the stretches between those rows, in the order taken
        for n, i in enumerate(order):
            lo, hi = edges[i], edges[i + 1]
            if reverse:                    # a row that adds belongs to the stretch that follows it: here the one below it
                lo, hi = lo + (1 if i else 0), hi + (1 if i < 3 else 0)
            if n:
                state += 2 ** (i if reverse else i - 1)
            for part in pieces(s * each + lo, s * each + hi):
                assert bool((y[part] == state).all()), (s, i)
                # the state before a row, all but at the stretch's first row in the order taken
                inner = slice(part.start, part.stop - (1 if reverse and n and part.stop == s * each + hi else 0))
                inner = slice(inner.start + (1 if not reverse and n and part.start == s * each + lo else 0), inner.stop)
                assert bool((dgate[inner] == state * float(dlast[s])).all()), (s, i)
        for part in pieces(s * each, (s + 1) * each):
            assert bool((dx[part] == float(dlast[s])).all())


def test_wide_rows():
    N, C = 1_150_000_000, 5
    cfg = cngp.RecurConfig(C, 1, cngp.F16, cngp.F16)
    gate, x = torch.ones((N, 1), dtype=torch.float16, device=DEV), torch.zeros((N, C), dtype=torch.float16, device=DEV)
    x[N // 7], x[N - 3000] = 3, 5
    h0 = torch.arange(C, device=DEV).float()[None] + 0.25
    _, last = cngp.recur_fwd(cfg, gate, x, h0=h0, y=False)
    assert torch.equal(last, h0 + 8)
