"""The gates' gradient of the recurrence in fp16 is a product with the states in 32 bits, not with those that the caller kept in fp16.

Tolerances: those of recur_ref.py without a rounding of the states.  Where the kernel completes the kept states by what their rounding took
off, a state is off by two more roundings of fp32 (inside the eight that the bound counts per row) and 2^-39.  With gradients of the states
below 64 and at most 130 channels to a sum that adds 2^-26, half of the half step of the smallest fp16 number that every comparison
allows; it is written beside the bound where gradients are larger."""
import numpy as np
import pytest
import torch

import paper_2312_17241_amd as cngp
import recur_ref as R
from paper_2312_17241_amd.module import recur

pytestmark = pytest.mark.gpu
DEV = "cuda"
REV, LOG, MIX = cngp.RECUR_REVERSE, cngp.RECUR_LOG_GATE, cngp.RECUR_MIX
F16 = cngp.F16


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def host(t):
    return t.detach().cpu().numpy().astype(np.float64)


def inputs(C, G, N, S, flags, seed, size=1.0):
    g = np.random.default_rng(seed)
    gate = -np.abs(g.normal(size=(N, G))) * 0.4 if flags & LOG else 1 / (1 + np.exp(-g.normal(size=(N, G)) - 2))
    x, h0 = g.normal(size=(N, C)) * size, g.normal(size=(S, C)) * size
    return (gate.astype(np.float16), x.astype(np.float16), h0.astype(np.float32), g.normal(size=(N, C)).astype(np.float16),
            g.normal(size=(S, C)).astype(np.float32))


def check(C, shared, lengths, flags, uniform=False, lead=0, seed=1):
    G, S, N = 1 if shared else C, len(lengths), lead + int(sum(lengths))
    off = None if uniform else np.concatenate([[lead], lead + np.cumsum(lengths)]).astype(np.int32)
    gate, x, h0, dy, dlast = inputs(C, G, N, S, flags, seed)
    cfg = cngp.RecurConfig(C, G, F16, F16, 0, flags)
    where = dict(h0=dev(h0), offsets=dev(off), sequences=S)
    y, _ = cngp.recur_fwd(cfg, dev(gate), dev(x), **where)
    sp = R.spans(N, S, off)
    ref = R.backward(gate.astype(np.float64), x.astype(np.float64), sp, h0.astype(np.float64), dy.astype(np.float64), dlast.astype(np.float64),
                     bool(flags & REV), bool(flags & LOG), bool(flags & MIX), 0.0)
    got = []
    for fill in (7.0, float("nan")):       # what the outputs held before does not matter
        dgate, dx = torch.full((N, G), fill, dtype=torch.float16, device=DEV), torch.full((N, C), fill, dtype=torch.float16, device=DEV)
        got.append(cngp.recur_bwd(cfg, dev(gate), dev(x), dy=dev(dy), dlast=dev(dlast), y=y, dgate=dgate, dx=dx, **where))
    inside = np.zeros(N, bool)
    for lo, hi in sp:
        inside[lo:hi] = True
    rows = torch.from_numpy(inside).to(DEV)
    assert all(torch.equal(a[rows] if a.shape[0] == N else a, b[rows] if b.shape[0] == N else b) for a, b in zip(*got))
    R.within("dgate", host(got[0][0])[inside], ref["dgate"][inside], ref["Eg"][inside], np.float16)
    R.within("dx", host(got[0][1])[inside], ref["dx"][inside], ref["Ex"][inside], np.float16)
    R.within("dh0", host(got[0][2]), ref["dh0"], ref["E0"])
    assert bool((got[0][1][~rows] == 7.0).all()) and bool((got[0][0][~rows] == 7.0).all())


@pytest.mark.parametrize("flags", [0, REV, LOG, REV | LOG | MIX, MIX])
@pytest.mark.parametrize("C,shared", [(1, True), (3, True), (4, False), (6, False), (16, False), (33, True), (66, False), (130, True)])
def test_gradient_of_fp16_gates(C, shared, flags):
    check(C, shared, [5, 0, 1, 64, 0, 63, 65, 130, 2, 0, 0, 17], flags, lead=3)
    check(C, shared, [40] * 12, flags, uniform=True)


@pytest.mark.parametrize("C,shared,lengths,uniform", [(64, False, [900] * 192, True), (32, False, [1] * 70, True), (8, True, [1] * 70, True),
                                                      (40, False, [9000, 3, 0, 5000], False), (3, True, [30000], True), (96, True, [6000], True),
                                                      (20, False, [300, 200, 2000, 1, 700] * 20, False)])
@pytest.mark.parametrize("flags", [0, REV | LOG | MIX])
def test_whole_long_sequences_cut_ones_and_single_rows(C, shared, lengths, uniform, flags):
    check(C, shared, lengths, flags, uniform)


def test_under_autograd_with_the_states_kept():
    gate, x, h0, dy, dlast = inputs(24, 24, 600, 3, 0, 2)
    leaves = [dev(a).requires_grad_() for a in (gate, x, h0)]
    y, last = recur(cngp.RecurConfig(24, 24, F16, F16), *leaves, sequences=3)
    torch.autograd.backward([y, last], [dev(dy), dev(dlast)])
    ref = R.backward(*(a.astype(np.float64) for a in (gate, x)), R.spans(600, 3, None), *(a.astype(np.float64) for a in (h0, dy, dlast)), False, False,
                     False, 0.0)
    R.within("dgate", host(leaves[0].grad), ref["dgate"], ref["Eg"], np.float16)


@pytest.mark.parametrize("size", [2.0 ** -12, 2.0 ** -19])
def test_states_that_fp16_holds_badly(size):
    """Below 2^-14 fp16 has fewer and fewer bits, below 2^-25 none."""
    C, S, N = 12, 5, 500
    gate, x, h0, dy, dlast = inputs(C, C, N, S, 0, 3, size)
    dy = (dy.astype(np.float64) * 512).astype(np.float16)
    cfg = cngp.RecurConfig(C, C, F16, F16)
    y, _ = cngp.recur_fwd(cfg, dev(gate), dev(x), h0=dev(h0), sequences=S)
    dgate, _, _ = cngp.recur_bwd(cfg, dev(gate), dev(x), dy=dev(dy), h0=dev(h0), y=y, sequences=S)
    ref = R.backward(*(a.astype(np.float64) for a in (gate, x)), R.spans(N, S, None), *(a.astype(np.float64) for a in (h0, dy)), None, False, False,
                     False, 0.0)
    R.within("dgate", host(dgate), ref["dgate"], ref["Eg"] + 2.0 ** -39 * np.abs(ref["dx"]) * 1.001, np.float16)


def test_states_beyond_fp16_and_not_finite_ones():
    """A state above 65504 is infinite in y; the gradient has it with eight bits.  One that is not finite stays in its sequence and channel."""
    C, lengths = 16, [10, 30, 7]
    off = dev(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32))
    cfg = cngp.RecurConfig(C, C, F16, F16)
    gate, x = torch.ones(47, C, dtype=torch.float16, device=DEV), torch.zeros(47, C, dtype=torch.float16, device=DEV)
    x[10], x[11], x[0] = 60000.0, 30000.0, 3.0
    dlast = torch.full((3, C), 2.0 ** -4, device=DEV)
    y, _ = cngp.recur_fwd(cfg, gate, x, offsets=off)
    assert bool(torch.isinf(y[11:40]).all())
    good = cngp.recur_bwd(cfg, gate, x, dlast=dlast, y=y, offsets=off)
    assert bool(((good[0][12:40] - 90000.0 * 2.0 ** -4).abs() <= 90000.0 * 2.0 ** -4 * (2.0 ** -7 + 2.0 ** -11)).all())
    assert bool((good[0][11] == 60000.0 * 2.0 ** -4).all()) and bool((good[0][1:10] == 3.0 * 2.0 ** -4).all())
    x[12, 5] = float("nan")
    y, _ = cngp.recur_fwd(cfg, gate, x, offsets=off)
    bad = cngp.recur_bwd(cfg, gate, x, dlast=dlast, y=y, offsets=off)
    keep = torch.ones(47, C, dtype=torch.bool, device=DEV)
    keep[13:40, 5] = False
    assert torch.equal(bad[0][keep], good[0][keep]) and bool(torch.isnan(bad[0][13:40, 5]).all()) and torch.equal(bad[1], good[1])


@pytest.mark.parametrize("C,shared,lengths", [(64, False, [900] * 192), (12, True, [40, 0, 700, 3]), (3, True, [40, 0, 700, 3]), (40, False, [9000, 3])])
def test_graph_replays_and_another_stream(C, shared, lengths):
    G, S, N = 1 if shared else C, len(lengths), sum(lengths)
    gate, x, h0, dy, dlast = (dev(a) for a in inputs(C, G, N, S, 0, 4))
    off = None if len(set(lengths)) == 1 else dev(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32))
    cfg = cngp.RecurConfig(C, G, F16, F16)
    y, dgate, dx, dh0 = torch.empty_like(x), torch.empty_like(gate), torch.empty_like(x), torch.empty_like(h0)
    last, size = torch.empty_like(h0), max(cngp.recur_workspace_bytes(cfg, N, S, b, off is not None, True) for b in (False, True))
    ws = torch.empty(max(size, 256), dtype=torch.uint8, device=DEV)

    def step():
        cngp.recur_fwd(cfg, gate, x, h0=h0, offsets=off, sequences=S, y=y, last=last, workspace=ws)
        cngp.recur_bwd(cfg, gate, x, dy=dy, dlast=dlast, h0=h0, y=y, offsets=off, sequences=S, dgate=dgate, dx=dx, dh0=dh0, workspace=ws)

    outs = [y, last, dgate, dx, dh0]
    step()
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for o in outs:
            o.fill_(float("nan"))
        ws.fill_(255)
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(o, w) for o, w in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for o in outs:
            o.fill_(float("nan"))
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
        step()


@pytest.mark.parametrize("C,shared", [(3, True), (24, False)])
def test_cut_sequences_far_behind_rows_of_no_sequence(C, shared):
    check(C, shared, [20000, 0, 7, 9000], REV | LOG | MIX, lead=12000)
    check(C, shared, [20000, 0, 7, 9000], 0, lead=12000)
