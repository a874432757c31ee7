"""A row of linear attention that is not finite: its sequence's earlier pieces of 64 rows, the other sequences and the heads that do not read it keep their bits."""
import numpy as np
import pytest
import torch

import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, F32 = cngp.F16, cngp.F32


def inputs(N, S, H, K, D, io, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.float16 if io == F16 else torch.float32
    r = lambda *s: torch.randn(s, generator=g)
    return dict(q=r(N, H, D).to(x), k=r(N, K, D).to(x), v=r(N, K, D).to(x), decay=-torch.rand(N, H, generator=g) * 0.2, h0=r(S, H, D, D), dy=r(N, H, D).to(x), dlast=r(S, H, D, D))


# two sequences of 100 rows, the row in the second one's second piece; three of 1300, cut into segments, the row in a later segment of the second
@pytest.mark.parametrize("D,each,S,bad", [(16, 100, 2, 170), (64, 100, 2, 170), (128, 100, 2, 170), (16, 1300, 3, 2300)])
@pytest.mark.parametrize("io", [F16, F32])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
def test_what_a_row_that_is_not_finite_leaves_alone(D, each, S, bad, io, value):
    H, K, N = 4, 2, each * S
    clean = inputs(N, S, H, K, D, io, D)
    cfg = cngp.AttendConfig(H, K, D, D, io, scale=0.2, flags=cngp.ATTEND_ROW_DECAY)
    first, piece = bad // each * each, bad // each * each + (bad % each) // 64 * 64
    others = [r for r in range(N) if not first <= r < first + each]

    def run(d):
        t = {n: a.to(DEV) for n, a in d.items()}
        where = dict(h0=t["h0"], sequences=S)
        y, last = cngp.attend_fwd(cfg, t["q"], t["k"], t["v"], t["decay"], **where)
        return [a.cpu() for a in (y, last) + cngp.attend_bwd(cfg, t["q"], t["k"], t["v"], t["decay"], dy=t["dy"], dlast=t["dlast"], **where)]

    want = run(clean)
    for name, head in (("q", 3), ("k", 1), ("v", 1), ("decay", 3), ("dy", 3)):
        if name == "decay" and value == float("-inf"):
            continue                                       # a decay like any other
        d = {n: a.clone() for n, a in clean.items()}
        if name == "decay":
            d[name][bad, head] = value
        else:
            d[name][bad, head, D // 2] = value
        got = run(d)
        y, last, dq, dk, dv, dd, dh0 = range(7)
        kv = head if name in ("k", "v") else head // 2        # the shared keys and values that the head reads, or that the row is of
        unread = [h for h in range(H) if h // 2 != kv] if name in ("k", "v") else [h for h in range(H) if h != head]
        same = lambda i, rows, heads=None: torch.equal(got[i][rows] if heads is None else got[i][rows][:, heads], want[i][rows] if heads is None else want[i][rows][:, heads])
        for i in (y, dq, dk, dv, dd):                         # other sequences
            assert same(i, others), (name, i)
        for i in (last, dh0):
            assert all(torch.equal(got[i][s], want[i][s]) for s in range(S) if s != bad // each), (name, i)
        for i in (y, dq, dd):                                 # heads that do not read it
            assert same(i, slice(None), unread), (name, i)
        for i in (last, dh0):
            assert same(i, slice(None), unread), (name, i)
        for i in (dk, dv):
            assert same(i, slice(None), [h for h in range(K) if h != kv]), (name, i)
        assert same(y, slice(first, piece)), name              # earlier pieces of the sequence
        if name in ("k", "v", "decay", "dy"):
            assert same(dq, slice(first, piece)), name
        read = [h for h in range(H) if h not in unread]
        if name == "dy":
            assert torch.equal(got[y], want[y]) and torch.equal(got[last], want[last])
            assert not bool(torch.isfinite(got[dq][bad, read]).all())
        else:
            assert not bool(torch.isfinite(got[y][bad, read]).all()), name
