"""fp32 columns of very different magnitudes in linear attention: what the two fp16 numbers of an operand hold.

Two parts to the bound, each six times the root of the sum of squares of independent errors (the recurrences over squares, mixer_ref.attend, give those sums):
    roundings of what is rounded: the count of decay_ref.py, times 2^-24 of each product;
    what is small beside the largest value that shares its power of two: that one is at least 2^13 as an operand, where the smallest fp16 number is 2^-24, so a value is off by
    2^-38 of the largest, evenly spread (a root of 3 less).  Six operands take part in a result: q, k, v, the scores, the state, what is added to it.  The largest of all
    rows and columns without decays stands for each.
Columns stay within 10^-11 of the largest here; below 10^-8 the second part is all there is."""
import numpy as np
import pytest
import torch

import mixer_ref as R
import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dk,dv", [(16, 16), (32, 32), (20, 50), (64, 64), (128, 128)])
@pytest.mark.parametrize("uneven", ["q", "k", "v", "dy", "all"])
def test_columns_of_all_magnitudes(dk, dv, uneven):
    N, H = 150, 2
    g = np.random.default_rng(dk + dv)
    held = lambda t: t.astype(np.float32).astype(np.float64)
    value = lambda *s: g.choice((-1.0, 1.0), s) * (0.5 + 0.5 * g.random(s))
    d = dict(q=value(N, H, dk), k=value(N, H, dk), v=value(N, H, dv), dy=value(N, H, dv))
    for n in d:
        if uneven in (n, "all"):
            d[n] = d[n] * 10.0 ** -(np.arange(d[n].shape[2]) % 12)
        d[n] = held(d[n])
    decay, h0, dlast = held(-0.1 * g.random((N, H))), held(value(1, H, dk, dv)), held(value(1, H, dk, dv))
    scale, spans = 0.25, [(0, N)]
    want = R.attend(d["q"], d["k"], d["v"], decay, spans, h0, scale, d["dy"], dlast)
    sq = lambda t: t * t
    top = lambda t: np.full(t.shape, np.abs(t).max() ** 2)
    seen = R.attend(sq(d["q"]), sq(d["k"]), sq(d["v"]), 2 * decay, spans, sq(h0), scale ** 2, sq(d["dy"]), sq(dlast))
    most = R.attend(top(d["q"]), top(d["k"]), top(d["v"]), 0 * decay, spans, top(h0), scale ** 2, top(d["dy"]), top(dlast))
    rounds = 24 + (dk + dv + 64) / 4 + 6 * (N // 64 + 1) + 64
    bound = {n: 6 * R.U * np.sqrt(rounds * seen[n]) + 6 * 2.0 ** -38 * np.sqrt(6 / 3 * most[n]) for n in want}
    cfg = cngp.AttendConfig(H, H, dk, dv, cngp.F32, scale=scale, flags=cngp.ATTEND_ROW_DECAY)
    to = lambda t: torch.from_numpy(t.astype(np.float32)).to(DEV)
    t = {n: to(a) for n, a in dict(d, decay=decay, h0=h0, dlast=dlast).items()}
    y, last = cngp.attend_fwd(cfg, t["q"], t["k"], t["v"], t["decay"], h0=t["h0"])
    dq, dk_, dv_, _, dh0 = cngp.attend_bwd(cfg, t["q"], t["k"], t["v"], t["decay"], dy=t["dy"], dlast=t["dlast"], h0=t["h0"])
    for n, got in (("y", y), ("last", last), ("dq", dq), ("dk", dk_), ("dv", dv_), ("dh0", dh0)):
        R.within(n, got.cpu().numpy(), want[n], bound[n])


@pytest.mark.parametrize("D", [16, 128])
def test_a_token_to_each_sequence_keeps_all_columns(D):
    """N == sequences: fp32 products as they are; a product, a sum and D additions to an entry."""
    N, H = 40, 2
    g = np.random.default_rng(D)
    held = lambda t: t.astype(np.float32).astype(np.float64)
    q, k, v = (held(g.normal(size=(N, H, D)) * 10.0 ** -(np.arange(D) % 12)) for _ in range(3))
    decay, h0 = held(-g.random((N, H))), held(g.normal(size=(N, H, D, D)) * 10.0 ** -(np.arange(D) % 12))
    spans = R.spans(N, N, None)
    args, mags = (q, k, v, decay, spans, h0, 1.0), (abs(q), abs(k), abs(v), decay, spans, abs(h0), 1.0)
    want, mag = R.attend(*args), R.attend(*mags)
    cfg = cngp.AttendConfig(H, H, D, D, cngp.F32, flags=cngp.ATTEND_ROW_DECAY)
    to = lambda t: torch.from_numpy(t.astype(np.float32)).to(DEV)
    y, last = cngp.attend_fwd(cfg, to(q), to(k), to(v), to(decay), h0=to(h0), sequences=N)
    R.within("last", last.cpu().numpy(), want["last"], 8 * R.U * mag["last"])
    R.within("y", y.cpu().numpy(), want["y"], (D + 12) * R.U * mag["y"])
