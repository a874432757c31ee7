"""The gradient of linear attention's decays on the GPU, within what fp32 sums may be off by (decay_ref.py); test_decay_bounds.py shows on the host that
a state left out at one chunk's end is not within it."""
import numpy as np
import pytest
import torch

import decay_ref as D
import mixer_ref as R
import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, F32 = cngp.F16, cngp.F32


def check(lengths, H=2, K=1, dk=8, dv=12, io=F32, rows=True, slow=True, lead=0, trail=0, longest=0, uniform=False, h0=True, dlast=True, seed=1):
    q, k, v, decay, start, dy, behind, off = D.inputs(lengths, H, K, dk, dv, rows, seed, slow, io == F16, lead, trail)
    N, S = q.shape[0], len(lengths)
    args = (q, k, v, np.broadcast_to(decay, (N, H)), R.spans(N, S, off), start if h0 else None, 0.25, dy, behind if dlast else None)
    want = R.attend(*args)["dg"]
    row, total = D.bounds(*args)
    cfg = cngp.AttendConfig(H, K, dk, dv, io, longest, 0.25, cngp.ATTEND_ROW_DECAY if rows else 0)
    to = lambda t, dtype: torch.from_numpy(np.ascontiguousarray(t)).to(dtype).to(DEV)
    x = torch.float16 if io == F16 else torch.float32
    f = torch.float32
    grads = cngp.attend_bwd(cfg, to(q, x), to(k, x), to(v, x), to(decay, f), dy=to(dy, x), dlast=to(behind, f) if dlast else None, h0=to(start, f) if h0 else None,
                            offsets=None if uniform else torch.from_numpy(off).to(DEV), sequences=S, dh0=False if seed % 2 else None)
    got = grads[3].cpu().numpy()
    if rows:
        inside = slice(int(off[0]), int(off[-1]))
        R.within("ddecay", got[inside], want[inside], row[inside])
    else:
        R.within("ddecay", got, want.sum(0), total)


@pytest.mark.parametrize("io,rows", [(F16, True), (F32, True), (F16, False), (F32, False)])
@pytest.mark.parametrize("case", [dict(lengths=[37, 4300, 11, 1100], longest=4300, lead=5), dict(lengths=[2300], H=1, dk=40, dv=8, uniform=True),
                                  dict(lengths=[1100, 1100], K=2, slow=False, uniform=True), dict(lengths=[1500, 2600, 7], lead=2900, longest=600, seed=2),
                                  dict(lengths=[1025, 1024, 1023], h0=False), dict(lengths=[3000], H=1, dlast=False, dk=16, dv=16), dict(lengths=[3000], H=1, h0=False, dlast=False, seed=2),
                                  dict(lengths=[1300], H=1, dk=64, dv=64, trail=70), dict(lengths=[1200], H=1, dk=128, dv=100), dict(lengths=[2100], H=4, K=2, dk=24, dv=33)])
def test_long_sequences(case, io, rows):
    check(io=io, rows=rows, **case)


@pytest.mark.parametrize("io,rows", [(F16, True), (F32, True), (F16, False), (F32, False)])
@pytest.mark.parametrize("case", [dict(lengths=[5, 0, 1, 64, 0, 63, 65, 130, 2, 0, 17], lead=3, trail=4), dict(lengths=[300] * 4, uniform=True, longest=300),
                                  dict(lengths=[70, 5, 200], H=4, K=1, dk=16, dv=16, seed=2), dict(lengths=[130, 128], K=2, dk=128, dv=128), dict(lengths=[200], dk=33, dv=7, slow=False)])
def test_short_sequences(case, io, rows):
    check(io=io, rows=rows, **case)


@pytest.mark.parametrize("io", [F16, F32])
def test_sums_over_long_sequences_for_many_heads(io):
    """Sixteen heads with memories of 16 rows over 4096: the root of mean squares of their errors, for which the count of roundings stands without the six of one result's
    bound, and a rounding for u / sqrt(3)."""
    N, H, Dim = 4096, 16, 16
    q, k, v, _, h0, dy, dlast, _ = D.inputs([N], H, H, Dim, Dim, False, 5, False, io == F16)
    decay = np.full(H, np.log1p(-2.0 ** -4)).astype(np.float32).astype(np.float64)
    args = (q, k, v, np.broadcast_to(decay, (N, H)), [(0, N)], h0, 0.25, dy, dlast)
    want, (_, total) = R.attend(*args)["dg"].sum(0), D.bounds(*args)
    x = torch.float16 if io == F16 else torch.float32
    to = lambda t, dtype: torch.from_numpy(np.ascontiguousarray(t)).to(dtype).to(DEV)
    f = torch.float32
    got = cngp.attend_bwd(cngp.AttendConfig(H, H, Dim, Dim, io, scale=0.25), to(q, x), to(k, x), to(v, x), to(decay, f), dy=to(dy, x), dlast=to(dlast, f), h0=to(h0, f))[3]
    off = (got.cpu().numpy() - want) / total
    share = float(np.sqrt((off ** 2).mean()))
    assert share <= 1 / (6 * np.sqrt(3)), share
