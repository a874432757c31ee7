"""Linear attention with a decay for each head on the GPU against the row-by-row evaluation in 64 bits (mixer_ref.py)."""
import numpy as np
import pytest
import torch

import mixer_ref as R
import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, F32 = cngp.F16, cngp.F32
NP = {F16: np.float16, F32: np.float32}


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def host(t):
    return t.cpu().numpy().astype(np.float64)


def make(N, S, H, K, dk, dv, io, rows, seed, slow=False):
    g = np.random.default_rng(seed)
    decay = -np.log1p(np.exp(g.normal(size=(N, H) if rows else (H,)) * 1.5 - (7 if slow else 3)))
    if rows:
        decay[g.random((N, H)) < 0.01] = -np.inf
        decay[g.random((N, H)) < 0.01] = -200.0
        decay[g.random((N, H)) < 0.02] = 0.0
    return dict(q=g.normal(size=(N, H, dk)).astype(NP[io]), k=g.normal(size=(N, K, dk)).astype(NP[io]), v=g.normal(size=(N, K, dv)).astype(NP[io]),
                decay=decay.astype(np.float32), h0=g.normal(size=(S, H, dk, dv)).astype(np.float32), dy=g.normal(size=(N, H, dv)).astype(NP[io]),
                dlast=g.normal(size=(S, H, dk, dv)).astype(np.float32))


def check(lengths, H=2, K=1, dk=16, dv=16, io=F32, rows=True, h0=True, dy=True, dlast=True, lead=0, trail=0, uniform=False, longest=0, seed=1, slow=False,
          backward=True, scale=0.25):
    off = None if uniform else np.concatenate([[lead], lead + np.cumsum(lengths)]).astype(np.int32)
    S, N = len(lengths), lead + int(np.sum(lengths)) + trail
    d = make(N, S, H, K, dk, dv, io, rows, seed, slow)
    inside = np.zeros(N, bool)
    sp = R.spans(N, S, off)
    for lo, hi in sp:
        inside[lo:hi] = True
    for n in ("q", "k", "v", "dy") + (("decay",) if rows else ()):        # rows of no sequence: not used, whatever they hold
        d[n][~inside] = np.nan
    cfg = cngp.AttendConfig(H, K, dk, dv, io, longest, scale, cngp.ATTEND_ROW_DECAY if rows else 0)
    f = {n: np.where(np.isfinite(t) | (n == "decay"), t, 0).astype(np.float64) for n, t in d.items()}
    f["decay"] = np.where(np.isnan(f["decay"]), 0, f["decay"])
    g = f["decay"] if rows else np.broadcast_to(f["decay"], (N, H))
    args = (f["q"], f["k"], f["v"], g, sp, f["h0"] if h0 else None, float(np.float32(scale)), f["dy"] if dy else None, f["dlast"] if dlast else None)
    want, bound = R.attend(*args), R.attend_bounds(*args)
    t = {n: dev(a) for n, a in d.items()}
    where = dict(h0=t["h0"] if h0 else None, offsets=dev(off), sequences=S)
    seven = lambda *shape: torch.full(shape, 7.0, dtype=t["q"].dtype, device=DEV)
    y, last = cngp.attend_fwd(cfg, t["q"], t["k"], t["v"], t["decay"], y=seven(N, H, dv), **where)
    R.within("y", host(y)[inside], want["y"][inside], bound["y"][inside], NP[io])
    R.within("last", host(last), want["last"], bound["last"])
    none, only = cngp.attend_fwd(cfg, t["q"], t["k"], t["v"], t["decay"], y=False, **where)
    assert none is None and (N == S and uniform or torch.equal(only, last))
    written = [("y", y)]
    if backward:
        ws = torch.full((max(cngp.attend_workspace_bytes(cfg, N, S, True, off is not None), 256),), 255, dtype=torch.uint8, device=DEV)
        call = lambda **kw: cngp.attend_bwd(cfg, t["q"], t["k"], t["v"], t["decay"], dy=t["dy"] if dy else None, dlast=t["dlast"] if dlast else None,
                                            workspace=ws, **where, **kw)
        dd = torch.full(d["decay"].shape, 7.0, device=DEV)
        dq, dk_, dv_, dd, dh0 = call(dq=seven(N, H, dk), dk=seven(N, K, dk), dv=seven(N, K, dv), ddecay=dd, dh0=torch.full(d["h0"].shape, 7.0, device=DEV))
        for name, got, key in (("dq", dq, "dq"), ("dk", dk_, "dk"), ("dv", dv_, "dv")):
            R.within(name, host(got)[inside], want[key][inside], bound[key][inside], NP[io])
        R.within("dh0", host(dh0), want["dh0"], bound["dh0"])
        if rows:
            R.within("ddecay", host(dd)[inside], want["dg"][inside], bound["dg"][inside])
        else:
            R.within("ddecay", host(dd), want["dg"].sum(0), bound["dg"].sum(0) + R.U * np.abs(want["dg"]).sum(0))
        again = call(ddecay=False, dh0=False)
        assert again[3] is None and again[4] is None
        for a, b in zip(again[:3], (dq, dk_, dv_)):
            assert torch.equal(a[torch.from_numpy(inside).to(DEV)], b[torch.from_numpy(inside).to(DEV)])
        written += [("dq", dq), ("dk", dk_), ("dv", dv_)] + ([("ddecay", dd)] if rows else [])
    for name, a in written:
        assert bool((a[torch.from_numpy(~inside).to(DEV)] == 7.0).all()), f"{name}: a row of no sequence was written"


RAGGED = [5, 0, 1, 64, 0, 63, 65, 130, 2, 0, 17]


@pytest.mark.parametrize("dk,dv", [(1, 1), (3, 5), (8, 8), (16, 16), (17, 40), (32, 33), (33, 32), (64, 64), (20, 100), (100, 12), (72, 48), (128, 128), (65, 127)])
@pytest.mark.parametrize("io", [F16, F32])
def test_dimensions_and_types(dk, dv, io):
    check(RAGGED, dk=dk, dv=dv, io=io, seed=dk + dv)


@pytest.mark.parametrize("H,K", [(1, 1), (3, 3), (4, 2), (6, 1), (9, 3)])
@pytest.mark.parametrize("io", [F16, F32])
@pytest.mark.parametrize("rows", [True, False])
def test_heads(H, K, io, rows):
    check(RAGGED, H=H, K=K, dk=24, dv=16, io=io, rows=rows, seed=H)


@pytest.mark.parametrize("kw", [dict(h0=False), dict(dy=False), dict(dlast=False), dict(h0=False, dlast=False), dict(lead=3, trail=5), dict(lead=100, trail=300),
                                dict(longest=130), dict(longest=1), dict(longest=2**31 - 1), dict(scale=0.0), dict(scale=-3.0)])
@pytest.mark.parametrize("io,rows", [(F16, True), (F32, False)])
def test_what_may_be_left_out(kw, io, rows):
    check(RAGGED, io=io, rows=rows, **kw)


@pytest.mark.parametrize("lengths,uniform", [([1], True), ([1] * 70, True), ([1] * 70, False), ([0, 0, 0], False), ([0], True), ([64] * 5, True), ([63] * 3, True),
                                             ([65] * 3, True), ([128, 128], True), ([1500], True), ([3, 1400, 0, 2], False), ([300] * 4, True)])
@pytest.mark.parametrize("io,rows", [(F16, True), (F32, False)])
def test_lengths(lengths, uniform, io, rows):
    check(lengths, io=io, rows=rows, uniform=uniform, slow=len(lengths) < 5)


@pytest.mark.parametrize("io", [F16, F32])
@pytest.mark.parametrize("rows", [True, False])
def test_long_sequences_are_cut_and_anchored(io, rows):
    """Rows enough for segments and for states kept on the way, in a sequence that starts off a boundary of either."""
    check([37, 4300, 11, 1100], H=2, K=1, dk=8, dv=12, io=io, rows=rows, slow=True, lead=5, longest=4300)
    check([4300], H=1, K=1, dk=40, dv=8, io=io, rows=rows, uniform=True)


@pytest.mark.parametrize("rows", [True, False])
def test_many_rows_before_the_first_sequence(rows):
    """More of them than a segment, or a stretch of the decays' gradient, has: their pieces belong to no sequence."""
    check([1500, 2600, 7], H=1, K=1, dk=8, dv=8, rows=rows, slow=True, lead=2900, longest=2600)
    check([1500, 2600, 7], H=2, K=1, dk=8, dv=8, rows=rows, slow=True, lead=2900, longest=600)       # ... of sequences that are longer than said


@pytest.mark.parametrize("sharp", [0.0, 0.3, 3.0])
@pytest.mark.parametrize("io", [F16, F32])
def test_decays_mild_and_sharp(io, sharp):
    """Chunks whose decay stays within 2^+-6 go by two factors to a pair, others by one exponential: both, and growth, against the same recurrence."""
    N, H, D = 200, 2, 32
    d = make(N, 1, H, H, D, D, io, True, 13)
    d["decay"] = np.where(np.arange(N)[:, None] % 3 == 0, -sharp, 0.25 * min(sharp, 0.3)).astype(np.float32) + np.zeros((N, H), np.float32)
    f = {n: a.astype(np.float64) for n, a in d.items()}
    args = (f["q"], f["k"], f["v"], f["decay"], [(0, N)], f["h0"], 0.2, f["dy"], f["dlast"])
    args = args[:6] + (float(np.float32(0.2)),) + args[7:]
    want, bound = R.attend(*args), R.attend_bounds(*args)
    cfg = cngp.AttendConfig(H, H, D, D, io, scale=0.2, flags=cngp.ATTEND_ROW_DECAY)
    t = {n: dev(a) for n, a in d.items()}
    y, last = cngp.attend_fwd(cfg, t["q"], t["k"], t["v"], t["decay"], h0=t["h0"])
    back = cngp.attend_bwd(cfg, t["q"], t["k"], t["v"], t["decay"], dy=t["dy"], dlast=t["dlast"], h0=t["h0"])
    R.within("y", host(y), want["y"], bound["y"], NP[io])
    R.within("last", host(last), want["last"], bound["last"])
    for name, got, key in zip(("dq", "dk", "dv", "ddecay", "dh0"), back, ("dq", "dk", "dv", "dg", "dh0")):
        R.within(name, host(got), want[key], bound[key], NP[io] if name in ("dq", "dk", "dv") else np.float32)


@pytest.mark.parametrize("D", [12, 40, 128])
@pytest.mark.parametrize("io", [F16, F32])
def test_gradients_of_sharp_decays(io, D):
    """Decays of e^-12: the gradient is what the rows before give, 10^-5 of the row's own product with itself, which must not enter its sums.  Bounds as
    in attend_bounds, with the magnitudes of q.dq and k.dk without that product."""
    N, H = 150, 2
    d = make(N, 1, H, H, D, D, io, True, 21)
    d["decay"][:] = -12.0
    f = {n: a.astype(np.float64) for n, a in d.items()}
    want = R.attend(f["q"], f["k"], f["v"], f["decay"], [(0, N)], None, 1.0, f["dy"])
    a = {n: np.abs(t) for n, t in f.items()}
    m = R.attend(a["q"], a["k"], a["v"], f["decay"], [(0, N)], None, 1.0, a["dy"])
    own = (a["q"] * a["k"]).sum(2) * (a["v"] * a["dy"]).sum(2)
    near = (a["q"] * m["dq"]).sum(2) + (a["k"] * m["dk"]).sum(2) - 2 * own
    bound = np.broadcast_to(R.rounds(D, D, N) * R.U * 3 * (m["dg"].max(0) + near.sum(0)), (N, H))
    cfg = cngp.AttendConfig(H, H, D, D, io, flags=cngp.ATTEND_ROW_DECAY)
    t = {n: dev(x) for n, x in d.items()}
    got = cngp.attend_bwd(cfg, t["q"], t["k"], t["v"], t["decay"], dy=t["dy"])
    R.within("ddecay", host(got[3]), want["dg"], bound)


def test_state_updated_in_place():
    for N, S, H, D in ((6, 6, 3, 20), (640, 2, 2, 64), (2600, 1, 1, 16)):
        d = make(N, S, H, H, D, D, F32, True, 5)
        t = {n: dev(a) for n, a in d.items()}
        cfg = cngp.AttendConfig(H, H, D, D, flags=cngp.ATTEND_ROW_DECAY)
        y, last = cngp.attend_fwd(cfg, t["q"], t["k"], t["v"], t["decay"], h0=t["h0"], sequences=S)
        state = t["h0"].clone()
        y2, same = cngp.attend_fwd(cfg, t["q"], t["k"], t["v"], t["decay"], h0=state, last=state, sequences=S)
        assert same is state and torch.equal(state, last) and torch.equal(y, y2)


@pytest.mark.parametrize("io", [F16, F32])
def test_a_prompt_and_then_token_by_token(io):
    """The states of a prompt taken on by single tokens give what the whole sequence gives at once."""
    S, T, H, K, D = 3, 70, 4, 2, 32
    d = make(S * (T + 5), S, H, K, D, D, io, True, 9)
    t = {n: dev(a) for n, a in d.items()}
    cfg = cngp.AttendConfig(H, K, D, D, io, scale=0.2, flags=cngp.ATTEND_ROW_DECAY)
    whole, last = cngp.attend_fwd(cfg, t["q"], t["k"], t["v"], t["decay"], h0=t["h0"], sequences=S)
    parts = lambda a, lo, hi: a.view(S, T + 5, *a.shape[1:])[:, lo:hi].reshape(-1, *a.shape[1:]).contiguous()
    inputs = lambda lo, hi: [parts(t[n], lo, hi) for n in ("q", "k", "v", "decay")]
    state = t["h0"].clone()
    got = [cngp.attend_fwd(cfg, *inputs(0, T), h0=state, last=state, sequences=S)[0].view(S, T, H, D)]
    for i in range(5):
        got.append(cngp.attend_fwd(cfg, *inputs(T + i, T + i + 1), h0=state, last=state, sequences=S)[0].view(S, 1, H, D))
    f = {n: a.astype(np.float64) for n, a in d.items()}
    b = R.attend_bounds(f["q"], f["k"], f["v"], f["decay"], R.spans(S * (T + 5), S, None), f["h0"], float(np.float32(0.2)))
    w = R.attend(f["q"], f["k"], f["v"], f["decay"], R.spans(S * (T + 5), S, None), f["h0"], float(np.float32(0.2)))
    R.within("tokens", host(torch.cat(got, 1)).reshape(w["y"].shape), w["y"], b["y"], NP[io])
    R.within("state", host(state), w["last"], b["last"])
    R.within("whole", host(whole), w["y"], b["y"], NP[io])


def test_values_of_all_magnitudes_in_fp16():
    """Scores, states and decayed values outside fp16's range, or in its subnormal part, are kept by scaled halves."""
    for size_q, size_k, size_v, size_h in ((40.0, 60.0, 1.0, 1e6), (1e-3, 1e-4, 1e-3, 1e-9), (1.0, 1e-5, 100.0, 0.0)):
        N, H, D = 150, 2, 48
        d = make(N, 1, H, H, D, D, F16, False, 3)
        for n, z in (("q", size_q), ("k", size_k), ("v", size_v)):
            d[n] = (d[n].astype(np.float64) * z).astype(np.float16)
        d["h0"] = (d["h0"] * size_h).astype(np.float32)
        f = {n: a.astype(np.float64) for n, a in d.items()}
        args = (f["q"], f["k"], f["v"], np.broadcast_to(f["decay"], (N, H)), [(0, N)], f["h0"], 1.0)
        want, bound = R.attend(*args), R.attend_bounds(*args)
        cfg = cngp.AttendConfig(H, H, D, D, F16)
        y, last = cngp.attend_fwd(cfg, *(dev(d[n]) for n in ("q", "k", "v", "decay")), h0=dev(d["h0"]))
        fits = np.abs(want["y"]) < 6e4
        # what is small against the largest score or state of a 32 x 32 tile keeps 2^-46 of that one
        R.within("y", host(y)[fits], want["y"][fits], bound["y"][fits] + 2.0 ** -36 * bound["y"].max() / R.U * 2.0 ** -8, np.float16)
        R.within("last", host(last), want["last"], bound["last"] + 2.0 ** -40 * np.abs(want["last"]).max())


def test_not_finite_stays_in_its_sequence_and_heads():
    N, S, H, K, D = 200, 2, 4, 2, 16
    for io in (F16, F32):
        d = make(N, S, H, K, D, D, io, True, 4)
        cfg = cngp.AttendConfig(H, K, D, D, io, flags=cngp.ATTEND_ROW_DECAY)
        run = lambda e: cngp.attend_fwd(cfg, *(dev(e[n]) for n in ("q", "k", "v", "decay")), h0=dev(e["h0"]), sequences=S)
        clean, _ = run(d)
        for n, at in (("v", (130, 1, 3)), ("k", (130, 1, 3)), ("decay", (130, 3)), ("q", (130, 3, 2))):
            e = {m: a.copy() for m, a in d.items()}
            e[n][at] = np.nan
            y, _ = run(e)
            assert torch.equal(y[:100], clean[:100]) and torch.equal(y[:, :2], clean[:, :2])
            assert bool(torch.isnan(y[130, 3]).any())
            assert torch.equal(y[100:100], clean[100:100])


def test_same_bits_again_and_workspaces_of_any_content():
    d = make(3000, 3, 4, 2, 48, 32, F16, False, 8)
    t = {n: dev(a) for n, a in d.items()}
    cfg = cngp.AttendConfig(4, 2, 48, 32, F16)
    need = cngp.attend_workspace_bytes(cfg, 3000, 3, True)
    ref = None
    for fill in (0, 255, 63):
        ws = torch.full((need,), fill, dtype=torch.uint8, device=DEV)
        got = cngp.attend_bwd(cfg, t["q"], t["k"], t["v"], t["decay"], dy=t["dy"], dlast=t["dlast"], h0=t["h0"], sequences=3, workspace=ws)
        assert ref is None or all(torch.equal(a, b) for a, b in zip(got, ref))
        ref = got


@pytest.mark.parametrize("io", [F16, F32])
def test_off_alignment(io):
    """Arrays that start off a 16-byte boundary, rows that no vector divides."""
    N, H, K, dk, dv = 130, 2, 1, 32, 16
    d = make(N, 1, H, K, dk, dv, io, True, 6)
    cfg = cngp.AttendConfig(H, K, dk, dv, io, flags=cngp.ATTEND_ROW_DECAY)

    def shifted(a):
        t = dev(a)
        room = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
        room[1:].copy_(t.view(-1))
        return room[1:].view(t.shape)

    call = lambda f: cngp.attend_fwd(cfg, *(f(d[n]) for n in ("q", "k", "v", "decay")), h0=f(d["h0"]), y=f(np.zeros((N, H, dv), NP[io])), last=f(np.zeros((1, H, dk, dv), np.float32)))
    assert all(torch.equal(a, b) for a, b in zip(call(dev), call(shifted)))
    back = lambda f: cngp.attend_bwd(cfg, *(f(d[n]) for n in ("q", "k", "v", "decay")), dy=f(d["dy"]), dlast=f(d["dlast"]), h0=f(d["h0"]), dq=f(np.zeros((N, H, dk), NP[io])),
                                     dk=f(np.zeros((N, K, dk), NP[io])), dv=f(np.zeros((N, K, dv), NP[io])))
    assert all(torch.equal(a, b) for a, b in zip(back(dev), back(shifted)))


def test_gradients_against_differences():
    """fp32, central differences of the library's own forward: the loss is quadratic at most in what is moved, so a difference has no error but rounding."""
    N, H, D = 70, 2, 8
    d = make(N, 1, H, H, D, D, F32, False, 12)
    t = {n: dev(a) for n, a in d.items()}
    cfg = cngp.AttendConfig(H, H, D, D, scale=0.3)
    loss = lambda u: sum(((a.double() * b.double()).sum() for a, b in zip(cngp.attend_fwd(cfg, u["q"], u["k"], u["v"], u["decay"], h0=u["h0"]), (t["dy"], t["dlast"]))))
    grads = dict(zip(("q", "k", "v", "decay", "h0"), cngp.attend_bwd(cfg, t["q"], t["k"], t["v"], t["decay"], dy=t["dy"], dlast=t["dlast"], h0=t["h0"])))
    scale = float(loss({n: a.abs() if n != "decay" else a for n, a in t.items()}).abs()) + 1.0
    r = torch.Generator(device=DEV).manual_seed(0)
    for n, g in grads.items():
        move = torch.randn(g.shape, generator=r, device=DEV)
        step = 0.125 if n != "decay" else 2.0 ** -9
        up, down = dict(t), dict(t)
        up[n], down[n] = t[n] + step * move, t[n] - step * move
        diff = float((loss(up) - loss(down)) / (2 * step))
        want = float((g.double() * move.double()).sum())
        # a loss of magnitude `scale` is off by 400 roundings at most, and the decays' third derivative enters with step^2 (|d^3| <= 64^3 losses)
        mags = float((g.double().abs() * move.double().abs()).sum())
        assert abs(diff - want) <= 400 * R.U * scale / step + 1e-3 * mags + (step ** 2 * 64 ** 2 * mags if n == "decay" else 0.0), (n, diff, want)
