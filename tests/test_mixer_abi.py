"""What the operators of the token mixer refuse, on the host: every check runs before anything is launched, so none of it needs a GPU."""
import ctypes

import numpy as np
import pytest
import torch

import mixer_ref as R
import paper_2312_17241_amd as cngp

lib = cngp._lib
P, P2 = ctypes.c_void_p(4096), ctypes.c_void_p(8192)          # aligned addresses that no refused call follows
OFF = ctypes.c_void_p(4100)
BIG = 1 << 50


def attend(**over):
    kw = dict(heads=4, kv_heads=2, key_dim=16, value_dim=24)
    kw.update(over)
    return cngp.AttendConfig(**kw)


def fwd(cfg, q=P, k=P, v=P, decay=P, N=6, offsets=None, S=3, h0=P, y=P, last=P, ws=P, size=BIG):
    return lib.cngp_attend_fwd(None if cfg is None else cfg._ref(), q, k, v, decay, N, offsets, S, h0, y, last, ws, size, None)


def bwd(cfg, q=P, k=P, v=P, decay=P, N=6, offsets=None, S=3, h0=P, dy=P, dlast=P, dq=P, dk=P, dv=P, dd=P, dh0=P2, ws=P, size=BIG):
    return lib.cngp_attend_bwd(None if cfg is None else cfg._ref(), q, k, v, decay, N, offsets, S, h0, dy, dlast, dq, dk, dv, dd, dh0, ws, size, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_attention_refuses(call):
    assert call(None) == cngp.ERR_NULL
    for over in (dict(heads=0), dict(heads=4097, kv_heads=1), dict(kv_heads=0), dict(kv_heads=3), dict(kv_heads=8), dict(key_dim=0), dict(key_dim=129), dict(value_dim=0),
                 dict(value_dim=129), dict(io_dtype=2), dict(longest=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(flags=2)):
        assert call(attend(**over)) == cngp.ERR_INVALID, over
        assert cngp.attend_workspace_bytes(attend(**over), 6, 3, True) == 0
    for kw in (dict(N=-1), dict(N=2**31), dict(S=-1), dict(S=2**31 - 1, N=2**31 - 2), dict(S=4), dict(S=0)):
        assert call(attend(), **kw) == cngp.ERR_INVALID, kw
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(decay=None)):
        assert call(attend(), **kw) == cngp.ERR_NULL, kw
    assert fwd(attend(), S=0, N=0) == cngp.OK and fwd(attend(), S=0, offsets=P) == cngp.OK        # no sequences: nothing to write
    assert bwd(attend(), S=0, N=0, dd=None) == cngp.OK


def test_attention_refuses_missing_outputs_and_workspaces():
    assert fwd(attend(), y=None, last=None) == cngp.ERR_NULL
    assert fwd(attend(), N=3, q=None, y=None) == cngp.ERR_NULL                                       # one row each, shared keys
    for kw in (dict(dy=None, dlast=None), dict(dq=None), dict(dk=None), dict(dv=None)):
        assert bwd(attend(), **kw) == cngp.ERR_NULL, kw
    assert bwd(attend(), dh0=P) == cngp.ERR_INVALID                                                  # dh0 is dlast
    need = cngp.attend_workspace_bytes(attend(), 6, 3, True)
    for kw in (dict(ws=None), dict(ws=OFF), dict(size=need - 1)):
        assert bwd(attend(), **kw) == cngp.ERR_WORKSPACE, kw
    long = cngp.attend_workspace_bytes(attend(), 100000, 1)
    assert long > 0
    for kw in (dict(ws=None), dict(ws=OFF), dict(size=long - 1)):
        assert fwd(attend(), N=100000, S=1, **kw) == cngp.ERR_WORKSPACE, kw


def test_attention_workspaces():
    for N, S in ((1, 1), (64, 64), (4096, 1), (2**17, 2**17), (2**20, 4), (20011, 1)):
        for cfg in (attend(), attend(flags=cngp.ATTEND_ROW_DECAY), attend(kv_heads=4), attend(key_dim=128, value_dim=100, io_dtype=cngp.F16)):
            for ragged in (False, True):
                a, b = cngp.attend_workspace_bytes(cfg, N, S, False, ragged), cngp.attend_workspace_bytes(cfg, N, S, True, ragged)
                assert a % 256 == 0 and b % 256 == 0 and b >= a
    assert cngp.attend_workspace_bytes(attend(), 2**18, 4096) == 0                                   # sequences enough: none is cut


def test_pieces_of_sequences_have_places_of_their_own():
    """Piece numbers begin / R + s + i and anchor slots begin / R + i (i >= 1), as the kernels form them, never meet and stay in their room."""
    g = np.random.default_rng(0)
    for R in (64, 256, 1024):
        for _ in range(40):
            S = int(g.integers(1, 40))
            lengths = np.where(g.random(S) < 0.3, g.integers(0, 3, S), g.integers(0, 5 * R, S))
            off = np.concatenate([[int(g.integers(0, 3 * R))], lengths]).cumsum()
            N = int(off[-1]) + int(g.integers(0, 100))
            pieces = [off[s] // R + s + i for s in range(S) for i in range(-(-int(lengths[s]) // R))]
            slots = [off[s] // R + i for s in range(S) for i in range(1, -(-int(lengths[s]) // R))]
            assert len(set(pieces)) == len(pieces) and all(0 <= p < N // R + S for p in pieces)
            assert len(set(slots)) == len(slots) and all(1 <= p < N // R + 1 for p in slots)
            bases = [off[s] // R + s for s in range(S)]
            for s in range(S):
                for i in range(-(-int(lengths[s]) // R)):
                    assert max(t for t in range(S) if bases[t] <= bases[s] + i) == s


def rotate(**over):
    kw = dict(heads=4, kv_heads=2, dim=16, pairs=(4, 4))
    kw.update(over)
    return cngp.RotateConfig(**kw)


def turn(cfg, q=P, k=P, N=5, position=P, omega=P, gq=P, gk=P, qo=P, ko=P):
    return lib.cngp_rotate_fwd(None if cfg is None else cfg._ref(), q, k, N, position, omega, gq, gk, qo, ko, None)


def turn_bwd(cfg, q=P, k=P, N=5, position=P, omega=P, gq=P, gk=P, qo=P, ko=P, dq=P, dk=P, dgq=P, dgk=P, ws=P, size=BIG):
    return lib.cngp_rotate_bwd(None if cfg is None else cfg._ref(), q, k, N, position, omega, gq, gk, qo, ko, dq, dk, dgq, dgk, ws, size, None)


@pytest.mark.parametrize("call", [turn, turn_bwd])
def test_rotation_refuses(call):
    assert call(None) == cngp.ERR_NULL
    for over in (dict(heads=-1), dict(heads=4097), dict(kv_heads=-1), dict(heads=0, kv_heads=0), dict(dim=0), dict(dim=513, pairs=(0,)), dict(pairs=(9,)), dict(pairs=(-1, 4)),
                 dict(pairs=(4, 4, 1)), dict(io_dtype=2), dict(eps=-1.0), dict(eps=float("nan")), dict(flags=8)):
        assert call(rotate(**over)) == cngp.ERR_INVALID, over
    for kw in (dict(N=-1), dict(N=2**31)):
        assert call(rotate(), **kw) == cngp.ERR_INVALID, kw
    for kw in (dict(qo=None), dict(ko=None), dict(position=None), dict(omega=None)):
        assert call(rotate(), **kw) == cngp.ERR_NULL, kw
    assert turn(rotate(), N=0) == cngp.OK and turn_bwd(rotate(), N=0) == cngp.OK
    with pytest.raises(ValueError):
        rotate(pairs=(1, 1, 1, 1, 1)).c()


def test_rotation_refuses_missing_arrays_and_workspaces():
    normed = rotate(flags=cngp.ROTATE_NORM)
    assert turn(rotate(), q=None) == cngp.ERR_NULL and turn(rotate(), k=None) == cngp.ERR_NULL
    assert turn_bwd(normed, q=None) == cngp.ERR_NULL and turn_bwd(normed, k=None) == cngp.ERR_NULL
    assert turn_bwd(rotate(), dq=None) == cngp.ERR_NULL and turn_bwd(rotate(), dk=None) == cngp.ERR_NULL
    need = cngp.rotate_workspace_bytes(normed, 5)
    assert need > 0 and need % 256 == 0 and cngp.rotate_workspace_bytes(rotate(), 5) == 0
    for kw in (dict(ws=None), dict(ws=OFF), dict(size=need - 1)):
        assert turn_bwd(normed, **kw) == cngp.ERR_WORKSPACE, kw


def ortho(**over):
    kw = dict(rows=200, cols=300)
    kw.update(over)
    return cngp.OrthoConfig(**kw)


def test_orthogonalising_refuses():
    call = lambda cfg, g=P, out=P, ws=P, size=BIG: lib.cngp_orthogonalise(None if cfg is None else cfg._ref(), g, out, ws, size, None)
    assert call(None) == cngp.ERR_NULL and call(ortho(), g=None) == cngp.ERR_NULL and call(ortho(), out=None) == cngp.ERR_NULL
    for over in (dict(rows=0), dict(rows=16385), dict(cols=0), dict(cols=16385), dict(batch=0), dict(batch=65536), dict(io_dtype=2), dict(steps=-1), dict(steps=33), dict(eps=-1.0),
                 dict(eps=float("inf")), dict(coefficients=(17.0, 0.0, 0.0)), dict(coefficients=(1.0, float("nan"), 0.0))):
        assert call(ortho(**over)) == cngp.ERR_INVALID, over
        assert cngp.orthogonalise_workspace_bytes(ortho(**over)) == 0
    need = cngp.orthogonalise_workspace_bytes(ortho())
    assert need > 0 and need % 256 == 0
    for kw in (dict(ws=None), dict(ws=OFF), dict(size=need - 1)):
        assert call(ortho(), **kw) == cngp.ERR_WORKSPACE, kw


def test_optimiser_step_refuses():
    def call(cfg=ortho(), opt=cngp.Muon(), w=P, m=P, g=P, ws=P, size=BIG):
        o = None if opt is None else ctypes.byref(opt.c())
        return lib.cngp_muon_step(None if cfg is None else cfg._ref(), o, w, None, m, g, 0, ws, size, None)
    for kw in (dict(cfg=None), dict(opt=None), dict(w=None), dict(m=None), dict(g=None)):
        assert call(**kw) == cngp.ERR_NULL, kw
    assert call(cfg=ortho(io_dtype=cngp.F16)) == cngp.ERR_UNSUPPORTED
    assert call(cfg=ortho(rows=0)) == cngp.ERR_INVALID
    for kw in (dict(lr=-1.0), dict(lr=float("inf")), dict(lr=float("nan")), dict(momentum=1.0), dict(momentum=-0.1), dict(weight_decay=-1.0), dict(grad_scale=float("inf")),
               dict(nesterov=2)):
        assert call(opt=cngp.Muon(**kw)) == cngp.ERR_INVALID, kw
    need = cngp.orthogonalise_workspace_bytes(ortho())
    for kw in (dict(ws=None), dict(ws=OFF), dict(size=need - 1)):
        assert call(**kw) == cngp.ERR_WORKSPACE, kw


def test_modules_refuse_gradients_that_they_do_not_give():
    from paper_2312_17241_amd.module import rotate as turned
    x = torch.zeros(6, 4, 16)
    for position, omega in ((torch.zeros(6, 2, requires_grad=True), torch.zeros(8)), (torch.zeros(6, 2), torch.zeros(8, requires_grad=True))):
        with pytest.raises(ValueError):
            turned(rotate(), x, torch.zeros(6, 2, 16), position, omega)


def test_binding_refuses_wrong_tensors():
    x = torch.zeros(6, 4, 16)
    with pytest.raises(TypeError):
        cngp.attend_fwd(attend(), x, torch.zeros(6, 2, 16), torch.zeros(6, 2, 24), torch.zeros(4))        # host tensors
    with pytest.raises(ValueError):
        cngp.attend_fwd(attend(), x, torch.zeros(6, 2, 16), torch.zeros(6, 2, 24), torch.zeros(4), offsets=torch.zeros(3, dtype=torch.int32), sequences=5)
    with pytest.raises(TypeError):
        cngp.rotate_fwd(rotate(), x, torch.zeros(6, 2, 16), torch.zeros(6, 2), torch.zeros(8))
    with pytest.raises(TypeError):
        cngp.orthogonalise(ortho(), torch.zeros(1, 200, 300))


def test_reference_gradients_against_differences():
    g = np.random.default_rng(1)
    N, H, K, dk, dv, S = 9, 2, 1, 3, 4, 2
    sp = [(0, 5), (5, 9)]
    d = dict(q=g.normal(size=(N, H, dk)), k=g.normal(size=(N, K, dk)), v=g.normal(size=(N, K, dv)), g=-g.random((N, H)), h0=g.normal(size=(S, H, dk, dv)))
    dy, dl = g.normal(size=(N, H, dv)), g.normal(size=(S, H, dk, dv))
    run = lambda e, **kw: R.attend(e["q"], e["k"], e["v"], e["g"], sp, e["h0"], 0.7, **kw)
    loss = lambda e: (lambda r: (r["y"] * dy).sum() + (r["last"] * dl).sum())(run(e))
    grads = run(d, dy=dy, dlast=dl)
    for n, key in (("q", "dq"), ("k", "dk"), ("v", "dv"), ("g", "dg"), ("h0", "dh0")):
        move = g.normal(size=d[n].shape)
        up, down = dict(d), dict(d)
        up[n], down[n] = d[n] + 1e-5 * move, d[n] - 1e-5 * move
        assert abs((loss(up) - loss(down)) / 2e-5 - (grads[key] * move).sum()) < 1e-6
    x, du, gamma, angle = g.normal(size=(3, 2, 8)), g.normal(size=(3, 2, 8)), g.normal(size=8), g.normal(size=(3, 3))
    for nxt in (False, True):
        f = lambda x, gamma: (R.rotate(x, angle, nxt, gamma, 1e-3, True)[0] * du).sum()
        _, dx, dg = R.rotate(x, angle, nxt, gamma, 1e-3, True, du)
        mx, mg = g.normal(size=x.shape), g.normal(size=8)
        assert abs((f(x + 1e-5 * mx, gamma) - f(x - 1e-5 * mx, gamma)) / 2e-5 - (dx * mx).sum()) < 1e-6
        assert abs((f(x, gamma + 1e-5 * mg) - f(x, gamma - 1e-5 * mg)) / 2e-5 - (dg * mg).sum()) < 1e-6
