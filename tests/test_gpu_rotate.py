"""Norms and rotation of queries and keys on the GPU against the same in 64 bits (mixer_ref.py).

Bounds: a component is a product of x, the inverse norm, gamma and a sine or cosine, two of them added: with u = 2^-24 the norm has dim / 2 + 6 roundings
(half of the sum's under the root), sine and cosine 4 u (angle after whole turns: 2^-24 of a turn, 2 pi u / 2, and two units for the functions), 6 for
the rest.  Backward: the mean of products adds dim + 8.  Everything times the largest components of the pair, bounded by the head's norm."""
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


def make(N, H, K, D, pairs, io, seed, far=0.0):
    g = np.random.default_rng(seed)
    position = (g.random((N, len(pairs))) * (2.0 if not far else far)).astype(np.float32)
    if far:
        position = np.floor(position)
    return dict(q=(g.normal(size=(N, H, D)) * 3).astype(NP[io]), k=g.normal(size=(N, K, D)).astype(NP[io]), position=position,
                omega=(10000.0 ** (-np.arange(sum(pairs)) / max(sum(pairs), 1))).astype(np.float32), gamma_q=(1 + 0.3 * g.normal(size=D)).astype(np.float32),
                gamma_k=(1 + 0.3 * g.normal(size=D)).astype(np.float32), dq=g.normal(size=(N, H, D)).astype(NP[io]), dk=g.normal(size=(N, K, D)).astype(NP[io]))


def check(N, H, K, D, pairs, io=F32, norm=True, nxt=False, gains=True, seed=1, far=0.0, eps=1e-6, shift=False, inplace=False):
    d = make(N, H, K, D, pairs, io, seed, far)
    flags = (cngp.ROTATE_NORM if norm else 0) | (cngp.ROTATE_NEXT if nxt else 0)
    cfg = cngp.RotateConfig(H, K, D, tuple(pairs), io, eps, flags)

    def put(a):
        t = dev(a)
        if not shift:
            return t
        room = torch.empty(t.numel() + 1, dtype=t.dtype, device=DEV)
        room[1:].copy_(t.view(-1))
        return room[1:].view(t.shape)

    t = {n: put(a) for n, a in d.items()}
    f = {n: a.astype(np.float64) for n, a in d.items()}
    axes = np.repeat(np.arange(len(pairs)), pairs)
    angle = f["position"][:, axes] * f["omega"]
    gam = dict(gamma_q=t["gamma_q"], gamma_k=t["gamma_k"]) if gains else {}
    q, k = (t["q"] if H else None), (t["k"] if K else None)
    keep = [None if a is None else a.clone() for a in (q, k)]
    outs = dict(q_out=q if H else True, k_out=k if K else True) if inplace else {}
    got = cngp.rotate_fwd(cfg, q, k, t["position"] if sum(pairs) else None, t["omega"] if sum(pairs) else None, **gam, **outs)
    q, k = keep
    start = {n: np.random.default_rng(7).normal(size=D).astype(np.float32) for n in ("q", "k")}
    into = dict(dgamma_q=dev(start["q"]) if gains and norm else False, dgamma_k=dev(start["k"]) if gains and norm else False)
    ups = [t["dq"] if H else None, t["dk"] if K else None]
    back = cngp.rotate_bwd(cfg, q, k, t["position"] if sum(pairs) else None, t["omega"] if sum(pairs) else None, *ups, **gam, **into,
                           **(dict(dq=ups[0] if H else True, dk=ups[1] if K else True) if inplace else {}))
    for i, (n, heads) in enumerate((("q", H), ("k", K))):
        if not heads:
            assert got[i] is None and back[i] is None
            continue
        gamma = f["gamma_" + n] if gains else np.ones(D)
        y, dx, dg = R.rotate(f[n], angle, nxt, gamma, eps, norm, f["d" + n])
        x = f[n]
        r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps) if norm else np.ones_like(x[..., :1])
        top = np.abs(x * r * (gamma if norm else 1)).max(-1, keepdims=True, initial=0.0)
        R.within("y " + n, host(got[i]), y, 2 * top * R.U * (D / 2 + 16 if norm else 10), NP[io])
        w = np.abs(f["d" + n]).max(-1, keepdims=True, initial=0.0) * (np.abs(gamma).max() if norm else 1)
        hat = np.abs(x * r)
        bound = 2 * w * R.U * 10 if not norm else r * 2 * (2 * w * R.U * (D / 2 + 16) + hat * (2 * w * hat).mean(-1, keepdims=True) * R.U * (2 * D + 32))
        R.within("dx " + n, host(back[i]), dx, bound, NP[io])
        if gains and norm:
            mag = (2 * np.abs(f["d" + n]).max(-1, keepdims=True, initial=0.0) * hat).sum((0, 1))
            terms = min(N * heads, 2 * N * heads / 256 + 1100) + D / 2 + 24         # a lane's own sums, then those of groups and workgroups
            R.within("dgamma " + n, host(back[2 + i]), dg + start[n], mag * R.U * terms + np.abs(start[n]) * R.U)


@pytest.mark.parametrize("D,pairs", [(1, (0,)), (2, (1,)), (8, (4,)), (7, (3,)), (12, (2, 2)), (36, (3, 3, 3)), (64, (32,)), (64, (8, 12, 12)), (128, (16, 24, 24)),
                                     (128, (64,)), (128, (32,)), (96, (10, 2, 3, 7)), (130, (65,)), (255, (100, 20)), (512, (256,)), (512, (0, 8)), (511, (1,))])
@pytest.mark.parametrize("nxt", [False, True])
@pytest.mark.parametrize("io", [F16, F32])
def test_dimensions_axes_and_types(D, pairs, nxt, io):
    check(5, 3, 2, D, pairs, io, True, nxt, seed=D)


@pytest.mark.parametrize("norm,gains", [(True, True), (True, False), (False, False), (False, True)])
@pytest.mark.parametrize("H,K", [(4, 1), (1, 0), (0, 2), (20, 5)])
@pytest.mark.parametrize("io,nxt", [(F16, False), (F32, True)])
def test_heads_and_norms(norm, gains, H, K, io, nxt):
    check(9, H, K, 40, (8, 8), io, norm, nxt, gains)


@pytest.mark.parametrize("N", [1, 2, 63, 64, 65, 1000, 20011])
@pytest.mark.parametrize("io", [F16, F32])
def test_rows(N, io):
    check(N, 2, 1, 24, (8, 4), io)


@pytest.mark.parametrize("io,nxt", [(F16, True), (F16, False), (F32, True), (F32, False)])
def test_alignment_and_in_place(io, nxt):
    check(33, 3, 2, 64, (16, 16), io, True, nxt, shift=True)
    check(33, 3, 2, 64, (16, 16), io, True, nxt, inplace=True)
    check(33, 3, 2, 30, (7, 8), io, False, nxt, inplace=True)


def test_far_positions_turn_as_exactly_as_near_ones():
    check(300, 2, 1, 64, (32,), F32, False, far=2.0 ** 24)
    check(300, 2, 1, 64, (16, 16), F32, True, far=2.0 ** 23)


def test_rows_of_zeros_and_without_rows():
    cfg = cngp.RotateConfig(2, 1, 16, (8,), F16, 0.0, cngp.ROTATE_NORM)
    z = lambda h: torch.zeros((3, h, 16), dtype=torch.float16, device=DEV)
    pos, om = torch.ones((3, 1), device=DEV), torch.ones(8, device=DEV)
    eps = cngp.RotateConfig(2, 1, 16, (8,), F16, 1e-6, cngp.ROTATE_NORM)
    q, k = cngp.rotate_fwd(eps, z(2), z(1), pos, om)
    assert not q.any() and not k.any()
    e = lambda h: torch.empty((0, h, 16), dtype=torch.float16, device=DEV)
    q, k = cngp.rotate_fwd(cfg, e(2), e(1), torch.empty((0, 1), device=DEV), om)
    assert q.shape == (0, 2, 16)
    gamma = torch.ones(16, device=DEV)
    zero = cngp.RotateConfig(2, 1, 16, (8,), F16, 1e-6, cngp.ROTATE_NORM | cngp.ZERO_GRADS)
    out = torch.full((16,), 7.0, device=DEV)
    cngp.rotate_bwd(zero, e(2), e(1), torch.empty((0, 1), device=DEV), om, e(2), e(1), gamma, gamma, dgamma_q=out)
    assert not out.any()


def test_same_bits_again():
    d = make(5000, 4, 2, 64, (32,), F16, 3)
    t = {n: dev(a) for n, a in d.items()}
    cfg = cngp.RotateConfig(4, 2, 64, (32,), F16, 1e-6, cngp.ROTATE_NORM | cngp.ZERO_GRADS)
    call = lambda: cngp.rotate_bwd(cfg, t["q"], t["k"], t["position"], t["omega"], t["dq"], t["dk"], t["gamma_q"], t["gamma_k"])
    a, b = call(), call()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_gradient_against_differences():
    d = make(6, 2, 1, 12, (2, 3), F32, 4)
    t = {n: dev(a) for n, a in d.items()}
    cfg = cngp.RotateConfig(2, 1, 12, (2, 3), F32, 1e-6, cngp.ROTATE_NORM)
    gr = cngp.rotate_bwd(cfg, t["q"], t["k"], t["position"], t["omega"], t["dq"], t["dk"], t["gamma_q"], t["gamma_k"])
    loss = lambda u: sum((a.double() * b.double()).sum() for a, b in
                         zip(cngp.rotate_fwd(cfg, u["q"], u["k"], u["position"], u["omega"], u["gamma_q"], u["gamma_k"]), (t["dq"], t["dk"])))
    r = torch.Generator(device=DEV).manual_seed(0)
    for n, g in zip(("q", "k", "gamma_q", "gamma_k"), gr):
        move = torch.randn(g.shape, generator=r, device=DEV)
        step = 2.0 ** -7
        up, down = dict(t), dict(t)
        up[n], down[n] = t[n] + step * move, t[n] - step * move
        diff, want = float((loss(up) - loss(down)) / (2 * step)), float((g.double() * move.double()).sum())
        mags = float((g.double().abs() * move.double().abs()).sum())
        # rounding of a loss of 216 terms below 20 each, and the third derivative of 1 / norm (heads of 12 components, norm above 1)
        assert abs(diff - want) <= 216 * 20 * 40 * R.U / step + 30 * step ** 2 * max(mags, 1.0), (n, diff, want)
