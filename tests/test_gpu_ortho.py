"""Orthogonalised updates on the GPU against the same products in 64 bits (mixer_ref.py).

Bound: with 22 bits to an operand and fp32 sums, a step's result has an error matrix of norm at most e = 2^-22 (4 + depth of the sums / 64) times
the operands' norms; singular values stay below 1.3, so each step adds at most 12 e (products with norms 1.3^2 * 4.8 and 1.3^4 * 2.04) and lifts what is there by
its largest slope, 3.4445.  Norms bound entries."""
import numpy as np
import pytest
import torch

import mixer_ref as R
import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, F32 = cngp.F16, cngp.F32
NP = {F16: np.float16, F32: np.float32}
MUON, CUBIC = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)


def as_fp32(c):
    return tuple(float(np.float32(v)) for v in c)


def bound(m, n, steps, slope=3.4445):
    e = 2.0 ** -22 * (4 + max(m, n) / 64)
    b = e
    for _ in range(steps):
        b = slope * b + 12 * e
    return b


def matrices(batch, m, n, seed, size=1e-2):
    g = np.random.default_rng(seed)
    low = g.normal(size=(batch, m, max(1, min(m, n) // 6))) @ g.normal(size=(batch, max(1, min(m, n) // 6), n))
    return (low + 0.5 * g.normal(size=(batch, m, n))) * size


@pytest.mark.parametrize("m,n", [(1, 1), (1, 7), (5, 1), (3, 3), (16, 16), (16, 64), (64, 32), (64, 64), (65, 64), (64, 129), (100, 30), (128, 128), (129, 127), (200, 333), (300, 70)])
@pytest.mark.parametrize("io", [F16, F32])
def test_shapes_and_types(m, n, io):
    g = matrices(2, m, n, m + n).astype(NP[io])
    cfg = cngp.OrthoConfig(m, n, 2, io)
    out = cngp.orthogonalise(cfg, torch.from_numpy(g).to(DEV))
    want = R.orthogonalise(g.astype(np.float64), 5, as_fp32(MUON), float(np.float32(1e-7)))
    R.within("out", out.cpu().numpy(), want, bound(m, n, 5), NP[io])


@pytest.mark.parametrize("steps", [0, 1, 2, 6])
@pytest.mark.parametrize("m,n", [(40, 56), (150, 90)])
@pytest.mark.parametrize("coefficients", [MUON, CUBIC])
def test_steps_and_coefficients(steps, m, n, coefficients):
    g = matrices(3, m, n, steps).astype(np.float32)
    cfg = cngp.OrthoConfig(m, n, 3, F32, steps, coefficients)
    out = cngp.orthogonalise(cfg, torch.from_numpy(g).to(DEV))
    want = R.orthogonalise(g.astype(np.float64), steps, as_fp32(coefficients), float(np.float32(1e-7)))
    R.within("out", out.cpu().numpy(), want, bound(m, n, steps))


@pytest.mark.parametrize("m,n", [(64, 64), (130, 200)])
def test_cubic_converges_to_orthogonal_rows(m, n):
    g = torch.randn((1, m, n), generator=torch.Generator().manual_seed(3)).to(DEV)
    q = torch.linalg.qr(g[0].double().cpu().T if m <= n else g[0].double().cpu())[0]
    g = (q.T * torch.linspace(0.3, 1.0, m).double()[:, None]).float().to(DEV)[None].contiguous()
    out = cngp.orthogonalise(cngp.OrthoConfig(m, n, 1, F32, 24, CUBIC), g)[0].double().cpu()
    assert float((out @ out.T - torch.eye(m, dtype=torch.float64)).abs().max()) < 1e-4


@pytest.mark.parametrize("size", [1e-30, 1e-12, 1e8, 1e30])
@pytest.mark.parametrize("m,n", [(32, 64), (200, 130)])
def test_sizes_of_the_entries(size, m, n):
    g = matrices(1, m, n, 5, size).astype(np.float32)
    out = cngp.orthogonalise(cngp.OrthoConfig(m, n, 1, F32, 5, MUON, 0.0), torch.from_numpy(g).to(DEV))
    want = R.orthogonalise(g.astype(np.float64), 5, as_fp32(MUON), 0.0)
    R.within("out", out.cpu().numpy(), want, bound(m, n, 5))


@pytest.mark.parametrize("m,n", [(32, 64), (200, 130)])
@pytest.mark.parametrize("io", [F16, F32])
def test_zeros_not_finite_in_place_and_alignment(m, n, io):
    g = torch.from_numpy(matrices(3, m, n, 6).astype(NP[io])).to(DEV)
    cfg = cngp.OrthoConfig(m, n, 3, io)
    clean = cngp.orthogonalise(cfg, g)
    dirty = g.clone()
    dirty[1] = 0
    dirty[2, 0, 0] = float("nan")
    out = cngp.orthogonalise(cfg, dirty)
    assert torch.equal(out[0], clean[0]) and not out[1].any() and not bool(torch.isfinite(out[2]).any())
    same = cngp.orthogonalise(cfg, dirty, out=dirty)
    assert same is dirty and torch.equal(same[:2], out[:2])
    room = torch.empty(g.numel() + 1, dtype=g.dtype, device=DEV)
    room[1:].copy_(g.view(-1))
    shifted = room[1:].view(g.shape)
    assert torch.equal(cngp.orthogonalise(cfg, shifted, out=torch.empty_like(room)[1:].view(g.shape)), clean)


def test_transposed_matrices_give_transposed_updates():
    for m, n in ((48, 64), (140, 300)):
        g = torch.from_numpy(matrices(2, m, n, 7).astype(np.float32)).to(DEV)
        a = cngp.orthogonalise(cngp.OrthoConfig(m, n, 2), g)
        b = cngp.orthogonalise(cngp.OrthoConfig(n, m, 2), g.transpose(1, 2).contiguous())
        assert float((a - b.transpose(1, 2)).abs().max()) <= 2 * bound(m, n, 5)


def test_same_bits_in_any_workspace_and_batch():
    g = torch.from_numpy(matrices(4, 150, 260, 8).astype(np.float32)).to(DEV)
    cfg = cngp.OrthoConfig(150, 260, 4)
    ref = cngp.orthogonalise(cfg, g)
    for fill in (0, 255):
        ws = torch.full((cngp.orthogonalise_workspace_bytes(cfg),), fill, dtype=torch.uint8, device=DEV)
        assert torch.equal(cngp.orthogonalise(cfg, g, workspace=ws), ref)


@pytest.mark.parametrize("batch,m,n", [(36, 640, 650), (36, 650, 640), (36, 640, 644), (4, 1000, 2100), (4, 2100, 1000), (1, 333, 1021), (3, 200, 1100)])
@pytest.mark.parametrize("io", [F16, F32])
def test_tiles_that_are_cut_along_the_contraction(batch, m, n, io):
    """Tiles that do not fill the card, or are left after those that do; the last matrices hold them."""
    g = matrices(batch, m, n, m).astype(NP[io])
    t = torch.from_numpy(g).to(DEV)
    steps = 2
    out = cngp.orthogonalise(cngp.OrthoConfig(m, n, batch, io, steps), t)
    some = sorted({0, batch - 2, batch - 1} - {-1})
    want = R.orthogonalise(g[some].astype(np.float64), steps, as_fp32(MUON), float(np.float32(1e-7)))
    R.within("out", out.cpu().numpy()[some], want, bound(m, n, steps), NP[io])
    assert torch.equal(cngp.orthogonalise(cngp.OrthoConfig(m, n, batch, io, steps), t), out)
    if io == F32:
        w, mom = torch.zeros_like(t), torch.zeros_like(t)
        cngp.muon_step(cngp.OrthoConfig(m, n, batch, steps=steps), cngp.Muon(1.0, 0.0, nesterov=False), w, None, mom, t)
        assert torch.equal(w, -out)


@pytest.mark.parametrize("m,n,batch", [(3, 5, 1), (64, 32, 2), (64, 128, 1), (100, 30, 3), (130, 260, 2), (300, 70, 1)])
@pytest.mark.parametrize("nesterov,clear,half", [(True, True, True), (False, False, False)])
@pytest.mark.parametrize("steps", [0, 5])
def test_optimiser_steps(m, n, batch, nesterov, clear, half, steps):
    """Three steps in a row against 64 bits, each from what the library left: the momentum and the weights are rounded twice each, the direction's
    own roundings (4 u of its terms) come into the orthogonalised matrix as noise of that share of its norm."""
    g = np.random.default_rng(m)
    shape = (batch, m, n) if batch > 1 else (m, n)
    master, mom = (torch.from_numpy(g.normal(size=shape).astype(np.float32)).to(DEV), torch.zeros(shape, device=DEV))
    cfg, opt = cngp.OrthoConfig(m, n, batch, steps=steps), cngp.Muon(0.02, 0.9, 0.1, 0.25, nesterov)
    copy = torch.empty(shape, dtype=torch.float16, device=DEV) if half else None
    mo, lr, wd = (float(np.float32(v)) for v in (0.9, 0.02, 0.1))
    for i in range(3):
        grad = torch.from_numpy(matrices(batch, m, n, i).astype(np.float32).reshape(shape)).to(DEV)
        w64, m64, g64 = (t.cpu().double().numpy().reshape(batch, m, n) for t in (master, mom, grad))
        cngp.muon_step(cfg, opt, master, copy, mom, grad, clear_grad=clear)
        new = mo * m64 + 0.25 * g64
        u, mag = (mo * new + 0.25 * g64, np.abs(mo * new) + np.abs(0.25 * g64)) if nesterov else (new, np.abs(mo * m64) + np.abs(0.25 * g64))
        R.within("momentum", mom.cpu().numpy().reshape(new.shape), new, 2 * R.U * (np.abs(mo * m64) + np.abs(0.25 * g64)))
        o = R.orthogonalise(u, steps, as_fp32(MUON), float(np.float32(1e-7)))
        noise = 4 * R.U * max(float(np.linalg.norm(b) / np.linalg.norm(a)) for a, b in zip(u, mag))
        want = w64 * (1 - lr * wd) - lr * o
        slack = lr * (bound(m, n, steps) + noise * 3.4445 ** steps) + R.U * (4 * np.abs(w64) + 2 * lr * np.abs(o))
        R.within("weights", master.cpu().numpy().reshape(want.shape), want, slack)
        if half:
            assert torch.equal(copy, master.half())
        assert bool((grad == 0).all()) == clear


def test_optimiser_step_of_nothing():
    """A gradient and momentum of zeros leave the weights, but for their decay."""
    for m, n in ((32, 16), (130, 70)):
        w = torch.randn(m, n, device=DEV)
        want, mom, grad = w * (1 - 0.5 * 0.25), torch.zeros(m, n, device=DEV), torch.zeros(m, n, device=DEV)
        cngp.muon_step(cngp.OrthoConfig(m, n, eps=0.0), cngp.Muon(0.5, 0.9, 0.25), w, None, mom, grad)
        assert torch.equal(w, want) and not mom.any()
