"""The mixer's operators together, as a model of rows along rays uses them: encodings -> queries, keys, values -> norms and rotation -> attention
with decays -> pixels -> squared error, back through all of it, and the weights moved by the orthogonalised step.  Held against the same
computation in 64 bits by torch's autograd on the CPU.

Tolerance: each stage is fp32 with at most a few hundred roundings of 2^-24 relative to the magnitudes it sums (heads of 16 columns, rays of at most
40 rows, weights' gradients over a thousand rows, each in sums of mixed sign): 1e-4 of the largest entry is above their product with room for the
cancellation of a gradient of random signs.  The step is held to the bound of one orthogonalisation of the gradient that it was given."""
import numpy as np
import pytest
import torch

import mixer_ref as R
import paper_2312_17241_amd as cngp
from paper_2312_17241_amd.module import Encoding, attend, rotate

pytestmark = pytest.mark.gpu
DEV = "cuda"
H, K, D, V = 4, 2, 16, 12


def close(name, got, want, rel=1e-4):
    got, want = got.detach().cpu().double(), want.detach().cpu().double()
    assert got.shape == want.shape and float((got - want).abs().max()) <= rel * float(want.abs().max()), name


def attend_64(q, k, v, g, offsets, h0, scale):
    y, last = [], []
    k, v = k.repeat_interleave(H // K, 1), v.repeat_interleave(H // K, 1)
    for s in range(len(offsets) - 1):
        st = h0[s]
        for r in range(int(offsets[s]), int(offsets[s + 1])):
            st = torch.exp(g[r])[:, None, None] * st + k[r][:, :, None] * v[r][:, None, :]
            y.append(scale * (st * q[r][:, :, None]).sum(1))
        last.append(st)
    return torch.stack(y), torch.stack(last)


def rotate_64(x, gamma, angle):
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * gamma
    p = angle.shape[1]
    a, b, c, s = x[..., :p], x[..., p:2 * p], torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    return torch.cat([a * c - b * s, a * s + b * c, x[..., 2 * p:]], -1)


def test_a_training_iteration_of_a_mixer_of_rows():
    g = torch.Generator().manual_seed(5)
    enc = Encoding(cngp.Config(d=3, L=8, F=2, N_f=2**10, N_c=2**8, N_p=4, N_min=4, N_max=64), seed=1)
    with torch.no_grad():
        enc.D_f_master.copy_(torch.randn(enc.D_f_master.shape, generator=g) * 0.3)
    lengths = torch.randint(1, 41, (40,), generator=g)
    lengths[::9] = 0
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), lengths.cumsum(0)]).int()
    N, S = int(offsets[-1]), 40
    x = torch.rand(N, 3, generator=g)
    width = (H + K) * D + K * V + H
    W = torch.randn(16, width, generator=g) * 0.4
    gains = [1 + 0.2 * torch.randn(D, generator=g) for _ in range(2)]
    h0, omega = torch.randn(S, H, D, V, generator=g) * 0.3, 2.0 ** torch.arange(6) * 1.0
    target = torch.rand(N, H, V, generator=g)
    cut = [H * D, K * D, K * V, H]

    def parts(z):
        q, k, v, d = torch.split(z, cut, 1)
        return (q.reshape(N, H, D).contiguous(), k.reshape(N, K, D).contiguous(), v.reshape(N, K, V).contiguous(),
                torch.nn.functional.logsigmoid(d + 2).contiguous())

    leaf = lambda t: t.to(DEV).requires_grad_()
    w, gq, gk, h = leaf(W), leaf(gains[0]), leaf(gains[1]), leaf(h0)
    y = enc(x.to(DEV))
    y.retain_grad()
    q, k, v, d = parts(y @ w)
    rc = cngp.RotateConfig(H, K, D, (2, 2, 2), flags=cngp.ROTATE_NORM)
    q, k = rotate(rc, q, k, x.to(DEV), omega.to(DEV), gq, gk)
    ac = cngp.AttendConfig(H, K, D, V, longest=40, scale=0.25, flags=cngp.ATTEND_ROW_DECAY)
    out, last = attend(ac, q, k, v, d, h, offsets.to(DEV))
    loss = ((out - target.to(DEV)) ** 2).sum() + (last ** 2).sum()
    loss.backward()

    leaf64 = lambda t: t.double().requires_grad_()
    y64, w64, gq64, gk64, h64 = y.detach().cpu().double().requires_grad_(), *map(leaf64, (W, *gains, h0))
    q, k, v, d = parts(y64 @ w64)
    angle = x.double().repeat_interleave(2, 1) * omega.double()
    out64, last64 = attend_64(rotate_64(q, gq64, angle), rotate_64(k, gk64, angle), v, d, offsets, h64, 0.25)
    (((out64 - target.double()) ** 2).sum() + (last64 ** 2).sum()).backward()
    close("outputs", out, out64)
    close("states", last, last64)
    for name, a, b in (("W", w, w64), ("gain of q", gq, gq64), ("gain of k", gk, gk64), ("h0", h, h64), ("encodings", y, y64)):
        close(name, a.grad, b.grad)

    # the weights' step: moves by lr times the orthogonalised gradient (momentum from zero: 1.95 times the gradient), to that operator's own bound
    before, grad = w.detach().clone(), w.grad.clone()
    cngp.muon_step(cngp.OrthoConfig(16, width), cngp.Muon(0.02, 0.95), before, None, torch.zeros_like(before), grad, clear_grad=True)
    o = R.orthogonalise(w.grad.cpu().double().numpy()[None], 5, tuple(float(np.float32(c)) for c in (3.4445, -4.7750, 2.0315)), 0.0)[0]
    error = 2.0 ** -22 * (5 + width / 64)
    for _ in range(5):
        error = 3.4445 * error + 12 * 2.0 ** -22 * (5 + width / 64)
    want = W.double().numpy() - float(np.float32(0.02)) * o
    R.within("step", before.cpu().numpy(), want, 0.02 * error + 4 * R.U * np.abs(want))
    assert not grad.any()


def leaves(io, seed, N=200, S=4):
    g = torch.Generator().manual_seed(seed)
    make = lambda *s: torch.randn(s, generator=g).to(io).to(DEV).requires_grad_()
    decay = (-torch.rand(N, H, generator=g)).to(DEV).requires_grad_()
    return make(N, H, D), make(N, K, D), make(N, K, V), decay, torch.randn(S, H, D, V, generator=g).to(DEV).requires_grad_()


AC = {torch.float16: cngp.AttendConfig(H, K, D, V, cngp.F16, flags=cngp.ATTEND_ROW_DECAY), torch.float32: cngp.AttendConfig(H, K, D, V, flags=cngp.ATTEND_ROW_DECAY)}


@pytest.mark.parametrize("io", [torch.float16, torch.float32])
def test_rows_of_no_sequence_are_zeros_with_gradients_of_zero(io):
    q, k, v, decay, h0 = leaves(io, 1)
    off = torch.tensor([3, 70, 70, 120, 190], dtype=torch.int32, device=DEV)
    with torch.no_grad():
        for t in (q, k, v, decay):
            t[:3] = float("nan")
            t[190:] = float("inf")
    y, last = attend(AC[io], q, k, v, decay, h0, off)
    assert not y[:3].any() and not y[190:].any() and bool(torch.isfinite(y).all())
    (y.float().sum() + last.sum()).backward()
    for t in (q, k, v, decay):
        assert not t.grad[:3].any() and not t.grad[190:].any() and bool(torch.isfinite(t.grad).all()) and bool(t.grad.any())


def test_outputs_that_are_not_used_and_leaves_without_gradients():
    q, k, v, decay, h0 = leaves(torch.float32, 2)
    y, last = attend(AC[torch.float32], q, k, v, decay, h0, None, 4)
    last.sum().backward(retain_graph=True)
    assert not q.grad.any() and bool(k.grad.any()) and bool(h0.grad.any())
    fixed = [t.detach() for t in (k, v, decay, h0)]
    q2 = q.detach().requires_grad_()
    y2, _ = attend(AC[torch.float32], q2, *fixed, None, 4)
    y2.sum().backward()
    q.grad = None
    y.sum().backward()
    assert torch.equal(q2.grad, q.grad) and all(t.grad is None for t in fixed)
    rc = cngp.RotateConfig(0, K, D, (8,), flags=cngp.ROTATE_NORM)
    none, k3 = rotate(rc, None, k, torch.ones(200, 1, device=DEV), torch.ones(8, device=DEV))
    k.grad = None
    (k3 * k3.detach()).sum().backward()
    assert none is None and k.grad.shape == k.shape


@pytest.mark.parametrize("io", [torch.float16, torch.float32])
def test_on_another_stream_and_captured(io):
    """Forward and backward captured into two graphs, replayed in turns with the program's own eager work in between: every replay is the eager result."""
    side = torch.cuda.Stream()
    cfg = AC[io]
    rc = cngp.RotateConfig(H, K, D, (8,), cfg.io_dtype, flags=cngp.ROTATE_NORM)
    N = 1300                                                # one sequence: cut, with anchors
    pos, om, gamma = torch.rand(N, 1, device=DEV), torch.rand(8, device=DEV), torch.ones(D, device=DEV)

    def run(q, k, v, decay, h0, dy):
        qr, kr = cngp.rotate_fwd(rc, q, k, pos, om, gamma, gamma)
        y, last = cngp.attend_fwd(cfg, qr, kr, v, decay, h0=h0, workspace=room)
        grads = cngp.attend_bwd(cfg, qr, kr, v, decay, dy=dy, dlast=last, h0=h0, workspace=room)
        return (y, last) + grads

    room = torch.empty(cngp.attend_workspace_bytes(cfg, N, 1, True), dtype=torch.uint8, device=DEV)    # one for both graphs
    ins = [[t.detach() for t in leaves(io, s, N, 1)] for s in (3, 4, 5)]
    dy = torch.randn(N, H, V, device=DEV).to(io)
    want = [[t.clone() for t in run(*i, dy)] for i in ins]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        other = run(*ins[2], dy)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want[2]))
    graphs = []
    for i in (0, 1):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = run(*ins[i], dy)
        graphs.append((g, out, want[i]))
    for turn in range(4):
        for g, out, ref in graphs if turn % 2 else graphs[::-1]:
            for t in out:
                t.zero_()
            room.fill_(255)
            g.replay()
            assert all(torch.equal(a, b) for a, b in zip(out, ref)), turn
            assert all(torch.equal(a, b) for a, b in zip(run(*ins[2], dy), want[2]))


def test_autograd_captured_with_its_forward():
    q, k, v, decay, h0 = leaves(torch.float32, 6)
    ac, rc = AC[torch.float32], cngp.RotateConfig(H, K, D, (8,), flags=cngp.ROTATE_NORM)
    pos, om, gamma = torch.rand(200, 1, device=DEV), torch.rand(8, device=DEV), torch.ones(D, device=DEV, requires_grad=True)

    def run():
        a, b = rotate(rc, q, k, pos, om, gamma, gamma)
        y, last = attend(ac, a, b, v, decay, h0, None, 4)
        return torch.autograd.grad((y * y.detach()).sum() + (last * last.detach()).sum(), (q, k, v, decay, h0, gamma))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [t.clone() for t in run()]
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = run()
    for _ in range(3):
        for t in out:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)


def test_optimiser_step_captured():
    for m, n in ((32, 64), (150, 200)):
        cfg = cngp.OrthoConfig(m, n)
        new = lambda: [torch.randn(m, n, generator=torch.Generator().manual_seed(s)).to(DEV) for s in (1, 2, 3)]
        room = torch.empty(max(cngp.orthogonalise_workspace_bytes(cfg), 256), dtype=torch.uint8, device=DEV)
        step = lambda a: cngp.muon_step(cfg, cngp.Muon(), a[0], None, a[1], a[2], workspace=room)
        eager, caught = new(), new()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(caught)
        for _ in range(3):
            step(eager)
            room.fill_(255)
            g.replay()
            assert all(torch.equal(a, b) for a, b in zip(eager, caught))
