"""The reference of the recurrence's gradient (recur_ref.py) against autograd and against differences, in 64 bits on the CPU."""
import numpy as np
import pytest
import torch

import recur_ref as R

LENGTHS = [4, 0, 1, 6]


def loss_of(gate, x, h0, dy, dlast, spans, reverse, log_gate, mix):
    a = gate.exp() if log_gate else gate
    total = 0.0
    for s, (lo, hi) in enumerate(spans):
        h = h0[s]
        for r in (range(hi - 1, lo - 1, -1) if reverse else range(lo, hi)):
            h = a[r] * h + (1 - a[r] if mix else 1.0) * x[r]
            total = total + (h * dy[r]).sum()
        total = total + (h * dlast[s]).sum()
    return total


@pytest.mark.parametrize("shared", [False, True])
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("log_gate", [False, True])
@pytest.mark.parametrize("mix", [False, True])
def test_gradients(shared, reverse, log_gate, mix):
    g = np.random.default_rng(3)
    N, C, S = sum(LENGTHS), 3, len(LENGTHS)
    spans = R.spans(N, S, np.concatenate([[0], np.cumsum(LENGTHS)]))
    gate = g.uniform(-1, -0.1, (N, 1 if shared else C)) if log_gate else g.uniform(-0.9, 0.9, (N, 1 if shared else C))
    x, h0, dy, dlast = g.normal(size=(N, C)), g.normal(size=(S, C)), g.normal(size=(N, C)), g.normal(size=(S, C))
    ref = R.backward(gate, x, spans, h0, dy, dlast, reverse, log_gate, mix)
    leaves = [torch.from_numpy(v).requires_grad_() for v in (gate, x, h0)]
    args = (torch.from_numpy(dy), torch.from_numpy(dlast), spans, reverse, log_gate, mix)
    loss_of(*leaves, *args).backward()
    for leaf, name in zip(leaves, ("dgate", "dx", "dh0")):
        assert np.allclose(leaf.grad.numpy(), ref[name], rtol=1e-12, atol=1e-12), name
    with torch.no_grad():
        for leaf, name in zip(leaves, ("dgate", "dx", "dh0")):
            flat, step = leaf.view(-1), 1e-6
            for i in range(0, flat.numel(), 5):
                old = flat[i].item()
                flat[i] = old + step
                up = float(loss_of(*leaves, *args))
                flat[i] = old - step
                down = float(loss_of(*leaves, *args))
                flat[i] = old
                assert abs((up - down) / (2 * step) - ref[name].reshape(-1)[i]) < 1e-7 * (1 + abs(ref[name].reshape(-1)[i])) + 1e-8, name


def test_bounds_hold_for_fp32_evaluated_in_pieces():
    """A sequence cut in pieces, each scanned from nothing and joined by the product of its gates, in numpy's fp32."""
    g = np.random.default_rng(5)
    T, C = 4096, 4
    gate = (1 / (1 + np.exp(-g.normal(size=(T, C)) - 4))).astype(np.float32)
    x = g.normal(size=(T, C)).astype(np.float32)
    ref = R.forward(gate.astype(np.float64), x.astype(np.float64), [(0, T)], None, False, False, False)
    for piece in (1, 8, 64, 1024):
        carry = np.zeros(C, np.float32)
        got = np.zeros((T, C), np.float32)
        for p in range(0, T, piece):
            A, B = np.ones(C, np.float32), np.zeros(C, np.float32)
            for r in range(p, p + piece):
                A, B = A * gate[r], gate[r] * B + x[r]
                got[r] = A * carry + B
            carry = got[p + piece - 1]
        R.within(f"pieces of {piece}", got.astype(np.float64), ref["y"], ref["Ey"])
