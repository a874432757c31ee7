"""Balance of the probing candidates on the GPU against the definition in 64 bits.

Tolerances, u = 2^-24.  A softmax weight: exponential of a rounded difference (|logit - max| u relative, plus two for the function), the
sum of N_p of them, a reciprocal and a product: (|v - max| + N_p + 6) u relative.  P: the same relative to itself, plus at most as many
roundings as the longest chain of additions (a lane's rows, then 6 + 2 + 64 steps: 200 is above all shapes here).  The loss adds N_p.
The gradient is relative to w N_p / W sigma (f + sum f sigma), the magnitude of its terms."""
import numpy as np
import pytest
import torch

import oracle
import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def config(L, N_c, N_p, top_k=0, flags=0, **kw):
    return cngp.Config(d=3, L=L, F=2, N_f=2**10, N_c=N_c, N_p=N_p, N_min=4, N_max=64, top_k=top_k, flags=flags, **kw)


def reference(v, rows, weight, top_k):
    L, N_c, N_p = v.shape
    order = np.argsort(-v, axis=2, kind="stable")
    winner = order[:, :, 0]
    kept = v.copy()
    if top_k:
        mask = np.zeros(v.shape, bool)
        np.put_along_axis(mask, order[:, :, :top_k], True, 2)
        kept[~mask] = -np.inf
    depth = kept - kept.max(2, keepdims=True)
    e = np.exp(depth)
    sigma = e / e.sum(2, keepdims=True)
    rel = (np.where(np.isfinite(depth), -depth, 0) + N_p + 6) * U
    counted = np.ones((L, N_c), bool) if rows is None else rows != 0
    W = counted.sum(1)
    one = np.maximum(W, 1)[:, None]
    counts = np.stack([((winner == k) & counted).sum(1) for k in range(N_p)], 1)
    f = counts / one
    P = (sigma * counted[..., None]).sum(1) / one
    EP = (sigma * rel * counted[..., None]).sum(1) / one + 200 * U * P
    loss, El = N_p * (f * P).sum(1), N_p * (f * (EP + (N_p + 4) * U * P)).sum(1)
    inner = (f[:, None, :] * sigma).sum(2, keepdims=True)
    Ei = (f[:, None, :] * sigma * (rel + (N_p + 2) * U)).sum(2, keepdims=True)
    scale = np.where(counted, abs(weight) * N_p / one, 0.0)[..., None]
    grad = np.sign(weight) * scale * sigma * (f[:, None, :] - inner)
    Eg = scale * sigma * ((rel + 8 * U) * (f[:, None, :] + inner) + Ei)
    return loss, El, counts, grad, Eg


def check(L, N_c, N_p, top_k=0, rows=None, weight=0.7, accumulate=False, seed=1, spread=1.0, dhat=None):
    g = np.random.default_rng(seed + N_c)
    v = (g.normal(size=(L, N_c, N_p)) * spread + g.normal(size=(L, 1, N_p)) * 0.3).astype(np.float32) if dhat is None else dhat
    if rows == "some":
        rows = (g.random((L, N_c)) < 0.6).astype(np.uint8) * g.integers(1, 256, (L, N_c)).astype(np.uint8)
    elif isinstance(rows, str) and rows == "none":
        rows = np.zeros((L, N_c), np.uint8)
        rows[1:, ::3] = 1                                # a level without counted rows
    held = v.copy()
    if rows is not None:                                  # what a row that is not counted holds does not matter
        held[rows == 0] = np.where(g.random((int((rows == 0).sum()), N_p)) < 0.5, np.nan, np.inf)
    cfg = config(L, N_c, N_p, top_k, 0 if accumulate else cngp.ZERO_GRADS)
    before = g.normal(size=v.shape).astype(np.float32) if accumulate else np.full(v.shape, np.nan, np.float32)
    ws = torch.full((max(cngp.probe_balance_workspace_bytes(cfg), 256),), 255, dtype=torch.uint8, device=DEV)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    rd = None if rows is None else dev(rows)
    loss, counts, grad = cngp.probe_balance(cfg, dev(held), weight, rows=rd, grad_Dhat_c=dev(before), workspace=ws)
    want, El, n, dg, Eg = reference(v.astype(np.float64), rows, weight, top_k if top_k < N_p else 0)
    assert counts.dtype == torch.int32 and np.array_equal(counts.cpu().numpy(), n)
    assert (np.abs(loss.cpu().numpy() - want) <= El + U * np.abs(want)).all(), (loss, want)
    start = before.astype(np.float64) if accumulate else 0.0
    off = np.abs(grad.cpu().numpy() - (start + dg))
    assert (off <= Eg + U * np.abs(start + dg) + 2.0 ** -140).all(), (off / (Eg + 1e-300)).max()
    if rows is not None and accumulate:
        assert np.array_equal(grad.cpu().numpy()[rows == 0], before[rows == 0])
    only = cngp.probe_balance(cfg, dev(held), weight, rows=rd, grad_Dhat_c=None)
    assert only[2] is None and torch.equal(only[0], loss) and torch.equal(only[1], counts)
    again = cngp.probe_balance(cfg, dev(held), weight, rows=rd, grad_Dhat_c=dev(before))
    assert torch.equal(again[0], loss) and torch.equal(again[2], grad)


@pytest.mark.parametrize("N_p", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("N_c", [1, 2, 4, 64, 256, 2048, 4096, 2**14])
@pytest.mark.parametrize("rows", [None, "some", "none"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_shapes(N_p, N_c, rows, accumulate):
    check(3, N_c, N_p, rows=rows, accumulate=accumulate)


@pytest.mark.parametrize("N_p,top_k", [(2, 1), (2, 2), (4, 1), (4, 3), (8, 2), (8, 7), (16, 1), (16, 4), (16, 16), (1, 1)])
@pytest.mark.parametrize("rows", [None, "some"])
@pytest.mark.parametrize("N_c", [1024, 8192])
def test_sparse_backward(N_p, top_k, rows, N_c):
    check(2, N_c, N_p, top_k, rows)


def test_ties_and_wide_logits():
    g = np.random.default_rng(7)
    for N_p in (2, 4, 8, 16):
        v = g.integers(-1, 2, (2, 512, N_p)).astype(np.float32)          # equal values everywhere: the lowest index wins
        check(2, 512, N_p, dhat=v)
        check(2, 512, N_p, top_k=N_p // 2, dhat=v)
    check(2, 4096, 16, spread=40.0)
    check(32, 2**15, 16, weight=-3.0)
    v = g.normal(size=(2, 256, 16)).astype(np.float32)
    v[:, :, 5:] = -np.inf                                                # candidates that are shut out
    check(2, 256, 16, dhat=v)
    v[:, :, 5:] = np.finfo(np.float32).min
    check(2, 256, 16, dhat=v)


def test_winners_are_those_of_the_bake_and_weights_those_of_the_backward():
    """counts = histogram of the baked index codebook, also for rows with NaN; and the loss is 1 where everything is even."""
    g = np.random.default_rng(3)
    for N_p in (2, 4, 8, 16):
        cfg = config(2, 2048, N_p)
        v = g.integers(-2, 3, (2, 2048, N_p)).astype(np.float32)
        v[g.random(v.shape) < 0.2] = np.nan
        d = torch.from_numpy(v).to(DEV)
        D_c = cngp.bake_probes(cfg, d).cpu().numpy()
        assert np.array_equal(D_c, oracle.bake_probes(v))
        counts = cngp.probe_balance(cfg, d)[1].cpu().numpy()
        assert np.array_equal(counts, np.stack([np.bincount(D_c[l], minlength=N_p) for l in range(2)]))
        even = torch.zeros(2, 2048, N_p, device=DEV)
        even.view(-1, N_p)[torch.arange(4096, device=DEV), torch.arange(4096, device=DEV) % N_p] = 1e-3
        loss, _, grad = cngp.probe_balance(cfg, even)
        assert bool((loss - 1).abs().max() < 1e-6)


def test_gradient_against_differences():
    """Where no winner changes, the loss of the GPU's own rows moves as its gradient says (in 64 bits, from the definition)."""
    g = np.random.default_rng(4)
    v = g.normal(size=(1, 32, 8)).astype(np.float32)
    cfg = config(1, 32, 8, flags=cngp.ZERO_GRADS)
    grad = cngp.probe_balance(cfg, torch.from_numpy(v).to(DEV), 1.0)[2].cpu().numpy()
    for i in range(0, 256, 7):
        up, down = v.astype(np.float64).copy(), v.astype(np.float64).copy()
        up.reshape(-1)[i] += 1e-6
        down.reshape(-1)[i] -= 1e-6
        diff = (reference(up, None, 1.0, 0)[0] - reference(down, None, 1.0, 0)[0])[0] / 2e-6
        assert abs(diff - grad.reshape(-1)[i]) < 1e-7


def test_unaligned_arrays_and_graph_replays():
    cfg = config(3, 4096, 16, flags=cngp.ZERO_GRADS)
    n = 3 * 4096 * 16
    flat = torch.randn(n + 1, device=DEV)
    v = flat[1:].view(3, 4096, 16)
    grad = torch.empty(n + 1, device=DEV)[1:].view(3, 4096, 16)
    loss, counts, _ = cngp.probe_balance(cfg, v, 0.5, grad_Dhat_c=grad)
    want = cngp.probe_balance(cfg, v.clone(), 0.5)
    assert torch.equal(loss, want[0]) and torch.equal(counts, want[1]) and torch.equal(grad, want[2])
    src = v.clone()
    out = [torch.empty_like(t) for t in want]
    ws = torch.empty(cngp.probe_balance_workspace_bytes(cfg), dtype=torch.uint8, device=DEV)
    step = lambda: cngp.probe_balance(cfg, src, 0.5, loss=out[0], counts=out[1], grad_Dhat_c=out[2], workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for o in out:
            o.fill_(9)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        step()
