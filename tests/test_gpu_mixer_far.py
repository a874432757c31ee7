"""The mixer's operators on arrays of more than 2^32 values or bytes: what the far end holds is what a small call gives for the same rows."""
import pytest
import torch

import paper_2312_17241_amd as cngp

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(autouse=True)
def give_back():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_attention_and_rotation_of_more_than_2_to_32_values():
    H, D, T, S = 33, 128, 512, 2**11 + 1                   # sequences of equal rows: whole in both calls
    g = torch.Generator(device=DEV).manual_seed(1)
    make = lambda *s: torch.randn(s, generator=g, device=DEV).half()
    q, k, v, decay = make(T, H, D), make(T, 1, D), make(T, 1, D), -torch.rand(T, H, generator=g, device=DEV)
    cfg = cngp.AttendConfig(H, 1, D, D, cngp.F16, scale=0.1, flags=cngp.ATTEND_ROW_DECAY)
    rcfg = cngp.RotateConfig(H, 1, D, (64,), cngp.F16, flags=cngp.ROTATE_NORM)
    position, omega = torch.rand(T, 1, generator=g, device=DEV) * 100, torch.rand(64, generator=g, device=DEV)
    turned = cngp.rotate_fwd(rcfg, q, k, position, omega)
    small, last = cngp.attend_fwd(cfg, q, k, v, decay)
    many = lambda t: t.repeat(S, *([1] * (t.dim() - 1)))
    assert S * T * H * D > 2**32
    Q, K, V, G = (many(t) for t in (q, k, v, decay))
    y, states = cngp.attend_fwd(cfg, Q, K, V, G, sequences=S, y=torch.empty_like(Q))
    for s in (0, 1, S // 2, S - 1):
        assert torch.equal(y[s * T:(s + 1) * T], small) and torch.equal(states[s], last[0]), s
    cngp.rotate_fwd(rcfg, Q, K, many(position), omega, q_out=y, k_out=K)
    for s in (0, 1, S // 2, S - 1):
        assert torch.equal(y[s * T:(s + 1) * T], turned[0]) and torch.equal(K[s * T:(s + 1) * T], turned[1]), s


def test_gradients_of_more_than_2_to_31_values():
    H, D, T, S = 33, 64, 512, 2**11 + 1
    g = torch.Generator(device=DEV).manual_seed(2)
    make = lambda *s: torch.randn(s, generator=g, device=DEV).half()
    q, k, v, dy, decay = make(T, H, D), make(T, 1, D), make(T, 1, D), make(T, H, D), -torch.rand(T, H, generator=g, device=DEV)
    cfg = cngp.AttendConfig(H, 1, D, D, cngp.F16, scale=0.1, flags=cngp.ATTEND_ROW_DECAY)
    small = cngp.attend_bwd(cfg, q, k, v, decay, dy=dy)
    many = lambda t: t.repeat(S, *([1] * (t.dim() - 1)))
    assert S * T * H * D > 2**31
    large = cngp.attend_bwd(cfg, many(q), many(k), many(v), many(decay), dy=many(dy), sequences=S)
    for s in (0, 1, S // 2, S - 1):
        for a, b in zip(small[:4], large[:4]):
            assert torch.equal(b[s * T:(s + 1) * T], a), s


def test_orthogonalising_more_than_2_to_31_values():
    m, batch = 16384, 9
    g = torch.Generator(device=DEV).manual_seed(3)
    G = torch.empty(batch, m, m, device=DEV)
    G[0] = torch.randn(m, m, generator=g, device=DEV)
    G[1:] = G[0]
    assert G.numel() > 2**31
    cfg = cngp.OrthoConfig(m, m, batch, steps=1)
    out = cngp.orthogonalise(cfg, G, out=G)
    # equal matrices; their tiles may be summed in other parts: 2^-22 of sums of 16384 products below 2^-6 each, times 4.8
    for i in range(1, batch):
        assert float((out[i] - out[0]).abs().max()) <= 1e-4 * float(out[0].abs().max())
    row = out[batch - 1, -1].double()
    assert bool(torch.isfinite(row).all()) and float(row.norm()) > 0


@pytest.mark.parametrize("io", [torch.float16, torch.float32])
def test_widest_heads_captured(io):
    """Workgroups with more LDS than is theirs unasked."""
    N, H, D = 600, 2, 128
    g = torch.Generator(device=DEV).manual_seed(4)
    make = lambda *s: torch.randn(s, generator=g, device=DEV).to(io)
    q, k, v, dy, decay = make(N, H, D), make(N, H, D), make(N, H, D), make(N, H, D), -torch.rand(N, H, generator=g, device=DEV)
    cfg = cngp.AttendConfig(H, H, D, D, cngp.F16 if io == torch.float16 else cngp.F32, scale=0.1, flags=cngp.ATTEND_ROW_DECAY)
    room = torch.empty(cngp.attend_workspace_bytes(cfg, N, 1, True), dtype=torch.uint8, device=DEV)

    def run():
        return cngp.attend_fwd(cfg, q, k, v, decay, workspace=room) + cngp.attend_bwd(cfg, q, k, v, decay, dy=dy, workspace=room)[:4]

    want = [t.clone() for t in run()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run()
    for _ in range(3):
        for t in out:
            t.zero_()
        room.fill_(255)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all(torch.equal(a, b) for a, b in zip(run(), want))
