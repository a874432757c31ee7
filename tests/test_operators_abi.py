"""What the operators around the encoding refuse, on the host: every check runs before anything is launched, so none of it needs a GPU."""
import ctypes

import pytest
import torch

import paper_2312_17241_amd as cngp

lib = cngp._lib
P = ctypes.c_void_p(4096)          # an aligned address that no refused call follows
OFF = ctypes.c_void_p(4100)
BIG = 1 << 40


def recur(**over):
    kw = dict(channels=8, gate_channels=8)
    kw.update(over)
    return cngp.RecurConfig(**kw)


def fwd(cfg, gate=P, x=P, N=6, offsets=None, S=3, h0=P, y=P, last=P, ws=P, size=BIG):
    return lib.cngp_recur_fwd(None if cfg is None else cfg._ref(), gate, x, N, offsets, S, h0, y, last, ws, size, None)


def bwd(cfg, gate=P, x=P, N=6, offsets=None, S=3, h0=P, y=P, dy=P, dlast=P, dgate=P, dx=P, dh0=P, ws=P, size=BIG):
    return lib.cngp_recur_bwd(None if cfg is None else cfg._ref(), gate, x, N, offsets, S, h0, y, dy, dlast, dgate, dx, dh0, ws, size, None)


@pytest.mark.parametrize("call", [fwd, bwd])
def test_recurrence_refuses(call):
    assert call(None) == cngp.ERR_NULL
    for over in (dict(channels=0), dict(channels=-1), dict(channels=65537, gate_channels=1), dict(gate_channels=2), dict(gate_channels=0),
                 dict(io_dtype=2), dict(gate_dtype=-1), dict(longest=-1), dict(flags=8)):
        assert call(recur(**over)) == cngp.ERR_INVALID, over
        assert cngp.recur_workspace_bytes(recur(**over), 6, 3, True) == 0
    for kw in (dict(N=-1), dict(N=2**31), dict(S=-1), dict(S=2**31 - 1, N=2**31 - 2), dict(S=4), dict(S=0)):
        assert call(recur(), **kw) == cngp.ERR_INVALID, kw
    for kw in (dict(gate=None), dict(x=None)):
        assert call(recur(), **kw) == cngp.ERR_NULL, kw
    assert call(recur(), S=0, N=0) == cngp.OK
    assert call(recur(), S=0, offsets=P) == cngp.OK            # no sequences: nothing to write


def test_recurrence_refuses_missing_outputs_and_workspaces():
    assert fwd(recur(), y=None, last=None) == cngp.ERR_NULL
    for kw in (dict(dy=None, dlast=None), dict(dgate=None), dict(dx=None)):
        assert bwd(recur(), **kw) == cngp.ERR_NULL, kw
    need = cngp.recur_workspace_bytes(recur(), 6, 3, True, False, False)
    assert need >= 6 * 8 * 4
    for kw in (dict(ws=None), dict(ws=OFF), dict(size=need - 1)):
        assert bwd(recur(), y=None, **kw) == cngp.ERR_WORKSPACE, kw


def test_recurrence_workspaces_grow_with_what_is_asked():
    for N, S in ((1, 1), (4096, 1), (2**17, 2**17), (2**20, 4), (20011, 1)):
        for C in (1, 3, 96, 1024):
            for G in {1, C}:
                cfg = recur(channels=C, gate_channels=G)
                for ragged in (False, True):
                    with_y = cngp.recur_workspace_bytes(cfg, N, S, True, ragged, True)
                    without = cngp.recur_workspace_bytes(cfg, N, S, True, ragged, False)
                    assert without >= with_y and with_y % 256 == 0 and without % 256 == 0
                    assert cngp.recur_workspace_bytes(cfg, N, S, False, ragged) % 256 == 0


def test_states_rounded_to_fp16_do_not_serve_fp32_gates():
    """The backward pass computes them again: it asks for the room of a call without them."""
    for io, gate, again in ((0, 0, False), (1, 1, False), (0, 1, False), (1, 0, True)):
        cfg = recur(io_dtype=io, gate_dtype=gate)
        room = lambda with_y: cngp.recur_workspace_bytes(cfg, 6, 3, True, False, with_y)
        assert (room(True) == room(False)) == again
        if again:
            assert bwd(cfg, ws=None) == cngp.ERR_WORKSPACE


def embed(**over):
    kw = dict(rows=10, dim=4)
    kw.update(over)
    return cngp.EmbedConfig(**kw)


def lookup(cfg, ids=P, N=5, table=P, base=P, y=P):
    return lib.cngp_embed_fwd(None if cfg is None else cfg._ref(), ids, N, table, base, y, None)


def lookup_bwd(cfg, ids=P, N=5, dy=P, grad=P, ws=P, size=BIG):
    return lib.cngp_embed_bwd(None if cfg is None else cfg._ref(), ids, N, dy, grad, ws, size, None)


@pytest.mark.parametrize("call", [lookup, lookup_bwd])
def test_lookup_refuses(call):
    assert call(None) == cngp.ERR_NULL
    for over in (dict(rows=0), dict(rows=2**31 - 1), dict(rows=-4), dict(dim=0), dict(dim=65537), dict(table_dtype=2), dict(io_dtype=-1),
                 dict(id_dtype=2), dict(scale=float("nan")), dict(scale=float("inf")), dict(flags=2)):
        assert call(embed(**over)) == cngp.ERR_INVALID, over
        assert cngp.embed_workspace_bytes(embed(**over), 5) == 0
    assert call(embed(), N=-1) == cngp.ERR_INVALID and call(embed(), N=2**31) == cngp.ERR_INVALID
    assert call(embed(), ids=None) == cngp.ERR_NULL
    assert call(embed(), N=0) == cngp.OK


def test_lookup_refuses_missing_arrays_and_workspaces():
    assert lookup(embed(), table=None) == cngp.ERR_NULL and lookup(embed(), y=None) == cngp.ERR_NULL
    assert lookup_bwd(embed(), dy=None) == cngp.ERR_NULL and lookup_bwd(embed(), grad=None) == cngp.ERR_NULL
    need = cngp.embed_workspace_bytes(embed(), 5)
    assert need > 0 and need % 256 == 0 and cngp.embed_workspace_bytes(embed(), 0) == 0
    for kw in (dict(ws=None), dict(ws=OFF), dict(size=need - 1)):
        assert lookup_bwd(embed(), **kw) == cngp.ERR_WORKSPACE, kw


def config(**over):
    kw = dict(d=3, L=4, F=2, N_f=2**8, N_c=2**6, N_p=8, N_min=4, N_max=64)
    kw.update(over)
    return cngp.Config(**kw)


def balance(cfg, v=P, rows=None, weight=1.0, loss=P, counts=P, grad=P, ws=P, size=BIG):
    return lib.cngp_probe_balance(None if cfg is None else cfg._ref(), v, rows, weight, loss, counts, grad, ws, size, None)


def test_balance_refuses():
    assert balance(None) == cngp.ERR_NULL
    assert balance(config(N_p=3)) == cngp.ERR_INVALID and balance(config(top_k=9)) == cngp.ERR_INVALID
    assert cngp.probe_balance_workspace_bytes(config(N_p=3)) == 0
    for kw in (dict(v=None), dict(loss=None), dict(counts=None)):
        assert balance(config(), **kw) == cngp.ERR_NULL, kw
    for w in (float("nan"), float("inf"), -float("inf")):
        assert balance(config(), weight=w) == cngp.ERR_INVALID
    assert cngp.probe_balance_workspace_bytes(config()) == 0               # a level of a few rows: one launch
    for big in (config(N_c=2**14), config(N_c=2**14, top_k=2)):
        need = cngp.probe_balance_workspace_bytes(big)
        assert need > 0 and need % 256 == 0
        for kw in (dict(ws=None), dict(ws=OFF), dict(size=need - 1)):
            assert balance(big, **kw) == cngp.ERR_WORKSPACE, kw


def test_binding_refuses_wrong_tensors():
    cfg, x = recur(), torch.zeros(6, 8)
    with pytest.raises(TypeError):
        cngp.recur_fwd(cfg, x, x)                              # host tensors
    with pytest.raises(ValueError):
        cngp.recur_fwd(cfg, x, x, offsets=torch.zeros(4, dtype=torch.int32), sequences=2)
    with pytest.raises(ValueError):
        cngp.recur_fwd(cfg, x, x, offsets=torch.zeros((2, 2), dtype=torch.int32))
    with pytest.raises(TypeError):
        cngp.embed_fwd(embed(), torch.zeros(5, dtype=torch.int64), torch.zeros(10, 4))
    with pytest.raises(TypeError):
        cngp.probe_balance(config(), torch.zeros(4, 64, 8))
