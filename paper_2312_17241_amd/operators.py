"""Operators around the encoding: the gated linear recurrence, the lookup of codes with its gradient, the balance of the probing
candidates.  Argument marshalling only, as in the rest of the binding: see include/cngp.h for what each call computes.

Tensors of one call lie on the current device; work goes to torch's current stream.  Workspaces that are not given are taken from
torch's allocator for the one call."""
import ctypes
from dataclasses import dataclass

import torch

from . import (ZERO_GRADS, _check, _dev, _lib, _Marshalled, _stream, _TORCH_DT, _ws)

I32, I64 = 0, 1
RECUR_REVERSE, RECUR_LOG_GATE, RECUR_MIX = 1, 2, 4
_CALL_BWD, _CALL_RAGGED, _CALL_NO_Y = 1, 2, 4
_ID_DT = {I32: torch.int32, I64: torch.int64}


class CRecurConfig(ctypes.Structure):
    _fields_ = [("channels", ctypes.c_int32), ("gate_channels", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
                ("gate_dtype", ctypes.c_int32), ("longest", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class CEmbedConfig(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("dim", ctypes.c_int32), ("table_dtype", ctypes.c_int32), ("io_dtype", ctypes.c_int32),
                ("id_dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


def _declare():
    vp, i64, sz, u32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_uint32
    for name, result, args in (
            ("cngp_recur_workspace_bytes", sz, [vp, i64, i64, u32]),
            ("cngp_recur_fwd", ctypes.c_int, [vp, vp, vp, i64, vp, i64, vp, vp, vp, vp, sz, vp]),
            ("cngp_recur_bwd", ctypes.c_int, [vp, vp, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]),
            ("cngp_embed_workspace_bytes", sz, [vp, i64]),
            ("cngp_embed_fwd", ctypes.c_int, [vp, vp, i64, vp, vp, vp, vp]),
            ("cngp_embed_bwd", ctypes.c_int, [vp, vp, i64, vp, vp, vp, sz, vp]),
            ("cngp_probe_balance_workspace_bytes", sz, [vp]),
            ("cngp_probe_balance", ctypes.c_int, [vp, vp, vp, ctypes.c_float, vp, vp, vp, vp, sz, vp])):
        f = getattr(_lib, name)
        f.restype, f.argtypes = result, args


_declare()


@dataclass(frozen=True)
class RecurConfig(_Marshalled):
    """A gated linear recurrence (cngp_recur_config); gate_channels is channels or 1."""
    channels: int
    gate_channels: int
    io_dtype: int = 0
    gate_dtype: int = 0
    longest: int = 0          # no sequence has more rows; 0 = unknown: one far longer than four times the mean is then walked alone, and slowly
    flags: int = 0            # RECUR_REVERSE | RECUR_LOG_GATE | RECUR_MIX

    def c(self):
        return CRecurConfig(self.channels, self.gate_channels, self.io_dtype, self.gate_dtype, self.longest, self.flags)


@dataclass(frozen=True)
class EmbedConfig(_Marshalled):
    """A table of codes (cngp_embed_config)."""
    rows: int
    dim: int
    table_dtype: int = 0
    io_dtype: int = 0
    id_dtype: int = I64
    scale: float = 1.0
    flags: int = 0            # ZERO_GRADS

    def c(self):
        return CEmbedConfig(self.rows, self.dim, self.table_dtype, self.io_dtype, self.id_dtype, self.scale, self.flags)


_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)      # the number alone: 0.1 us against 0.6


def _on_current_device(*tensors):
    """The kernels go to the current device's stream: a tensor of another device would be reached through the wrong one."""
    here = _device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"tensors must lie on the current device (cuda:{here}), got one on {t.device}")


def _maybe(t, dtype, shape, name):
    return None if t is None else _dev(t, dtype, shape, name)


def _room(need, workspace, like):
    """The workspace to pass: the caller's, or one for this call."""
    if workspace is None and need:
        workspace = like.new_empty(need, dtype=torch.uint8)
    return workspace


def _need(query, cfg, *sizes):
    """Bytes of a call's workspace, kept with the configuration: host arithmetic, but a microsecond through ctypes."""
    try:
        rooms = cfg._rooms
    except AttributeError:
        rooms = {}
        object.__setattr__(cfg, "_rooms", rooms)
    need = rooms.get((query, sizes))
    if need is None:
        if len(rooms) >= 256:
            rooms.clear()
        need = rooms[query, sizes] = int(getattr(_lib, query)(cfg._ref(), *sizes))
    return need


def _out(given, shape, dtype, like, name):
    """(tensor, pointer).  True: a new tensor, made from `like` where that has the shape and type (a third less time); a tensor: itself,
    checked; None / False: not wanted."""
    if given is True:
        given = torch.empty_like(like) if like.shape == shape and like.dtype is dtype else like.new_empty(shape, dtype=dtype)
        return given, given.data_ptr()
    if given is None or given is False:
        return None, None
    return given, _dev(given, dtype, shape, name)


def _sequences(N, offsets, sequences):
    if offsets is not None:
        if offsets.dim() != 1 or offsets.shape[0] < 1:
            raise ValueError("offsets must have sequences + 1 entries")
        count = offsets.shape[0] - 1
        if sequences is not None and sequences != count:
            raise ValueError(f"offsets describe {count} sequences, not {sequences}")
        return count
    return 1 if sequences is None else sequences


def recur_workspace_bytes(cfg: RecurConfig, N, sequences, backward=False, ragged=False, with_y=True) -> int:
    call = (_CALL_BWD if backward else 0) | (_CALL_RAGGED if ragged else 0) | (0 if with_y or not backward else _CALL_NO_Y)
    return _need("cngp_recur_workspace_bytes", cfg, N, sequences, call)


def recur_fwd(cfg: RecurConfig, gate, x, h0=None, offsets=None, sequences=None, y=True, last=True, workspace=None):
    """cngp_recur_fwd: (y, last).  y, last: True for a new tensor, a tensor to write, False / None if not wanted.
    offsets int32 [sequences + 1], or None for `sequences` (1 unless given) of equal length."""
    N, C = x.shape
    S = _sequences(N, offsets, sequences)
    y, yp = _out(y, (N, C), _TORCH_DT[cfg.io_dtype], x, "y")
    last, lp = _out(last, (S, C), torch.float32, x if h0 is None else h0, "last")
    gp, xp = _dev(gate, _TORCH_DT[cfg.gate_dtype], (N, cfg.gate_channels), "gate"), _dev(x, _TORCH_DT[cfg.io_dtype], (N, cfg.channels), "x")
    hp, op = _maybe(h0, torch.float32, (S, C), "h0"), _maybe(offsets, torch.int32, (S + 1,), "offsets")
    _on_current_device(gate, x, h0, offsets, y, last, workspace)
    workspace = _room(_need("cngp_recur_workspace_bytes", cfg, N, S, 0 if offsets is None else _CALL_RAGGED), workspace, x)
    _check(_lib.cngp_recur_fwd(cfg._ref(), gp, xp, N, op, S, hp, yp, lp, *_ws(workspace), _stream()))
    return y, last


def recur_bwd(cfg: RecurConfig, gate, x, dy=None, dlast=None, h0=None, y=None, offsets=None, sequences=None, dgate=True, dx=True, dh0=None,
              workspace=None):
    """cngp_recur_bwd: (dgate, dx, dh0).  y: the forward's states if kept (else, and where they are fp16, computed again: the gates' gradient
    takes states in 32 bits).  dh0: as `last` of the forward; None gives one where h0 is given.  Rows that belong to no sequence are left as
    they are in the gradients, undefined in new ones."""
    N, C = x.shape
    S = _sequences(N, offsets, sequences)
    io, gt = _TORCH_DT[cfg.io_dtype], _TORCH_DT[cfg.gate_dtype]
    gp, xp = _dev(gate, gt, (N, cfg.gate_channels), "gate"), _dev(x, io, (N, cfg.channels), "x")
    hp, op, yp = _maybe(h0, torch.float32, (S, C), "h0"), _maybe(offsets, torch.int32, (S + 1,), "offsets"), _maybe(y, io, (N, C), "y")
    dyp, dlp = _maybe(dy, io, (N, C), "dy"), _maybe(dlast, torch.float32, (S, C), "dlast")
    dgate, dgp = _out(dgate, (N, cfg.gate_channels), gt, gate, "dgate")
    dx, dxp = _out(dx, (N, C), io, x, "dx")
    dh0, dhp = _out(h0 is not None if dh0 is None else dh0, (S, C), torch.float32, x if dlast is None else dlast, "dh0")
    _on_current_device(gate, x, h0, offsets, y, dy, dlast, dgate, dx, dh0, workspace)
    workspace = _room(recur_workspace_bytes(cfg, N, S, True, offsets is not None, y is not None), workspace, x)
    _check(_lib.cngp_recur_bwd(cfg._ref(), gp, xp, N, op, S, hp, yp, dyp, dlp, dgp, dxp, dhp, *_ws(workspace), _stream()))
    return dgate, dx, dh0


def embed_workspace_bytes(cfg: EmbedConfig, N) -> int:
    return _need("cngp_embed_workspace_bytes", cfg, N)


def embed_fwd(cfg: EmbedConfig, ids, table, base=None, y=None):
    """cngp_embed_fwd: base + scale * table[ids], io_dtype [N, dim]; y may be base (added in place)."""
    N, io = ids.shape[0], _TORCH_DT[cfg.io_dtype]
    y, yp = _out(True if y is None else y, (N, cfg.dim), io, ids if base is None else base, "y")
    ip, tp = _dev(ids, _ID_DT[cfg.id_dtype], (N,), "ids"), _dev(table, _TORCH_DT[cfg.table_dtype], (cfg.rows, cfg.dim), "table")
    bp = _maybe(base, io, (N, cfg.dim), "base")
    _on_current_device(ids, table, base, y)
    _check(_lib.cngp_embed_fwd(cfg._ref(), ip, N, tp, bp, yp, _stream()))
    return y


def embed_bwd(cfg: EmbedConfig, ids, dy, grad_table=None, workspace=None):
    """cngp_embed_bwd: float32 [rows, dim], accumulated into grad_table if given (written with ZERO_GRADS)."""
    N = ids.shape[0]
    if grad_table is None:
        make = torch.empty if cfg.flags & ZERO_GRADS else torch.zeros
        grad_table = make((cfg.rows, cfg.dim), dtype=torch.float32, device=ids.device)
    ip, dp = _dev(ids, _ID_DT[cfg.id_dtype], (N,), "ids"), _dev(dy, _TORCH_DT[cfg.io_dtype], (N, cfg.dim), "dy")
    gp = _dev(grad_table, torch.float32, (cfg.rows, cfg.dim), "grad_table")
    _on_current_device(ids, dy, grad_table, workspace)
    workspace = _room(embed_workspace_bytes(cfg, N), workspace, ids)
    _check(_lib.cngp_embed_bwd(cfg._ref(), ip, N, dp, gp, *_ws(workspace), _stream()))
    return grad_table


def probe_balance_workspace_bytes(cfg) -> int:
    return _need("cngp_probe_balance_workspace_bytes", cfg)


def probe_balance(cfg, Dhat_c, weight=1.0, rows=None, grad_Dhat_c=True, loss=None, counts=None, workspace=None):
    """cngp_probe_balance: (loss [L], counts int32 [L, N_p], grad_Dhat_c).  grad_Dhat_c: True for a new one, a tensor to accumulate into
    (or to write, with ZERO_GRADS), False / None if not wanted.  rows: uint8 [L, N_c], 0 = not counted."""
    shape = (cfg.L, cfg.N_c, cfg.N_p)
    dp = _dev(Dhat_c, torch.float32, shape, "Dhat_c")
    loss, lp = _out(True if loss is None else loss, (cfg.L,), torch.float32, Dhat_c, "loss")
    counts, cp = _out(True if counts is None else counts, (cfg.L, cfg.N_p), torch.int32, Dhat_c, "counts")
    if grad_Dhat_c is True and not cfg.flags & ZERO_GRADS:
        grad_Dhat_c = torch.zeros(shape, dtype=torch.float32, device=Dhat_c.device)
    grad_Dhat_c, gp = _out(grad_Dhat_c, shape, torch.float32, Dhat_c, "grad_Dhat_c")
    rp = _maybe(rows, torch.uint8, (cfg.L, cfg.N_c), "rows")
    _on_current_device(Dhat_c, rows, loss, counts, grad_Dhat_c, workspace)
    workspace = _room(probe_balance_workspace_bytes(cfg), workspace, Dhat_c)
    _check(_lib.cngp_probe_balance(cfg._ref(), dp, rp, float(weight), lp, cp, gp, *_ws(workspace), _stream()))
    return loss, counts, grad_Dhat_c
