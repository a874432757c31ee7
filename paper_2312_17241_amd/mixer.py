"""Operators of a token mixer beside the encoding: linear attention with a decay for each head, norms of queries and keys with the rotation by
their positions, the orthogonalised update of the matrices around them.  Argument marshalling only, as in the rest of the binding: see
include/cngp.h for what each call computes.

Tensors of one call lie on the current device; work goes to torch's current stream.  Workspaces that are not given are taken from
torch's allocator for the one call."""
import ctypes
from dataclasses import dataclass

import torch

from . import ZERO_GRADS, _check, _dev, _lib, _Marshalled, _stream, _TORCH_DT, _ws
from .operators import _maybe, _need, _on_current_device, _out, _room, _sequences

ATTEND_ROW_DECAY = 1
ROTATE_NORM, ROTATE_NEXT = 2, 4          # beside ZERO_GRADS = 1
_CALL_BWD, _CALL_RAGGED, _CALL_NO_DDECAY = 1, 2, 4


class CAttendConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("heads", "kv_heads", "key_dim", "value_dim", "io_dtype", "longest")] + [
        ("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


class CRotateConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("heads", "kv_heads", "dim", "axes")] + [
        ("pairs", ctypes.c_int32 * 4), ("io_dtype", ctypes.c_int32), ("eps", ctypes.c_float), ("flags", ctypes.c_uint32)]


class COrthoConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("batch", "rows", "cols", "io_dtype", "steps")] + [
        (n, ctypes.c_float) for n in ("a", "b", "c", "eps")] + [("flags", ctypes.c_uint32)]


class CMuon(ctypes.Structure):
    _fields_ = [(n, ctypes.c_float) for n in ("lr", "momentum", "weight_decay", "grad_scale")] + [("nesterov", ctypes.c_int32)]


def _declare():
    vp, i64, sz, u32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_uint32
    for name, result, args in (
            ("cngp_attend_workspace_bytes", sz, [vp, i64, i64, u32]),
            ("cngp_attend_fwd", ctypes.c_int, [vp] * 5 + [i64, vp, i64] + [vp] * 4 + [sz, vp]),
            ("cngp_attend_bwd", ctypes.c_int, [vp] * 5 + [i64, vp, i64] + [vp] * 9 + [sz, vp]),
            ("cngp_rotate_workspace_bytes", sz, [vp, i64]),
            ("cngp_rotate_fwd", ctypes.c_int, [vp] * 3 + [i64] + [vp] * 7),
            ("cngp_rotate_bwd", ctypes.c_int, [vp] * 3 + [i64] + [vp] * 11 + [sz, vp]),
            ("cngp_orthogonalise_workspace_bytes", sz, [vp]),
            ("cngp_orthogonalise", ctypes.c_int, [vp] * 4 + [sz, vp]),
            ("cngp_muon_step", ctypes.c_int, [vp] * 6 + [ctypes.c_int, vp, sz, vp])):
        f = getattr(_lib, name)
        f.restype, f.argtypes = result, args


_declare()


@dataclass(frozen=True)
class AttendConfig(_Marshalled):
    """Linear attention with a decay for each head (cngp_attend_config)."""
    heads: int
    kv_heads: int
    key_dim: int
    value_dim: int
    io_dtype: int = 0
    longest: int = 0          # no sequence has more rows; 0 = unknown: as in RecurConfig
    scale: float = 1.0
    flags: int = 0            # ATTEND_ROW_DECAY

    def c(self):
        return CAttendConfig(self.heads, self.kv_heads, self.key_dim, self.value_dim, self.io_dtype, self.longest, self.scale, self.flags)


def _decay_shape(cfg, N):
    return (N, cfg.heads) if cfg.flags & ATTEND_ROW_DECAY else (cfg.heads,)


def attend_workspace_bytes(cfg: AttendConfig, N, sequences, backward=False, ragged=False, ddecay=True) -> int:
    """backward: of attend_bwd; ddecay: with the decays' gradient, which takes most of it."""
    return _need("cngp_attend_workspace_bytes", cfg, N, sequences, (_CALL_BWD if backward else 0) | (_CALL_RAGGED if ragged else 0) | (0 if ddecay else _CALL_NO_DDECAY))


def attend_fwd(cfg: AttendConfig, q, k, v, decay, h0=None, offsets=None, sequences=None, y=True, last=True, workspace=None):
    """cngp_attend_fwd: (y, last).  q [N, heads, key_dim], k [N, kv_heads, key_dim], v [N, kv_heads, value_dim], decay float32 [heads] or
    [N, heads].  y, last: True for a new tensor, a tensor to write, False / None if not wanted.  offsets int32 [sequences + 1], or None for
    `sequences` (1 unless given) of equal length.  Rows that belong to no sequence are left as they are in y, undefined in a new one."""
    N, io = k.shape[0], _TORCH_DT[cfg.io_dtype]
    S = _sequences(N, offsets, sequences)
    state = (S, cfg.heads, cfg.key_dim, cfg.value_dim)
    y, yp = _out(y, (N, cfg.heads, cfg.value_dim), io, k if q is None else q, "y")
    last, lp = _out(last, state, torch.float32, k if h0 is None else h0, "last")
    qp = _maybe(q, io, (N, cfg.heads, cfg.key_dim), "q")
    kp, vp = _dev(k, io, (N, cfg.kv_heads, cfg.key_dim), "k"), _dev(v, io, (N, cfg.kv_heads, cfg.value_dim), "v")
    dp, hp = _dev(decay, torch.float32, _decay_shape(cfg, N), "decay"), _maybe(h0, torch.float32, state, "h0")
    op = _maybe(offsets, torch.int32, (S + 1,), "offsets")
    _on_current_device(q, k, v, decay, h0, offsets, y, last, workspace)
    workspace = _room(_need("cngp_attend_workspace_bytes", cfg, N, S, 0 if offsets is None else _CALL_RAGGED), workspace, k)
    _check(_lib.cngp_attend_fwd(cfg._ref(), qp, kp, vp, dp, N, op, S, hp, yp, lp, *_ws(workspace), _stream()))
    return y, last


def attend_bwd(cfg: AttendConfig, q, k, v, decay, dy=None, dlast=None, h0=None, offsets=None, sequences=None, dq=True, dk=True, dv=True, ddecay=True,
               dh0=None, workspace=None):
    """cngp_attend_bwd: (dq, dk, dv, ddecay, dh0).  dh0: as `last` of the forward; None gives one where h0 is given.  Rows that belong to no
    sequence are left as they are in the gradients, undefined in new ones."""
    N, io = q.shape[0], _TORCH_DT[cfg.io_dtype]
    S = _sequences(N, offsets, sequences)
    state = (S, cfg.heads, cfg.key_dim, cfg.value_dim)
    qs, ks, vs = (N, cfg.heads, cfg.key_dim), (N, cfg.kv_heads, cfg.key_dim), (N, cfg.kv_heads, cfg.value_dim)
    qp, kp, vp = _dev(q, io, qs, "q"), _dev(k, io, ks, "k"), _dev(v, io, vs, "v")
    gp, hp = _dev(decay, torch.float32, _decay_shape(cfg, N), "decay"), _maybe(h0, torch.float32, state, "h0")
    op = _maybe(offsets, torch.int32, (S + 1,), "offsets")
    dyp, dlp = _maybe(dy, io, (N, cfg.heads, cfg.value_dim), "dy"), _maybe(dlast, torch.float32, state, "dlast")
    dq, dqp = _out(dq, qs, io, q, "dq")
    dk, dkp = _out(dk, ks, io, k, "dk")
    dv, dvp = _out(dv, vs, io, v, "dv")
    ddecay, ddp = _out(ddecay, _decay_shape(cfg, N), torch.float32, decay, "ddecay")
    dh0, dhp = _out(h0 is not None if dh0 is None else dh0, state, torch.float32, q if h0 is None else h0, "dh0")
    _on_current_device(q, k, v, decay, dy, dlast, h0, offsets, dq, dk, dv, ddecay, dh0, workspace)
    workspace = _room(attend_workspace_bytes(cfg, N, S, True, offsets is not None, ddecay is not None), workspace, q)
    _check(_lib.cngp_attend_bwd(cfg._ref(), qp, kp, vp, gp, N, op, S, hp, dyp, dlp, dqp, dkp, dvp, ddp, dhp, *_ws(workspace), _stream()))
    return dq, dk, dv, ddecay, dh0


@dataclass(frozen=True)
class RotateConfig(_Marshalled):
    """Norms and rotation of queries and keys (cngp_rotate_config); pairs: how many each axis turns."""
    heads: int
    kv_heads: int
    dim: int
    pairs: tuple
    io_dtype: int = 0
    eps: float = 1e-6
    flags: int = 0            # ROTATE_NORM | ROTATE_NEXT | ZERO_GRADS

    def c(self):
        if not 1 <= len(self.pairs) <= 4:
            raise ValueError("pairs must name one to four axes")
        return CRotateConfig(self.heads, self.kv_heads, self.dim, len(self.pairs), (ctypes.c_int32 * 4)(*self.pairs), self.io_dtype, self.eps, self.flags)


def rotate_workspace_bytes(cfg: RotateConfig, N) -> int:
    return _need("cngp_rotate_workspace_bytes", cfg, N)


def _angles(cfg, N, position, omega):
    pairs = sum(cfg.pairs)
    if not pairs:
        return None, None
    return _dev(position, torch.float32, (N, len(cfg.pairs)), "position"), _dev(omega, torch.float32, (pairs,), "omega")


def rotate_fwd(cfg: RotateConfig, q, k, position, omega, gamma_q=None, gamma_k=None, q_out=True, k_out=True):
    """cngp_rotate_fwd: (q_out, k_out).  q [N, heads, dim], k [N, kv_heads, dim] (None where the config has no such heads), position float32
    [N, axes], omega float32 [pairs].  q_out, k_out: True for a new tensor, or a tensor to write, which may be the input."""
    N, io, D = (k if q is None else q).shape[0], _TORCH_DT[cfg.io_dtype], cfg.dim
    qs, ks = (N, cfg.heads, D), (N, cfg.kv_heads, D)
    qp, kp = _dev(q, io, qs, "q") if cfg.heads else None, _dev(k, io, ks, "k") if cfg.kv_heads else None
    q_out, qo = _out(bool(cfg.heads) and q_out, qs, io, q, "q_out")
    k_out, ko = _out(bool(cfg.kv_heads) and k_out, ks, io, k, "k_out")
    pp, wp = _angles(cfg, N, position, omega)
    gq, gk = _maybe(gamma_q, torch.float32, (D,), "gamma_q"), _maybe(gamma_k, torch.float32, (D,), "gamma_k")
    _on_current_device(q, k, position, omega, gamma_q, gamma_k, q_out, k_out)
    _check(_lib.cngp_rotate_fwd(cfg._ref(), qp, kp, N, pp, wp, gq, gk, qo, ko, _stream()))
    return q_out, k_out


def rotate_bwd(cfg: RotateConfig, q, k, position, omega, dq_out, dk_out, gamma_q=None, gamma_k=None, dq=True, dk=True, dgamma_q=None, dgamma_k=None,
               workspace=None):
    """cngp_rotate_bwd: (dq, dk, dgamma_q, dgamma_k).  q, k: the forward's inputs (ROTATE_NORM only, else unused).  dq, dk: True for a new
    tensor, or a tensor to write, which may be dq_out / dk_out.  dgamma_q, dgamma_k: a tensor to accumulate into (or write, with ZERO_GRADS);
    None gives one where there is a gamma; False: not wanted."""
    N, io, D = (dk_out if dq_out is None else dq_out).shape[0], _TORCH_DT[cfg.io_dtype], cfg.dim
    qs, ks, norm = (N, cfg.heads, D), (N, cfg.kv_heads, D), bool(cfg.flags & ROTATE_NORM)
    qp, kp = _dev(q, io, qs, "q") if cfg.heads and norm else None, _dev(k, io, ks, "k") if cfg.kv_heads and norm else None
    dqo, dko = _dev(dq_out, io, qs, "dq_out") if cfg.heads else None, _dev(dk_out, io, ks, "dk_out") if cfg.kv_heads else None
    dq, dqp = _out(bool(cfg.heads) and dq, qs, io, dq_out, "dq")
    dk, dkp = _out(bool(cfg.kv_heads) and dk, ks, io, dk_out, "dk")
    gains = []
    for given, gamma, heads, name in ((dgamma_q, gamma_q, cfg.heads, "dgamma_q"), (dgamma_k, gamma_k, cfg.kv_heads, "dgamma_k")):
        if given is None and gamma is not None and norm and heads:
            given = gamma.new_empty(D) if cfg.flags & ZERO_GRADS else gamma.new_zeros(D)
        gains.append(_out(given, (D,), torch.float32, gamma, name))
    (dgamma_q, dgq), (dgamma_k, dgk) = gains
    pp, wp = _angles(cfg, N, position, omega)
    gq, gk = _maybe(gamma_q, torch.float32, (D,), "gamma_q"), _maybe(gamma_k, torch.float32, (D,), "gamma_k")
    _on_current_device(q, k, position, omega, gamma_q, gamma_k, dq_out, dk_out, dq, dk, dgamma_q, dgamma_k, workspace)
    if dgq or dgk:
        workspace = _room(rotate_workspace_bytes(cfg, N), workspace, dk_out if dq_out is None else dq_out)
    _check(_lib.cngp_rotate_bwd(cfg._ref(), qp, kp, N, pp, wp, gq, gk, dqo, dko, dqp, dkp, dgq, dgk, *_ws(workspace), _stream()))
    return dq, dk, dgamma_q, dgamma_k


@dataclass(frozen=True)
class OrthoConfig(_Marshalled):
    """Orthogonalised updates of `batch` matrices [rows, cols] (cngp_ortho_config)."""
    rows: int
    cols: int
    batch: int = 1
    io_dtype: int = 0
    steps: int = 5
    coefficients: tuple = (3.4445, -4.7750, 2.0315)
    eps: float = 1e-7

    def c(self):
        return COrthoConfig(self.batch, self.rows, self.cols, self.io_dtype, self.steps, *self.coefficients, self.eps, 0)


def orthogonalise_workspace_bytes(cfg: OrthoConfig) -> int:
    return _need("cngp_orthogonalise_workspace_bytes", cfg)


def orthogonalise(cfg: OrthoConfig, g, out=True, workspace=None):
    """cngp_orthogonalise of g [batch, rows, cols]; out: True for a new tensor, or a tensor to write, which may be g."""
    shape, io = (cfg.batch, cfg.rows, cfg.cols), _TORCH_DT[cfg.io_dtype]
    gp = _dev(g, io, shape, "g")
    out, op = _out(out, shape, io, g, "out")
    _on_current_device(g, out, workspace)
    workspace = _room(orthogonalise_workspace_bytes(cfg), workspace, g)
    _check(_lib.cngp_orthogonalise(cfg._ref(), gp, op, *_ws(workspace), _stream()))
    return out


@dataclass
class Muon:
    """Hyper-parameters of an orthogonalised optimiser step (cngp_muon)."""
    lr: float = 2e-2
    momentum: float = 0.95
    weight_decay: float = 0.0
    grad_scale: float = 1.0
    nesterov: bool = True

    def c(self):
        return CMuon(self.lr, self.momentum, self.weight_decay, self.grad_scale, int(self.nesterov))


def muon_step(cfg: OrthoConfig, opt: Muon, master, half_copy, m, grad, clear_grad=False, workspace=None):
    """cngp_muon_step on float32 matrices [batch, rows, cols] (or [rows, cols] of one); half_copy (float16, same shape) may be None.
    Updates master and m in place."""
    shape = (cfg.rows, cfg.cols) if cfg.batch == 1 and master.dim() == 2 else (cfg.batch, cfg.rows, cfg.cols)
    mp, sp, gp = _dev(master, torch.float32, shape, "master"), _dev(m, torch.float32, shape, "m"), _dev(grad, torch.float32, shape, "grad")
    hp = _maybe(half_copy, torch.float16, shape, "half_copy")
    _on_current_device(master, half_copy, m, grad, workspace)
    workspace = _room(orthogonalise_workspace_bytes(cfg), workspace, master)
    o = opt.c()
    _check(_lib.cngp_muon_step(cfg._ref(), ctypes.byref(o), mp, hp, sp, gp, int(bool(clear_grad)), *_ws(workspace), _stream()))
