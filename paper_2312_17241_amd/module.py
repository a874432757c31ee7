"""torch.nn.Modules and autograd functions around the library's entry points, for training loops: the encoding, codes per image or
object that are added to it, the recurrence that composites a ray's decoded samples, and the mixer of a ray's or sequence's rows (attention with
decays, norms and rotation of its queries and keys).

Holds the codebooks of the encoding (Sec. 3: feature codebook D_f, confidence values D^_c, baked index
codebook D_c), their gradient arrays and optimiser moments as device tensors, and wires encode_fwd /
encode_bwd into autograd so that a decoder written in PyTorch can be trained on top of it.  Marshalling
only: every operation on the codebooks runs in the library's kernels (forward, backward, optimiser step
fused with the bake); nothing here computes on them with PyTorch.

Choices the paper leaves open (stated, not claimed): D_f starts uniform in +-1e-4 as in the hash-grid
encoding the method extends; D^_c starts uniform in +-1e-4 (every candidate nearly equally likely, the
first bake picks an arbitrary one); the optimiser is Adam.
"""
import functools

import torch
from torch.autograd.function import once_differentiable

from . import (Adam, AttendConfig, Config, EmbedConfig, F32, I64, RECUR_LOG_GATE, RECUR_MIX, RECUR_REVERSE, RecurConfig, RotateConfig, ZERO_GRADS,
               _TORCH_DT, F16, adam_step, adam_step_bake, alloc_workspace, attend_bwd, attend_fwd, bake_probes, embed_bwd, embed_fwd, encode_bwd,
               encode_bwd_input, encode_fwd, probe_balance, recur_bwd, recur_fwd, rotate_bwd, rotate_fwd, workspace_bytes)


class _Encode(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, hook, enc):
        ctx.enc = enc
        ctx.save_for_backward(x)
        return encode_fwd(enc.cfg, x, enc.D_f, enc.D_c, workspace=enc._workspace(x.shape[0]))

    @staticmethod
    def backward(ctx, dy):
        enc = ctx.enc
        (x,) = ctx.saved_tensors
        dy = dy.contiguous().to(_TORCH_DT[enc.cfg.io_dtype])
        encode_bwd(enc.cfg, x, enc.D_f, enc.Dhat_c, dy, enc.grad_D_f, enc.grad_Dhat_c,
                   workspace=enc._workspace(x.shape[0]))          # accumulates (+=)
        grad_x = encode_bwd_input(enc.cfg, x, enc.D_f, enc.D_c, dy) if ctx.needs_input_grad[0] else None
        return grad_x, torch.zeros((), dtype=torch.float32, device=dy.device), None


class Encoding(torch.nn.Module):
    """y = enc(x): x float32 [N, d] in [0,1]^d -> [N, L*F].  Call enc.step(opt_f, opt_c) after backward()."""

    def __init__(self, cfg: Config, device="cuda", seed=0):
        super().__init__()
        if cfg.flags & ZERO_GRADS:
            raise ValueError("the module accumulates gradients across backward calls: pass a Config without ZERO_GRADS")
        self.cfg = cfg
        g = torch.Generator(device="cpu").manual_seed(seed)
        fs, cs = (cfg.L, cfg.N_f, cfg.F), (cfg.L, cfg.N_c, cfg.N_p)
        uni = lambda shape: ((torch.rand(shape, generator=g) * 2 - 1) * 1e-4).to(device)
        self.D_f_master = uni(fs)
        self.D_f = self.D_f_master.half() if cfg.feat_dtype == F16 else self.D_f_master
        self.Dhat_c = uni(cs)
        self.D_c = bake_probes(cfg, self.Dhat_c)
        zeros = lambda shape: torch.zeros(shape, dtype=torch.float32, device=device)
        self.grad_D_f, self.m_f, self.v_f = zeros(fs), zeros(fs), zeros(fs)
        self.grad_Dhat_c, self.m_c, self.v_c = zeros(cs), zeros(cs), zeros(cs)
        self._hook = torch.nn.Parameter(torch.zeros((), device=device))   # lets autograd reach backward()
        self._ws = None
        self._ws_n = -1
        self.steps = 0

    def _workspace(self, n):
        if n != self._ws_n:
            need = workspace_bytes(self.cfg, n)
            if self._ws is None or self._ws.numel() < need:
                self._ws = alloc_workspace(self.cfg, n, self.D_f.device)
            self._ws_n = n
        return self._ws

    def forward(self, x):
        return _Encode.apply(x, self._hook, self)

    def balance(self, weight, rows=None):
        """Adds the gradient of weight * sum(loss) to that of the confidence values, loss as in cngp_probe_balance, and returns
        (loss [L], winners per candidate [L, N_p]).  Call it after backward(), before step().  rows: uint8 [L, N_c], 0 = not counted."""
        loss, counts, _ = probe_balance(self.cfg, self.Dhat_c, weight, rows=rows, grad_Dhat_c=self.grad_Dhat_c)
        return loss, counts

    def step(self, opt_f: Adam, opt_c: Adam):
        """Optimiser step on both codebooks fused with the bake; clears the gradient arrays."""
        self.steps += 1
        of = Adam(opt_f.lr, opt_f.beta1, opt_f.beta2, opt_f.eps, opt_f.grad_scale, self.steps)
        oc = Adam(opt_c.lr, opt_c.beta1, opt_c.beta2, opt_c.eps, opt_c.grad_scale, self.steps)
        cfg = Config(**{**self.cfg.__dict__, "flags": self.cfg.flags | ZERO_GRADS})
        half = self.D_f if self.cfg.feat_dtype == F16 else None
        adam_step_bake(cfg, of, oc, (self.D_f_master, half, self.m_f, self.v_f, self.grad_D_f),
                       (self.Dhat_c, self.m_c, self.v_c, self.grad_Dhat_c, self.D_c))


class _LookUp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, base, hook, codes, ids):
        ctx.codes, ctx.has_base = codes, base is not None
        ctx.save_for_backward(ids)
        return embed_fwd(codes.cfg, ids, codes.table, base=base)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        dy = dy.contiguous()
        if ctx.needs_input_grad[1]:                                              # frozen codes: the gradient of base alone
            embed_bwd(ctx.codes.cfg, *ctx.saved_tensors, dy, ctx.codes.grad_table)  # accumulates (+=)
        return (dy if ctx.has_base else None), None, None, None


class Codes(torch.nn.Module):
    """A code per image, object or token: y = codes(ids, base) = base + scale * table[ids], base the encodings [N, dim] (or None).
    Ids outside the table are padding.  Call codes.step(opt) after backward().  After codes.requires_grad_(False) the table collects no gradient."""

    def __init__(self, rows, dim, io_dtype=F32, id_dtype=I64, scale=1.0, device="cuda", seed=0):
        super().__init__()
        self.cfg = EmbedConfig(rows, dim, F32, io_dtype, id_dtype, scale)
        g = torch.Generator(device="cpu").manual_seed(seed)
        # entries of an Adam step are moved four at a time: an array of its own, on 16 bytes
        self.table = ((torch.rand((rows, dim), generator=g) * 2 - 1) * 1e-4).to(device)
        zeros = lambda: torch.zeros((rows, dim), dtype=torch.float32, device=device)
        self.grad_table, self.m, self.v = zeros(), zeros(), zeros()
        self._hook = torch.nn.Parameter(torch.zeros((), device=device))         # lets autograd reach backward()
        self.steps = 0

    def forward(self, ids, base=None):
        # a leaf of its own for every call: one that an earlier graph holds would bind a captured backward to that graph's stream
        return _LookUp.apply(base, self._hook.detach().requires_grad_(self._hook.requires_grad), self, ids)

    def step(self, opt: Adam):
        """Adam on the table (every entry: those that no id chose too); clears the gradient."""
        self.steps += 1
        adam_step(Adam(opt.lr, opt.beta1, opt.beta2, opt.eps, opt.grad_scale, self.steps), self.table, None, self.m, self.v, self.grad_table,
                  clear_grad=True)


class _Recur(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate, x, h0, cfg, offsets, sequences, keep):
        y, last = recur_fwd(cfg, gate, x, h0=h0, offsets=offsets, sequences=sequences, y=keep)
        if y is not None and offsets is not None:                                # rows of no sequence are not written
            rows = torch.arange(x.shape[0], device=x.device)
            y.masked_fill_(((rows < offsets[0]) | (rows >= offsets[-1]))[:, None], 0.0)
        ctx.cfg, ctx.sequences, ctx.keep = cfg, sequences, keep
        ctx.set_materialize_grads(False)                                         # an output that the loss does not use costs no zeros
        ctx.save_for_backward(gate, x, h0, offsets, y)
        return (y, last) if keep else last

    @staticmethod
    @once_differentiable
    def backward(ctx, *grads):
        gate, x, h0, offsets, y = ctx.saved_tensors
        dy, dlast = grads if ctx.keep else (None, grads[0])
        if dy is None and dlast is None:
            return (None,) * 7
        dy = None if dy is None else dy.contiguous()
        dlast = None if dlast is None else dlast.contiguous()
        make = torch.empty_like if offsets is None else torch.zeros_like         # rows of no sequence have gradient 0
        dgate, dx, dh0 = recur_bwd(ctx.cfg, gate, x, dy=dy, dlast=dlast, h0=h0, y=y, offsets=offsets, sequences=ctx.sequences,
                                   dgate=make(gate), dx=make(x))
        return dgate, dx, dh0, None, None, None, None


def recur(cfg: RecurConfig, gate, x, h0=None, offsets=None, sequences=None, keep=True):
    """The gated linear recurrence with gradients: (y, last), or last alone with keep=False (then the states are computed again by the
    backward pass).  See cngp_recur_fwd.  As with any torch function, a backward pass is captured into a graph together with its forward, while no
    eager graph of the same gate, x or h0 lives."""
    return _Recur.apply(gate, x, h0, cfg, offsets, sequences, keep)


@functools.lru_cache(maxsize=64)
def _composite_config(channels, colour, depth, longest):
    code = {t: c for c, t in _TORCH_DT.items()}
    for name, dtype in (("colour", colour), ("depth", depth)):
        if dtype not in code:
            raise TypeError(f"{name} must be float32 or float16, got {dtype}")
    return RecurConfig(channels, 1, code[colour], code[depth], longest, RECUR_LOG_GATE | RECUR_MIX | RECUR_REVERSE)


def composite(depth, colour, background=None, offsets=None, rays=None, longest=0):
    """Pixels [rays, C] float32 of rays whose samples lie one behind the other, nearest first: depth [N] are the samples' optical depths
    (density times step, >= 0), colour [N, C] what they emit, background [rays, C] float32 what lies behind (None: black).
    offsets int32 [rays + 1], or None for `rays` rays of equal length; longest: most samples of a ray, to be given where a few rays may have
    very many (without it a ray of 2^20 samples among 4095 of 64 takes 8 ms in place of 30 us)."""
    if depth.dim() != 1 or colour.dim() != 2:
        raise ValueError(f"depth must be [N] and colour [N, C], got {tuple(depth.shape)} and {tuple(colour.shape)}")
    cfg = _composite_config(colour.shape[1], colour.dtype, depth.dtype, longest)
    return recur(cfg, -depth[:, None], colour, background, offsets, rays, keep=False)


class _Attend(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, decay, h0, cfg, offsets, sequences):
        y, last = attend_fwd(cfg, q, k, v, decay, h0=h0, offsets=offsets, sequences=sequences)
        if offsets is not None:                                                  # rows of no sequence are not written
            rows = torch.arange(q.shape[0], device=q.device)
            y.masked_fill_(((rows < offsets[0]) | (rows >= offsets[-1]))[:, None, None], 0.0)
        ctx.cfg, ctx.sequences = cfg, sequences
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(q, k, v, decay, h0, offsets)
        return y, last

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dlast):
        q, k, v, decay, h0, offsets = ctx.saved_tensors
        if dy is None and dlast is None:
            return (None,) * 8
        dy = None if dy is None else dy.contiguous()
        dlast = None if dlast is None else dlast.contiguous()
        make = torch.empty_like if offsets is None else torch.zeros_like         # rows of no sequence have gradient 0
        grads = attend_bwd(ctx.cfg, q, k, v, decay, dy=dy, dlast=dlast, h0=h0, offsets=offsets, sequences=ctx.sequences, dq=make(q), dk=make(k),
                           dv=make(v), ddecay=make(decay) if ctx.needs_input_grad[3] else False, dh0=h0 is not None and ctx.needs_input_grad[4])
        return (*grads[:3], *(g if need else None for g, need in zip(grads[3:], ctx.needs_input_grad[3:5])), None, None, None)


def attend(cfg: AttendConfig, q, k, v, decay, h0=None, offsets=None, sequences=None):
    """Linear attention with a decay per head, with gradients: (y, last).  See cngp_attend_fwd.  A backward pass is captured into a graph as with recur()."""
    return _Attend.apply(q, k, v, decay, h0, cfg, offsets, sequences)


class _Rotate(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, gamma_q, gamma_k, position, omega, cfg):
        ctx.cfg = cfg
        ctx.save_for_backward(q, k, gamma_q, gamma_k, position, omega)
        return rotate_fwd(cfg, q, k, position, omega, gamma_q, gamma_k)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk):
        q, k, gamma_q, gamma_k, position, omega = ctx.saved_tensors
        dq = dq if dq is None else dq.contiguous()
        dk = dk if dk is None else dk.contiguous()
        wanted = lambda i: None if ctx.needs_input_grad[i] else False
        return (*rotate_bwd(ctx.cfg, q, k, position, omega, dq, dk, gamma_q, gamma_k, dgamma_q=wanted(2), dgamma_k=wanted(3)), None, None, None)


def rotate(cfg: RotateConfig, q, k, position, omega, gamma_q=None, gamma_k=None):
    """Norms and rotation of queries and keys, with gradients of q, k and the gains: (q, k).  See cngp_rotate_fwd.  A backward pass is captured
    into a graph as with recur()."""
    for name, t in (("position", position), ("omega", omega)):
        if t is not None and t.requires_grad:
            raise ValueError(f"{name} gets no gradient: detach it")
    return _Rotate.apply(q, k, gamma_q, gamma_k, position, omega, cfg)
