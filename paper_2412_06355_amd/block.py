"""Python binding of a block's operators and of its training step (include/dendsn_block.h).

The gated delta rule (forward, backward, one token at a time), the root-mean-square norm
(forward in the rows' type or in 8 bits, backward) and an AdamW step over many tensors.  As in
the token-sequence binding, the functions named like the C entry points take the C arguments
(tensors in place of pointers); ``delta_rule``, ``rms_norm``, ``adamw`` and their companions
check shapes, allocate the outputs and call them.  Everything is computed by the library's HIP
kernels, on the current stream of the tensors' device, which has to be the current device; there
is no fallback.
"""

from __future__ import annotations

import ctypes
import dataclasses
import struct
from dataclasses import dataclass

from .binding import IO
from .binding import lib as _lib
from .sequence import _bytes, _check, _expect, _io_dtype, _nbytes, _ptr, _row_stride, _stream, _workspace, seq_lib

STATE = {"f32": 0, "e4m3": 1}
DELTA_CHUNK = 64   # steps between the delta rule's checkpoints
STATE_BLOCK = 256  # values that share a scale in 8-bit optimizer states

_DELTA_STRIDES = tuple(f"{n}_{d}" for n in ("q", "k", "v", "g", "beta", "o", "grad_o") for d in "tbh")


class dendsn_delta_cfg(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int64) for k in ("T", "batch", "H", "Hk", "K", "V") + _DELTA_STRIDES] + \
               [("io", ctypes.c_int32), ("scale", ctypes.c_float)]


class dendsn_norm_cfg(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int64) for k in ("N", "D", "ld_x", "ld_residual", "ld_y", "ld_sum", "ld_grad_y",
                                                 "ld_grad_sum", "ld_grad_x")] + \
               [("io", ctypes.c_int32), ("eps", ctypes.c_float)]


class dendsn_adamw_cfg(ctypes.Structure):
    _fields_ = [(k, ctypes.c_double) for k in ("lr", "beta1", "beta2", "eps", "weight_decay")] + \
               [("state", ctypes.c_int32)]


class dendsn_adamw_tensor(ctypes.Structure):
    _fields_ = [("n", ctypes.c_int64)] + \
               [(k, ctypes.c_void_p) for k in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")] + \
               [("grad_io", ctypes.c_int32)]


_P, _Z, _I64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64
_SIZE = ctypes.POINTER(ctypes.c_size_t)
_DELTA, _NORM, _ADAMW = (ctypes.POINTER(c) for c in (dendsn_delta_cfg, dendsn_norm_cfg, dendsn_adamw_cfg))

_SIGS = {
    "dendsn_delta_ckpt_bytes": (ctypes.c_int, [_DELTA, _SIZE]),
    "dendsn_delta_workspace_bytes": (ctypes.c_int, [_DELTA, ctypes.c_int32, _SIZE]),
    "dendsn_delta_forward": (ctypes.c_int, [_DELTA] + [_P] * 11 + [_Z, _P]),
    "dendsn_delta_backward": (ctypes.c_int, [_DELTA] + [_P] * 16 + [_Z, _P]),
    "dendsn_delta_step": (ctypes.c_int, [_DELTA] + [_P] * 5 + [_I64] + [_P] * 4),
    "dendsn_norm_forward": (ctypes.c_int, [_NORM] + [_P] * 7),
    "dendsn_norm_forward_e4m3": (ctypes.c_int, [_NORM] + [_P] * 8),
    "dendsn_norm_workspace_bytes": (ctypes.c_int, [_NORM, _SIZE]),
    "dendsn_norm_backward": (ctypes.c_int, [_NORM] + [_P] * 8 + [_Z, _P]),
    "dendsn_norm_backward_residual": (ctypes.c_int, [_NORM] + [_P] * 9 + [_Z, _P]),
    "dendsn_adamw_step": (ctypes.c_int, [_ADAMW, _P, _I64, _I64, _P, _P, ctypes.c_uint64, _P]),
}

BLOCK_EXPORTS = tuple(_SIGS)

_bound = None


def block_lib():
    """The library with this header's entry points bound (once)."""
    global _bound
    if _bound is None:
        seq_lib()
        handle = _lib()
        for name, (res, args) in _SIGS.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _bound = handle
    return _bound


# ---------------------------------------------------------------------------
# Gated delta rule
# ---------------------------------------------------------------------------
@dataclass(frozen=True)
class DeltaRuleConfig:
    """S[t] = a S[t-1] + k (beta (v - a S[t-1]^T k))^T and o[t] = scale S[t]^T q, a = exp(g), over T
    steps, batch sequences and H heads, whose states are K by V.  q and k have Hk heads (0: H), each
    shared by H / Hk of the others.  ``scale`` None: K^-0.5.  Tensors are [T, batch, heads, values]
    (g, beta: [T, batch, H]) views of any strides whose innermost one is 1 (g, beta: any)."""

    T: int
    batch: int
    H: int
    K: int
    V: int
    io: str = "f32"
    Hk: int = 0
    scale: float | None = None

    def with_(self, **kw) -> "DeltaRuleConfig":
        return dataclasses.replace(self, **kw)

    def to_c(self, q=None, k=None, v=None, g=None, beta=None, o=None, grad_o=None) -> dendsn_delta_cfg:
        """The C struct with the strides of the given tensors (None: contiguous)."""
        Hk, s = self.Hk or self.H, []
        for t, heads, width in ((q, Hk, self.K), (k, Hk, self.K), (v, self.H, self.V), (g, self.H, 1), (beta, self.H, 1),
                                (o, self.H, self.V), (grad_o, self.H, self.V)):
            s += (self.batch * heads * width, heads * width, width) if t is None else t.stride()[:3]
        return dendsn_delta_cfg(self.T, self.batch, self.H, Hk, self.K, self.V, *s, IO[self.io],
                                self.K ** -0.5 if self.scale is None else self.scale)


def dendsn_delta_ckpt_bytes(cfg: DeltaRuleConfig) -> int:
    return _bytes(block_lib().dendsn_delta_ckpt_bytes, ctypes.byref(cfg.to_c()))


def dendsn_delta_workspace_bytes(cfg: DeltaRuleConfig, backward: bool) -> int:
    return _bytes(block_lib().dendsn_delta_workspace_bytes, ctypes.byref(cfg.to_c()), int(backward))


def dendsn_delta_forward(cfg: DeltaRuleConfig, q, k, v, g, beta, s0, lengths, o, s_last, ckpt, workspace, stream=None):
    st = stream if stream is not None else _stream(q.device)
    _check(block_lib().dendsn_delta_forward(ctypes.byref(cfg.to_c(q, k, v, g, beta, o)), _ptr(q), _ptr(k), _ptr(v),
                                            _ptr(g), _ptr(beta), _ptr(s0), _ptr(lengths), _ptr(o), _ptr(s_last),
                                            _ptr(ckpt), _ptr(workspace), _nbytes(workspace), st))


def dendsn_delta_backward(cfg: DeltaRuleConfig, q, k, v, g, beta, lengths, ckpt, grad_o, grad_s_last, grad_q, grad_k,
                          grad_v, grad_g, grad_beta, grad_s0, workspace, stream=None):
    st = stream if stream is not None else _stream(q.device)
    _check(block_lib().dendsn_delta_backward(ctypes.byref(cfg.to_c(q, k, v, g, beta, None, grad_o)), _ptr(q), _ptr(k),
                                             _ptr(v), _ptr(g), _ptr(beta), _ptr(lengths), _ptr(ckpt), _ptr(grad_o),
                                             _ptr(grad_s_last), _ptr(grad_q), _ptr(grad_k), _ptr(grad_v), _ptr(grad_g),
                                             _ptr(grad_beta), _ptr(grad_s0), _ptr(workspace), _nbytes(workspace), st))


def _delta_step_cfg(cfg, q, k, v, g, beta, o):
    s = []
    for t in (q, k, v, g, beta, o):
        s += (0, *t.stride()[:2])
    return dendsn_delta_cfg(cfg.T, cfg.batch, cfg.H, cfg.Hk or cfg.H, cfg.K, cfg.V, *s, 0, 0, 0, IO[cfg.io],
                            cfg.K ** -0.5 if cfg.scale is None else cfg.scale)


def dendsn_delta_step(cfg: DeltaRuleConfig, q, k, v, g, beta, slots, state, o, stream=None):
    st = stream if stream is not None else _stream(q.device)
    c = _delta_step_cfg(cfg, q, k, v, g, beta, o)
    _check(block_lib().dendsn_delta_step(ctypes.byref(c), _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta),
                                         state.shape[0], _ptr(slots), _ptr(state), _ptr(o), st))


def _check_delta(cfg, lead, q, k, v, g, beta):
    """The inputs' shapes, types and device; returns (dtype, device)."""
    dt, dev, Hk = _io_dtype(cfg.io), q.device, cfg.Hk or cfg.H
    _expect(q, "q", (*lead, Hk, cfg.K), dt, dev, rows=True)
    _expect(k, "k", (*lead, Hk, cfg.K), dt, dev, rows=True)
    _expect(v, "v", (*lead, cfg.H, cfg.V), dt, dev, rows=True)
    for t, name in ((g, "g"), (beta, "beta")):
        if t is None or t.shape != (*lead, cfg.H) or t.dtype != dt or t.device != dev:
            raise ValueError(f"{name}: expected {(*lead, cfg.H)} {dt} on {dev}")
    return dt, dev


def delta_rule(cfg: DeltaRuleConfig, q, k, v, g, beta, s0=None, lengths=None, *, save_ckpt: bool = True, workspace=None):
    """Returns (o [T, batch, H, V] io, s_last [batch, H, K, V] fp32, ckpt or None).  ``s0``
    [batch, H, K, V] fp32 is the state before the first step (None: 0).  Steps at and past ``lengths``
    [batch] (int32) are no part of a sequence: o is 0 there and s_last the state before them.
    ``ckpt`` is what the backward needs."""
    import torch

    _, dev = _check_delta(cfg, (cfg.T, cfg.batch), q, k, v, g, beta)
    states = (cfg.batch, cfg.H, cfg.K, cfg.V)
    _expect(s0, "s0", states, torch.float32, dev, optional=True)
    _expect(lengths, "lengths", (cfg.batch,), torch.int32, dev, optional=True)
    st, fn = _stream(dev), block_lib()
    o = q.new_empty((cfg.T, cfg.batch, cfg.H, cfg.V))
    last = torch.empty(states, dtype=torch.float32, device=dev)
    c = cfg.to_c(q, k, v, g, beta, o)
    ckpt = None
    if save_ckpt:
        ckpt = torch.empty((_bytes(fn.dendsn_delta_ckpt_bytes, ctypes.byref(c)),), dtype=torch.uint8, device=dev)
    ws = _workspace(_bytes(fn.dendsn_delta_workspace_bytes, ctypes.byref(c), 0), workspace, dev)
    _check(fn.dendsn_delta_forward(ctypes.byref(c), _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(s0),
                                   _ptr(lengths), _ptr(o), _ptr(last), _ptr(ckpt), _ptr(ws), _nbytes(ws), st))
    return o, last, ckpt


def delta_rule_backward(cfg: DeltaRuleConfig, q, k, v, g, beta, lengths, ckpt, grad_o, grad_s_last=None, *,
                        workspace=None):
    """Returns a dict with grad_q, grad_k [T, batch, Hk, K], grad_v [T, batch, H, V], grad_g, grad_beta
    [T, batch, H] io and grad_s0 [batch, H, K, V] fp32, the gradients of sum(grad_o * o) +
    sum(grad_s_last * s_last)."""
    import torch

    dt, dev = _check_delta(cfg, (cfg.T, cfg.batch), q, k, v, g, beta)
    states = (cfg.batch, cfg.H, cfg.K, cfg.V)
    _expect(lengths, "lengths", (cfg.batch,), torch.int32, dev, optional=True)
    _expect(grad_o, "grad_o", (cfg.T, cfg.batch, cfg.H, cfg.V), dt, dev, rows=True)
    _expect(grad_s_last, "grad_s_last", states, torch.float32, dev, optional=True)
    st, fn = _stream(dev), block_lib()
    c = cfg.to_c(q, k, v, g, beta, None, grad_o)
    need = _bytes(fn.dendsn_delta_ckpt_bytes, ctypes.byref(c))
    if need and (ckpt is None or ckpt.dtype != torch.uint8 or ckpt.device != dev or not ckpt.is_contiguous()
                 or ckpt.numel() < need):
        raise ValueError(f"ckpt must be the forward's checkpoints: contiguous uint8 on {dev}, {need} bytes")
    lead = (cfg.T, cfg.batch)
    out = dict(grad_q=q.new_empty((*lead, cfg.Hk or cfg.H, cfg.K)), grad_k=q.new_empty((*lead, cfg.Hk or cfg.H, cfg.K)),
               grad_v=q.new_empty((*lead, cfg.H, cfg.V)), grad_g=q.new_empty((*lead, cfg.H)),
               grad_beta=q.new_empty((*lead, cfg.H)), grad_s0=torch.empty(states, dtype=torch.float32, device=dev))
    ws = _workspace(_bytes(fn.dendsn_delta_workspace_bytes, ctypes.byref(c), 1), workspace, dev)
    _check(fn.dendsn_delta_backward(ctypes.byref(c), _ptr(q), _ptr(k), _ptr(v), _ptr(g), _ptr(beta), _ptr(lengths),
                                    _ptr(ckpt), _ptr(grad_o), _ptr(grad_s_last), *(_ptr(t) for t in out.values()),
                                    _ptr(ws), _nbytes(ws), st))
    return out


def delta_rule_step(cfg: DeltaRuleConfig, q, k, v, g, beta, state, slots=None):
    """One token of each of cfg.batch requests (cfg.T = 1; q, k [batch, Hk, K], v [batch, H, V], g, beta
    [batch, H]): updates ``state`` [held, H, K, V] (fp32) in place at ``slots`` [batch] (int32; None:
    state b for request b) and returns o [batch, H, V].  A request whose slot is no row of
    ``state`` is idle: o is 0."""
    import torch

    _, dev = _check_delta(cfg, (cfg.batch,), q, k, v, g, beta)
    _expect(state, "state", (state.shape[0], cfg.H, cfg.K, cfg.V), torch.float32, dev)
    _expect(slots, "slots", (cfg.batch,), torch.int32, dev, optional=True)
    st = _stream(dev)
    o = q.new_empty((cfg.batch, cfg.H, cfg.V))
    c = _delta_step_cfg(cfg, q, k, v, g, beta, o)
    _check(block_lib().dendsn_delta_step(ctypes.byref(c), q.data_ptr(), k.data_ptr(), v.data_ptr(), g.data_ptr(),
                                         beta.data_ptr(), state.shape[0], _ptr(slots), state.data_ptr(), o.data_ptr(), st))
    return o


# ---------------------------------------------------------------------------
# Root-mean-square norm
# ---------------------------------------------------------------------------
@dataclass(frozen=True)
class RMSNormConfig:
    """y = s rstd weight over N rows of D values: s = x, or x + residual; rstd = (mean s^2 + eps)^-1/2."""

    N: int
    D: int
    io: str = "f32"
    eps: float = 1e-6

    def with_(self, **kw) -> "RMSNormConfig":
        return dataclasses.replace(self, **kw)

    def to_c(self, x=None, residual=None, y=None, sum=None, grad_y=None, grad_sum=None, grad_x=None) -> dendsn_norm_cfg:
        """The C struct with the row strides of the given tensors (None: contiguous)."""
        ld = [self.D if t is None or self.N < 2 else int(t.stride(0)) for t in (x, residual, y, sum, grad_y, grad_sum, grad_x)]
        return dendsn_norm_cfg(self.N, self.D, *ld, IO[self.io], self.eps)


def dendsn_norm_workspace_bytes(cfg: RMSNormConfig) -> int:
    return _bytes(block_lib().dendsn_norm_workspace_bytes, ctypes.byref(cfg.to_c()))


def dendsn_norm_forward(cfg: RMSNormConfig, x, residual, weight, y, sum, rstd, stream=None):
    st = stream if stream is not None else _stream(x.device)
    _check(block_lib().dendsn_norm_forward(ctypes.byref(cfg.to_c(x, residual, y, sum)), _ptr(x), _ptr(residual),
                                           _ptr(weight), _ptr(y), _ptr(sum), _ptr(rstd), st))


def dendsn_norm_forward_e4m3(cfg: RMSNormConfig, x, residual, weight, y, scale, sum, rstd, stream=None):
    st = stream if stream is not None else _stream(x.device)
    _check(block_lib().dendsn_norm_forward_e4m3(ctypes.byref(cfg.to_c(x, residual, y, sum)), _ptr(x), _ptr(residual),
                                                _ptr(weight), _ptr(y), _ptr(scale), _ptr(sum), _ptr(rstd), st))


def dendsn_norm_backward(cfg: RMSNormConfig, x, weight, rstd, grad_y, grad_sum, grad_x, grad_weight, workspace, stream=None):
    st = stream if stream is not None else _stream(x.device)
    c = cfg.to_c(x, None, None, None, grad_y, grad_sum, grad_x)
    _check(block_lib().dendsn_norm_backward(ctypes.byref(c), _ptr(x), _ptr(weight), _ptr(rstd), _ptr(grad_y),
                                            _ptr(grad_sum), _ptr(grad_x), _ptr(grad_weight), _ptr(workspace),
                                            _nbytes(workspace), st))


def dendsn_norm_backward_residual(cfg: RMSNormConfig, x, residual, weight, rstd, grad_y, grad_sum, grad_x, grad_weight,
                                  workspace, stream=None):
    st = stream if stream is not None else _stream(x.device)
    c = cfg.to_c(x, residual, None, None, grad_y, grad_sum, grad_x)
    _check(block_lib().dendsn_norm_backward_residual(ctypes.byref(c), _ptr(x), _ptr(residual), _ptr(weight), _ptr(rstd),
                                                     _ptr(grad_y), _ptr(grad_sum), _ptr(grad_x), _ptr(grad_weight),
                                                     _ptr(workspace), _nbytes(workspace), st))


def _check_norm(cfg, x, weight, residual):
    dt, dev = _io_dtype(cfg.io), x.device
    _expect(x, "x", (cfg.N, cfg.D), dt, dev, rows=True)
    _expect(weight, "weight", (cfg.D,), dt, dev, optional=True)
    _expect(residual, "residual", (cfg.N, cfg.D), dt, dev, optional=True, rows=True)
    return dt, dev


def rms_norm(cfg: RMSNormConfig, x, weight=None, residual=None):
    """Returns (y [N, D] io, rstd [N] fp32, sum [N, D] io or None): the norm of x [N, D], or of
    ``sum`` = x + residual, times ``weight`` [D].  Rows may lie apart."""
    import torch

    _, dev = _check_norm(cfg, x, weight, residual)
    st = _stream(dev)
    y = x.new_empty((cfg.N, cfg.D))
    summed = None if residual is None else x.new_empty((cfg.N, cfg.D))
    rstd = torch.empty((cfg.N,), dtype=torch.float32, device=dev)
    _check(block_lib().dendsn_norm_forward(ctypes.byref(cfg.to_c(x, residual)), _ptr(x), _ptr(residual), _ptr(weight),
                                           _ptr(y), _ptr(summed), _ptr(rstd), st))
    return y, rstd, summed


def rms_norm_e4m3(cfg: RMSNormConfig, x, weight=None, residual=None):
    """As ``rms_norm`` with rows in 8 bits: (y [N, D] float8_e4m3fn, scale [N] fp32, rstd, sum); a row
    is y * scale."""
    import torch

    _, dev = _check_norm(cfg, x, weight, residual)
    st = _stream(dev)
    y = torch.empty((cfg.N, cfg.D), dtype=torch.float8_e4m3fn, device=dev)
    summed = None if residual is None else x.new_empty((cfg.N, cfg.D))
    scale, rstd = (torch.empty((cfg.N,), dtype=torch.float32, device=dev) for _ in range(2))
    _check(block_lib().dendsn_norm_forward_e4m3(ctypes.byref(cfg.to_c(x, residual)), _ptr(x), _ptr(residual),
                                                _ptr(weight), _ptr(y), _ptr(scale), _ptr(summed), _ptr(rstd), st))
    return y, scale, rstd, summed


def rms_norm_backward(cfg: RMSNormConfig, x, weight, rstd, grad_y, grad_sum=None, *, residual=None, workspace=None):
    """Returns a dict with grad_x [N, D] io (also the residual's) and, where there is a ``weight``,
    grad_weight [D] io: the gradients of sum(grad_y * y) + sum(grad_sum * sum).  ``x`` is the
    forward's, or the sum that it gave, which has io's bits; with the forward's ``residual`` beside its
    x their sum is formed again in fp32, as y had it, for one more array read."""
    import torch

    dt, dev = _check_norm(cfg, x, weight, residual)
    _expect(rstd, "rstd", (cfg.N,), torch.float32, dev)
    _expect(grad_y, "grad_y", (cfg.N, cfg.D), dt, dev, rows=True)
    _expect(grad_sum, "grad_sum", (cfg.N, cfg.D), dt, dev, optional=True, rows=True)
    st, fn = _stream(dev), block_lib()
    out = dict(grad_x=x.new_empty((cfg.N, cfg.D)))
    c = cfg.to_c(x, residual, None, None, grad_y, grad_sum)
    ws = None
    if weight is not None:
        out["grad_weight"] = x.new_empty((cfg.D,))
        ws = _workspace(_bytes(fn.dendsn_norm_workspace_bytes, ctypes.byref(c)), workspace, dev)
    _check(fn.dendsn_norm_backward_residual(ctypes.byref(c), _ptr(x), _ptr(residual), _ptr(weight), _ptr(rstd), _ptr(grad_y),
                                            _ptr(grad_sum), _ptr(out["grad_x"]), _ptr(out.get("grad_weight")), _ptr(ws),
                                            _nbytes(ws), st))
    return out


# ---------------------------------------------------------------------------
# AdamW
# ---------------------------------------------------------------------------
@dataclass(frozen=True)
class AdamWConfig:
    """An AdamW step's numbers.  ``state`` "f32", or "e4m3": m and the root of v in 8 bits, in
    blocks of 256 values with a scale each."""

    lr: float = 1e-3
    beta1: float = 0.9
    beta2: float = 0.999
    eps: float = 1e-8
    weight_decay: float = 0.01
    state: str = "f32"

    def with_(self, **kw) -> "AdamWConfig":
        return dataclasses.replace(self, **kw)

    def to_c(self) -> dendsn_adamw_cfg:
        return dendsn_adamw_cfg(self.lr, self.beta1, self.beta2, self.eps, self.weight_decay, STATE[self.state])


def dendsn_adamw_step(cfg: AdamWConfig, tensors, count: int, step: int, step_dev, grad_scale, seed: int, stream):
    """``tensors``: a ctypes array of dendsn_adamw_tensor, or its bytes."""
    _check(block_lib().dendsn_adamw_step(ctypes.byref(cfg.to_c()), ctypes.cast(tensors, _P), count, step,
                                         _ptr(step_dev), _ptr(grad_scale), seed, stream))


def adamw_states(cfg: AdamWConfig, params):
    """The states before the first step, one tuple a tensor of ``params``: (m, v) fp32, or (m, m_scale,
    root, root_scale) with m and the root of v in float8_e4m3fn."""
    import torch

    def of(p):
        if cfg.state == "f32":
            return torch.zeros_like(p), torch.zeros_like(p)
        code = lambda: torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)
        scale = lambda: torch.ones((-(-p.numel() // STATE_BLOCK),), dtype=torch.float32, device=p.device)
        return code(), scale(), code(), scale()

    return [of(p) for p in params]


def adamw(cfg: AdamWConfig, params, grads, states, step, *, copies=None, grad_scale=None, seed: int = 0):
    """One step, in place, over lists of tensors: ``params`` fp32, ``grads`` fp32 or bf16 of the same
    shapes, ``states`` as ``adamw_states`` gives them; all contiguous.  ``step`` is its number from 1
    on, an int or an int32 tensor [1] on the GPU; ``copies``, a list of bf16 tensors (or None in a
    place), receive the new parameters rounded; ``grad_scale`` [1] fp32 multiplies the gradients;
    ``seed`` is that of the random rounding of 8-bit states.  What is written (params, states, scales,
    copies) may appear once, and may not overlap otherwise (not checked); a gradient may be shared."""
    import torch

    count = len(params)
    if len(grads) != count or len(states) != count or (copies is not None and len(copies) != count):
        raise ValueError(f"{count} params, {len(grads)} grads, {len(states)} states"
                         + ("" if copies is None else f", {len(copies)} copies"))
    if count == 0:
        return
    dev = params[0].device
    f32, bf16, f8 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
    eight = STATE[cfg.state] == 1
    state_type, parts = (f8, 4) if eight else (f32, 2)

    pack = struct.Struct("@q7Pi4x").pack_into
    array = bytearray(ctypes.sizeof(dendsn_adamw_tensor) * count)
    gpu, here, ms, vs, c, at, written = dev.type == "cuda", params[0].get_device(), 0, 0, 0, 0, []
    for i, (p, g, s) in enumerate(zip(params, grads, states)):
        if len(s) != parts:
            raise ValueError(f"states of tensor {i}: {len(s)} tensors, expected {parts}")
        if g is None:
            raise ValueError(f"grad of tensor {i} is required")
        m, v, shape = s[0], s[parts // 2], p.shape
        # of hundreds of tensors: in few steps whether all is well, else what is not
        if not (gpu and p.dtype is f32 and p.is_contiguous() and p.get_device() == here
                and g.is_contiguous() and g.get_device() == here and g.shape == shape
                and m.dtype is state_type and m.is_contiguous() and m.get_device() == here and m.shape == shape
                and v.dtype is state_type and v.is_contiguous() and v.get_device() == here and v.shape == shape):
            for t, name, dtype in ((p, "param", f32), (g, "grad", None), (m, "m", state_type),
                                   (v, "root" if eight else "v", state_type)):
                _expect(t, f"{name} of tensor {i}", shape, dtype, dev)
        half = g.dtype is bf16
        if not half and g.dtype is not f32:
            raise ValueError(f"grad of tensor {i}: expected torch.float32 or torch.bfloat16")
        n = p.numel()
        if eight:
            for t, name in ((s[1], "m_scale"), (s[3], "root_scale")):
                _expect(t, f"{name} of tensor {i}", (-(-n // STATE_BLOCK),), f32, dev)
            ms, vs = s[1].data_ptr(), s[3].data_ptr()
            written += (ms, vs)
        if copies is not None:
            c = copies[i]
            _expect(c, f"copy of tensor {i}", shape, bf16, dev, optional=True)
            c = 0 if c is None else c.data_ptr()
            written.append(c)
        pa, ma, va = p.data_ptr(), m.data_ptr(), v.data_ptr()
        written += (pa, ma, va)
        pack(array, at, n, pa, g.data_ptr(), ma, va, ms, vs, c, half)
        at += 72
    # two blocks of a launch would race on an array that is written and there twice (0: empty)
    if len(set(written)) != len(written) and len(set(written) - {0}) != len(written) - written.count(0):
        raise ValueError("params, states, copies: an array that is written appears twice")
    step_dev = None
    if isinstance(step, torch.Tensor):
        _expect(step, "step", (1,), torch.int32, dev)
        step, step_dev = 1, step
    _expect(grad_scale, "grad_scale", (1,), f32, dev, optional=True)
    dendsn_adamw_step(cfg, (ctypes.c_char * len(array)).from_buffer(array), count, int(step), step_dev, grad_scale, seed, _stream(dev))
