"""Python binding of the token-sequence operators (include/dendsn_seq.h).

Embedding rows and their gradient, the gated leaky scan over time (forward,
backward, one token at a time) and the softmax cross entropy of a linear readout
with its gradients.  As in the layer's binding, the functions named like the C
entry points take the C arguments (tensors in place of pointers); ``embedding``,
``gated_scan``, ``linear_ce`` and their companions check shapes, allocate the
outputs and call them.  Everything is computed by the library's HIP kernels, on
the current stream of the tensors' device, which has to be the current device; there is no
fallback.
"""

from __future__ import annotations

import ctypes
import dataclasses
from dataclasses import dataclass

from .binding import IO, DendSNError, _check_device
from .binding import lib as _lib

GATE = {"sigmoid": 0, "decay": 1}
SCAN_TILE = 64   # steps between the scan's checkpoints


class dendsn_embed_cfg(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int64) for k in ("n", "V", "D", "ld_table", "ld_out")] + \
               [("io", ctypes.c_int32), ("index", ctypes.c_int32), ("scale", ctypes.c_float)]


class dendsn_scan_cfg(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int64) for k in (
        "T", "batch", "D", "x_t", "x_b", "g_t", "g_b", "h_t", "h_b", "grad_h_t", "grad_h_b", "grad_x_t", "grad_x_b",
        "grad_g_t", "grad_g_b")] + [("io", ctypes.c_int32), ("gate", ctypes.c_int32), ("leaky", ctypes.c_int32)]


class dendsn_ce_cfg(ctypes.Structure):
    _fields_ = [(k, ctypes.c_int64) for k in ("N", "V", "D", "ld_hidden", "ld_weight", "ld_grad_hidden",
                                                 "ld_grad_weight")] + \
               [("io", ctypes.c_int32), ("index", ctypes.c_int32), ("logit_scale", ctypes.c_float)]


_P, _Z = ctypes.c_void_p, ctypes.c_size_t
_SIZE = ctypes.POINTER(ctypes.c_size_t)

_SIGS = {
    "dendsn_embed_forward": (ctypes.c_int, [ctypes.POINTER(dendsn_embed_cfg)] + [_P] * 4),
    "dendsn_embed_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(dendsn_embed_cfg), _SIZE]),
    "dendsn_embed_backward": (ctypes.c_int, [ctypes.POINTER(dendsn_embed_cfg)] + [_P] * 4 + [_Z, _P]),
    "dendsn_scan_ckpt_bytes": (ctypes.c_int, [ctypes.POINTER(dendsn_scan_cfg), _SIZE]),
    "dendsn_scan_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(dendsn_scan_cfg), ctypes.c_int32, _SIZE]),
    "dendsn_scan_forward": (ctypes.c_int, [ctypes.POINTER(dendsn_scan_cfg)] + [_P] * 8 + [_Z, _P]),
    "dendsn_scan_backward": (ctypes.c_int, [ctypes.POINTER(dendsn_scan_cfg)] + [_P] * 10 + [_Z, _P]),
    "dendsn_scan_step": (ctypes.c_int, [ctypes.POINTER(dendsn_scan_cfg), _P, _P, ctypes.c_int64, _P, _P, _P, _P]),
    "dendsn_ce_workspace_bytes": (ctypes.c_int, [ctypes.POINTER(dendsn_ce_cfg), ctypes.c_int32, _SIZE]),
    "dendsn_ce_workspace_bytes_at": (ctypes.c_int, [ctypes.POINTER(dendsn_ce_cfg), ctypes.c_int32, _P, _P, _SIZE]),
    "dendsn_ce_forward": (ctypes.c_int, [ctypes.POINTER(dendsn_ce_cfg)] + [_P] * 6 + [_Z, _P]),
    "dendsn_ce_train": (ctypes.c_int, [ctypes.POINTER(dendsn_ce_cfg)] + [_P] * 9 + [_Z, _P]),
    "dendsn_seq_last_error": (ctypes.c_char_p, []),
}

SEQ_EXPORTS = tuple(_SIGS)

_bound = None


def seq_lib():
    """The library with this header's entry points bound (once)."""
    global _bound
    if _bound is None:
        handle = _lib()
        for name, (res, args) in _SIGS.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _bound = handle
    return _bound


def _check(status: int):
    if status != 0:
        raise DendSNError(status, seq_lib().dendsn_seq_last_error().decode())


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"a tensor on {t.device}: the library takes GPU memory alone")
    return t.data_ptr()


def _stream(device):
    """The current stream of the GPU that the tensors lie on, which has to be the current one: a
    serving step's calls are a few microseconds long, so the handle is asked for without building a
    Stream object."""
    import torch

    if device.type != "cuda" or device.index != torch._C._cuda_getDevice():
        _check_device(device)  # raises
    return torch._C._cuda_getCurrentRawStream(device.index)


def dendsn_seq_last_error() -> str:
    return seq_lib().dendsn_seq_last_error().decode()


def _bytes(fn, *args) -> int:
    out = ctypes.c_size_t(0)
    _check(fn(*args, ctypes.byref(out)))
    return out.value


def _nbytes(t):
    """The bytes of a workspace: as many as its elements' only where they lie one after another."""
    if t is None:
        return 0
    if not t.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return t.nbytes


def _io_dtype(io):
    import torch

    return torch.bfloat16 if io == "bf16" else torch.float32


def _index_code(t, name):
    import torch

    if t.dtype == torch.int64:
        return 1
    if t.dtype == torch.int32:
        return 0
    raise ValueError(f"{name}: dtype {t.dtype} is neither torch.int32 nor torch.int64")


def _expect(t, name, shape, dtype, device, optional=False, rows=False):
    """Shape, type, device and layout: contiguous, or with ``rows`` any strides whose
    innermost one is 1."""
    if t is None:
        if optional:
            return
        raise ValueError(f"{name} is required")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)} != {tuple(shape)}")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name}: dtype {t.dtype} != {dtype}")
    if t.device != device:
        raise ValueError(f"{name}: on {t.device}, expected {device}")
    if rows:
        if t.shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: the values of a row must be adjacent")
    elif not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _workspace(nbytes, workspace, device):
    """The caller's scratch, or one from torch's allocator."""
    import torch

    if workspace is None and nbytes:
        return torch.empty((nbytes,), dtype=torch.uint8, device=device)
    if workspace is not None and workspace.device != device:
        raise ValueError(f"workspace: on {workspace.device}, expected {device}")
    return workspace


# ---------------------------------------------------------------------------
# Embedding
# ---------------------------------------------------------------------------
@dataclass(frozen=True)
class EmbeddingConfig:
    """n tokens looked up in a table of V rows of D values; out = scale * table[ids].
    An id outside [0, V) names no row: its out row is 0 and it has no gradient."""

    n: int
    V: int
    D: int
    io: str = "f32"
    scale: float = 1.0
    index: str = "i64"        # of the C entry points' ids; the calls below go by the tensor
    ld_table: int = 0         # 0: D
    ld_out: int = 0

    def with_(self, **kw) -> "EmbeddingConfig":
        return dataclasses.replace(self, **kw)

    def to_c(self) -> dendsn_embed_cfg:
        return dendsn_embed_cfg(self.n, self.V, self.D, self.ld_table or self.D, self.ld_out or self.D, IO[self.io],
                                1 if self.index == "i64" else 0, self.scale)


def dendsn_embed_workspace_bytes(cfg: EmbeddingConfig) -> int:
    return _bytes(seq_lib().dendsn_embed_workspace_bytes, ctypes.byref(cfg.to_c()))


def dendsn_embed_forward(cfg: EmbeddingConfig, ids, table, out, stream=None):
    st = stream if stream is not None else _stream(out.device)
    _check(seq_lib().dendsn_embed_forward(ctypes.byref(cfg.to_c()), _ptr(ids), _ptr(table), _ptr(out), st))


def dendsn_embed_backward(cfg: EmbeddingConfig, ids, grad_out, grad_table, workspace, stream=None):
    st = stream if stream is not None else _stream(grad_table.device)
    _check(seq_lib().dendsn_embed_backward(ctypes.byref(cfg.to_c()), _ptr(ids), _ptr(grad_out), _ptr(grad_table),
                                           _ptr(workspace), _nbytes(workspace), st))


def _row_stride(t, D):
    return max(int(t.stride(0)), D) if t.shape[0] > 1 else D


def embedding(cfg: EmbeddingConfig, ids, table):
    """The rows [n, D] of ``ids`` [n] (int32 or int64) in ``table`` [V, D] (rows may lie apart)."""
    dt, dev = _io_dtype(cfg.io), table.device
    _expect(ids, "ids", (cfg.n,), None, dev)
    _expect(table, "table", (cfg.V, cfg.D), dt, dev, rows=True)
    if table.shape[0] > 1 and table.stride(0) < cfg.D:
        raise ValueError("table: rows overlap")
    index, st = _index_code(ids, "ids"), _stream(dev)
    # (a serving step's lookup: the struct and the output by the shortest way)
    out = table.new_empty((cfg.n, cfg.D))
    c = dendsn_embed_cfg(cfg.n, cfg.V, cfg.D, _row_stride(table, cfg.D), cfg.D, IO[cfg.io], index, cfg.scale)
    _check(seq_lib().dendsn_embed_forward(ctypes.byref(c), ids.data_ptr(), table.data_ptr(), out.data_ptr(), st))
    return out


def embedding_backward(cfg: EmbeddingConfig, ids, grad_out, workspace=None):
    """The table's gradient [V, D] of ``grad_out`` [n, D] (rows may lie apart, or be one
    row broadcast): every row written, sums in an order fixed by the ids."""
    import torch

    dt, dev = _io_dtype(cfg.io), grad_out.device
    _expect(ids, "ids", (cfg.n,), None, dev)
    _expect(grad_out, "grad_out", (cfg.n, cfg.D), dt, dev, rows=True)
    index, st = _index_code(ids, "ids"), _stream(dev)
    grad_table = torch.empty((cfg.V, cfg.D), dtype=dt, device=dev)
    c = cfg.to_c()
    c.index, c.ld_table = index, cfg.D
    c.ld_out = int(grad_out.stride(0)) if cfg.n > 1 else cfg.D
    ws = _workspace(_bytes(seq_lib().dendsn_embed_workspace_bytes, ctypes.byref(c)), workspace, dev)
    _check(seq_lib().dendsn_embed_backward(ctypes.byref(c), _ptr(ids), _ptr(grad_out), _ptr(grad_table), _ptr(ws),
                                           _nbytes(ws), st))
    return grad_table


# ---------------------------------------------------------------------------
# Gated scan
# ---------------------------------------------------------------------------
@dataclass(frozen=True)
class GatedScanConfig:
    """h[t] = a[t] h[t-1] + w[t] x[t] over T steps, batch sequences and D channels:
    a = sigmoid(g) (gate "sigmoid") or g ("decay"), w = 1 - a (``leaky``) or 1.  Tensors
    are [T, batch, D] views of any strides whose innermost one is 1."""

    T: int
    batch: int
    D: int
    io: str = "f32"
    gate: str = "sigmoid"
    leaky: bool = True

    def with_(self, **kw) -> "GatedScanConfig":
        return dataclasses.replace(self, **kw)

    def to_c(self, x=None, g=None, h=None, grad_h=None, grad_x=None, grad_g=None) -> dendsn_scan_cfg:
        """The C struct with the strides of the given [T, batch, D] tensors (None: contiguous)."""
        dense = (self.batch * self.D, self.D)
        s = [v for t in (x, g, h, grad_h, grad_x, grad_g) for v in (dense if t is None else t.stride()[:2])]
        return dendsn_scan_cfg(self.T, self.batch, self.D, *s, IO[self.io], GATE[self.gate], int(self.leaky))

    def ckpt_values(self) -> int:
        """The fp32 values of the checkpoints (dendsn_scan_ckpt_bytes / 4)."""
        return -(-self.T // SCAN_TILE) * self.batch * self.D


def dendsn_scan_ckpt_bytes(cfg: GatedScanConfig) -> int:
    return _bytes(seq_lib().dendsn_scan_ckpt_bytes, ctypes.byref(cfg.to_c()))


def dendsn_scan_workspace_bytes(cfg: GatedScanConfig, backward: bool) -> int:
    return _bytes(seq_lib().dendsn_scan_workspace_bytes, ctypes.byref(cfg.to_c()), int(backward))


def dendsn_scan_forward(cfg: GatedScanConfig, x, g, h0, lengths, h, h_last, ckpt, workspace, stream=None):
    st = stream if stream is not None else _stream(x.device)
    _check(seq_lib().dendsn_scan_forward(ctypes.byref(cfg.to_c(x, g, h)), _ptr(x), _ptr(g), _ptr(h0), _ptr(lengths),
                                         _ptr(h), _ptr(h_last), _ptr(ckpt), _ptr(workspace), _nbytes(workspace), st))


def dendsn_scan_backward(cfg: GatedScanConfig, x, g, lengths, ckpt, grad_h, grad_h_last, grad_x, grad_g, grad_h0,
                         workspace, stream=None):
    st = stream if stream is not None else _stream(x.device)
    c = cfg.to_c(x, g, None, grad_h, grad_x, grad_g)
    _check(seq_lib().dendsn_scan_backward(ctypes.byref(c), _ptr(x), _ptr(g), _ptr(lengths), _ptr(ckpt), _ptr(grad_h),
                                          _ptr(grad_h_last), _ptr(grad_x), _ptr(grad_g), _ptr(grad_h0),
                                          _ptr(workspace), _nbytes(workspace), st))


def _step_cfg(cfg, x, g, h):
    return dendsn_scan_cfg(cfg.T, cfg.batch, cfg.D, 0, x.stride(0), 0, g.stride(0), 0, h.stride(0), 0, 0, 0, 0, 0, 0,
                           IO[cfg.io], GATE[cfg.gate], cfg.leaky)


def dendsn_scan_step(cfg: GatedScanConfig, x, g, slots, state, h, stream=None):
    st = stream if stream is not None else _stream(x.device)
    _check(seq_lib().dendsn_scan_step(ctypes.byref(_step_cfg(cfg, x, g, h)), _ptr(x), _ptr(g), state.shape[0],
                                      _ptr(slots), _ptr(state), _ptr(h), st))


def _check_scan(cfg, x, g, lengths):
    import torch

    dt, dev, shape = _io_dtype(cfg.io), x.device, (cfg.T, cfg.batch, cfg.D)
    _expect(x, "x", shape, dt, dev, rows=True)
    _expect(g, "g", shape, dt, dev, rows=True)
    _expect(lengths, "lengths", (cfg.batch,), torch.int32, dev, optional=True)
    return dt, dev, shape


def gated_scan(cfg: GatedScanConfig, x, g, h0=None, lengths=None, *, save_ckpt: bool = True, workspace=None):
    """Returns (h [T, batch, D] io, h_last [batch, D] fp32, ckpt or None).  ``h0`` [batch, D]
    fp32 is the state before the first step (None: 0).  Steps at and past ``lengths``
    [batch] (int32) are no part of a sequence: h is 0 there and h_last the state before
    them.  ``ckpt`` is what the backward needs."""
    import torch

    dt, dev, shape = _check_scan(cfg, x, g, lengths)
    _expect(h0, "h0", shape[1:], torch.float32, dev, optional=True)
    st = _stream(dev)
    h = x.new_empty(shape)
    h_last = torch.empty(shape[1:], dtype=torch.float32, device=dev)
    c, fn = cfg.to_c(x, g, h), seq_lib()
    ckpt = torch.empty((cfg.ckpt_values(),), dtype=torch.float32, device=dev) if save_ckpt else None
    ws = _workspace(_bytes(fn.dendsn_scan_workspace_bytes, ctypes.byref(c), 0), workspace, dev)
    _check(fn.dendsn_scan_forward(ctypes.byref(c), _ptr(x), _ptr(g), _ptr(h0), _ptr(lengths), _ptr(h), _ptr(h_last),
                                  _ptr(ckpt), _ptr(ws), _nbytes(ws), st))
    return h, h_last, ckpt


def gated_scan_backward(cfg: GatedScanConfig, x, g, lengths, ckpt, grad_h, grad_h_last=None, *, workspace=None):
    """Returns a dict with grad_x and grad_g [T, batch, D] io and grad_h0 [batch, D] fp32, the
    gradients of sum(grad_h * h) + sum(grad_h_last * h_last)."""
    import torch

    dt, dev, shape = _check_scan(cfg, x, g, lengths)
    _expect(grad_h, "grad_h", shape, dt, dev, rows=True)
    _expect(grad_h_last, "grad_h_last", shape[1:], torch.float32, dev, optional=True)
    need = 4 * cfg.ckpt_values()
    if need and (ckpt is None or ckpt.dtype != torch.float32 or ckpt.device != dev or not ckpt.is_contiguous()
                 or ckpt.numel() * 4 < need):
        raise ValueError(f"ckpt must be the forward's checkpoints: contiguous float32 on {dev}, {need} bytes")
    st, fn = _stream(dev), seq_lib()
    out = dict(grad_x=x.new_empty(shape), grad_g=x.new_empty(shape),
               grad_h0=torch.empty(shape[1:], dtype=torch.float32, device=dev))
    c = cfg.to_c(x, g, None, grad_h, out["grad_x"], out["grad_g"])
    ws = _workspace(_bytes(fn.dendsn_scan_workspace_bytes, ctypes.byref(c), 1), workspace, dev)
    _check(fn.dendsn_scan_backward(ctypes.byref(c), _ptr(x), _ptr(g), _ptr(lengths), _ptr(ckpt), _ptr(grad_h),
                                   _ptr(grad_h_last), _ptr(out["grad_x"]), _ptr(out["grad_g"]),
                                   _ptr(out["grad_h0"]), _ptr(ws), _nbytes(ws), st))
    return out


def gated_scan_step(cfg: GatedScanConfig, x, g, state, slots=None):
    """One token of each of cfg.batch requests (cfg.T = 1): updates ``state`` [held, D] (fp32) in
    place at the rows ``slots`` [batch] (int32; None: row b for request b) and returns h
    [batch, D].  A request whose slot is no row of ``state`` is idle: h is 0."""
    import torch

    dt, dev, shape = _io_dtype(cfg.io), x.device, (cfg.batch, cfg.D)
    _expect(x, "x", shape, dt, dev, rows=True)
    _expect(g, "g", shape, dt, dev, rows=True)
    _expect(state, "state", (state.shape[0], cfg.D), torch.float32, dev)
    _expect(slots, "slots", (cfg.batch,), torch.int32, dev, optional=True)
    st = _stream(dev)
    h = x.new_empty(shape)
    _check(seq_lib().dendsn_scan_step(ctypes.byref(_step_cfg(cfg, x, g, h)), x.data_ptr(), g.data_ptr(), state.shape[0],
                                      _ptr(slots), state.data_ptr(), h.data_ptr(), st))
    return h


# ---------------------------------------------------------------------------
# Linear cross entropy
# ---------------------------------------------------------------------------
@dataclass(frozen=True)
class LinearCEConfig:
    """Softmax cross entropy of the logits logit_scale * hidden weight^T: N rows, V classes,
    D features.  A row whose target is outside [0, V) is ignored."""

    N: int
    V: int
    D: int
    io: str = "f32"
    logit_scale: float = 1.0
    index: str = "i64"        # of the C entry points' targets; the calls below go by the tensor
    ld_hidden: int = 0        # 0: D
    ld_weight: int = 0
    ld_grad_hidden: int = 0
    ld_grad_weight: int = 0

    def with_(self, **kw) -> "LinearCEConfig":
        return dataclasses.replace(self, **kw)

    def to_c(self) -> dendsn_ce_cfg:
        return dendsn_ce_cfg(self.N, self.V, self.D, self.ld_hidden or self.D, self.ld_weight or self.D,
                             self.ld_grad_hidden or self.D, self.ld_grad_weight or self.D, IO[self.io],
                             1 if self.index == "i64" else 0, self.logit_scale)


def dendsn_ce_workspace_bytes(cfg: LinearCEConfig, train: bool) -> int:
    return _bytes(seq_lib().dendsn_ce_workspace_bytes, ctypes.byref(cfg.to_c()), int(train))


def dendsn_ce_workspace_bytes_at(cfg: LinearCEConfig, train: bool, hidden, weight) -> int:
    return _bytes(seq_lib().dendsn_ce_workspace_bytes_at, ctypes.byref(cfg.to_c()), int(train), _ptr(hidden), _ptr(weight))


def dendsn_ce_forward(cfg: LinearCEConfig, hidden, weight, targets, loss, lse, workspace, stream=None):
    st = stream if stream is not None else _stream(weight.device)
    _check(seq_lib().dendsn_ce_forward(ctypes.byref(cfg.to_c()), _ptr(hidden), _ptr(weight), _ptr(targets), _ptr(loss),
                                       _ptr(lse), _ptr(workspace), _nbytes(workspace), st))


def dendsn_ce_train(cfg: LinearCEConfig, hidden, weight, targets, row_weight, loss, lse, grad_hidden, grad_weight,
                    workspace, stream=None):
    st = stream if stream is not None else _stream(weight.device)
    _check(seq_lib().dendsn_ce_train(ctypes.byref(cfg.to_c()), _ptr(hidden), _ptr(weight), _ptr(targets),
                                     _ptr(row_weight), _ptr(loss), _ptr(lse), _ptr(grad_hidden), _ptr(grad_weight),
                                     _ptr(workspace), _nbytes(workspace), st))


def _check_ce(cfg, hidden, weight, targets):
    dt, dev = _io_dtype(cfg.io), weight.device
    _expect(hidden, "hidden", (cfg.N, cfg.D), dt, dev, rows=True)
    _expect(weight, "weight", (cfg.V, cfg.D), dt, dev, rows=True)
    _expect(targets, "targets", (cfg.N,), None, dev)
    for t, name in ((hidden, "hidden"), (weight, "weight")):
        if t.shape[0] > 1 and t.stride(0) < cfg.D:
            raise ValueError(f"{name}: rows overlap")
    c = cfg.to_c()
    c.index = _index_code(targets, "targets")
    c.ld_hidden, c.ld_weight = _row_stride(hidden, cfg.D), _row_stride(weight, cfg.D)
    c.ld_grad_hidden = c.ld_grad_weight = cfg.D
    return dt, dev, c


def linear_ce(cfg: LinearCEConfig, hidden, weight, targets, *, workspace=None):
    """Returns (loss [N], lse [N]), fp32: lse = log sum exp of a row's logits, loss = lse minus
    the target's logit; both 0 in ignored rows.  ``hidden`` [N, D] and ``weight`` [V, D] may
    have rows that lie apart; ``targets`` [N] are int32 or int64."""
    import torch

    _, dev, c = _check_ce(cfg, hidden, weight, targets)
    st = _stream(dev)
    loss, lse = (torch.empty((cfg.N,), dtype=torch.float32, device=dev) for _ in range(2))
    fn = seq_lib()
    ws = _workspace(_bytes(fn.dendsn_ce_workspace_bytes_at, ctypes.byref(c), 0, _ptr(hidden), _ptr(weight)), workspace, dev)
    _check(fn.dendsn_ce_forward(ctypes.byref(c), _ptr(hidden), _ptr(weight), _ptr(targets), _ptr(loss), _ptr(lse),
                                _ptr(ws), _nbytes(ws), st))
    return loss, lse


def linear_ce_train(cfg: LinearCEConfig, hidden, weight, targets, row_weight=None, *, workspace=None):
    """Returns a dict with loss and lse [N] (as ``linear_ce``) and the gradients grad_hidden [N, D]
    and grad_weight [V, D] of sum(row_weight * loss); ``row_weight`` [N] fp32, None: 1."""
    import torch

    dt, dev, c = _check_ce(cfg, hidden, weight, targets)
    _expect(row_weight, "row_weight", (cfg.N,), torch.float32, dev, optional=True)
    st = _stream(dev)
    out = dict(loss=torch.empty((cfg.N,), dtype=torch.float32, device=dev),
               lse=torch.empty((cfg.N,), dtype=torch.float32, device=dev),
               grad_hidden=torch.empty((cfg.N, cfg.D), dtype=dt, device=dev),
               grad_weight=torch.empty((cfg.V, cfg.D), dtype=dt, device=dev))
    fn = seq_lib()
    ws = _workspace(_bytes(fn.dendsn_ce_workspace_bytes_at, ctypes.byref(c), 1, _ptr(hidden), _ptr(weight)), workspace, dev)
    _check(fn.dendsn_ce_train(ctypes.byref(c), _ptr(hidden), _ptr(weight), _ptr(targets), _ptr(row_weight),
                              _ptr(out["loss"]), _ptr(out["lse"]), _ptr(out["grad_hidden"]), _ptr(out["grad_weight"]),
                              _ptr(ws), _nbytes(ws), st))
    return out
