"""Binding of libzvc_ffn.so (C ABI in include/zvc_ffn.h): the gated half of a
feed-forward block and dropout, forward and backward.

Argument marshalling only, in the manner of `zvc`: the caller owns every
tensor, outputs included, and work is enqueued on the given or the current
stream.  Tensors are 2-D with contiguous rows (any row stride), except that
zvc_dropout takes contiguous tensors of any shape too.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import importlib
import os
import warnings
from typing import Optional

import torch

from .zvc import ZVC_E_ARG, ZvcError, _check, _stream_handle

_PKG = os.path.dirname(os.path.abspath(__file__))
LIBRARY = os.path.join(_PKG, "libzvc_ffn.so")

ZVC_FP32, ZVC_FP16, ZVC_BF16 = range(3)
TYPES = {torch.float32: ZVC_FP32, torch.float16: ZVC_FP16, torch.bfloat16: ZVC_BF16}
ZVC_RELU, ZVC_SILU, ZVC_GELU, ZVC_GELU_TANH = range(4)
ACTIVATIONS = {"relu": ZVC_RELU, "silu": ZVC_SILU, "gelu": ZVC_GELU, "gelu_tanh": ZVC_GELU_TANH}
MAX_COLUMNS, MAX_ROWS = 1 << 21, 1 << 28

# every symbol include/zvc_ffn.h declares
EXPORTS = ("zvc_dropout_fraction", "zvc_dropout", "zvc_glu_workspace_bytes", "zvc_glu_forward", "zvc_glu_backward")

_lib = None
_calls = None       # the calls, see _native()


def load() -> ctypes.CDLL:
    """Load the built library (paper_1705_01626_amd/libzvc_ffn.so) and declare signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIBRARY):
        raise ImportError("%s is not built: run `python -m paper_1705_01626_amd.build` (there is no CPU "
                          "fallback)" % LIBRARY)
    lib = ctypes.CDLL(LIBRARY)
    vp, sz, ci, u64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_uint64
    drop = [u64, u64, u64, vp]
    lib.zvc_dropout_fraction.restype = u64
    lib.zvc_dropout_fraction.argtypes = [ctypes.c_double]
    lib.zvc_dropout.restype = ci
    lib.zvc_dropout.argtypes = [vp, sz, vp, sz, vp, sz, sz, sz, ci, *drop, vp]
    lib.zvc_glu_workspace_bytes.restype = sz
    lib.zvc_glu_workspace_bytes.argtypes = [sz, sz, sz, ci, ci, ci]
    lib.zvc_glu_forward.restype = ci
    lib.zvc_glu_forward.argtypes = [vp, sz, vp, vp, sz, vp, sz, vp, vp, sz, sz, sz, sz, ci, ci, *drop, vp, sz, vp]
    lib.zvc_glu_backward.restype = ci
    lib.zvc_glu_backward.argtypes = [vp, sz, vp, sz, vp, vp, sz, vp, vp, sz, vp, sz, vp, vp, sz, sz, sz, sz, ci, ci,
                                     *drop, vp, sz, vp]
    _lib = lib
    return lib


def _native():
    """The calls, integers in and status out (see zvc._native)."""
    global _calls
    calls = _calls
    if calls is None:
        lib = load()
        try:
            calls = importlib.import_module(__package__ + "._calls")
        except ModuleNotFoundError:
            warnings.warn("paper_1705_01626_amd._calls is not built for this interpreter (`python -m "
                          "paper_1705_01626_amd.build`): calls go through ctypes", RuntimeWarning, stacklevel=3)
            _calls = lib
            return lib
        calls.open_ffn(LIBRARY)
        _calls = calls
    return calls


# ---- arguments -------------------------------------------------------------------
def _refuse(where: str, what: str):
    raise ZvcError(ZVC_E_ARG, "%s (%s)" % (where, what))


def _type(t: torch.Tensor, where: str) -> int:
    code = TYPES.get(t.dtype)
    if code is None:
        _refuse(where, "element type %s; fp32, fp16 and bf16 are taken" % t.dtype)
    return code


def _matrix(t: torch.Tensor, rows: int, cols: int, like: torch.Tensor, where: str, name: str) -> int:
    """The row stride of a rows x cols tensor of like's type and device."""
    row, col = t.stride() if t.dim() == 2 else (0, 0)
    # (what nearly every call has, with few of the attribute lookups that a call's host time goes to)
    if col == 1 and row >= cols and t.shape == (rows, cols) and t.dtype is like.dtype and t.get_device() == like.get_device():
        return row if rows > 1 else cols               # (one row has no next one, however far away that would be)
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != cols:
        _refuse(where, "%s is %s, %d x %d expected" % (name, tuple(t.shape), rows, cols))
    if t.dtype != like.dtype or t.device != like.device:
        _refuse(where, "%s is %s on %s, the first tensor is %s on %s" % (name, t.dtype, t.device, like.dtype, like.device))
    if (col != 1 and cols > 1) or (row < cols and rows > 1):
        _refuse(where, "%s has strides %s: rows have to be contiguous and apart" % (name, t.stride()))
    return row if rows > 1 else cols


def _fraction(p: float, where: str) -> int:
    if not 0.0 <= p <= 1.0:
        _refuse(where, "p = %r, 0 to 1 expected" % (p,))
    return round(p * 4294967296.0)


def _word(d_offset: Optional[torch.Tensor], like: torch.Tensor, where: str) -> int:
    if d_offset is None:
        return 0
    if d_offset.dtype != torch.int64 or d_offset.numel() < 1 or d_offset.device != like.device:
        _refuse(where, "d_offset has to be an int64 tensor on the inputs' device")
    return d_offset.data_ptr()


def _on_gpu(where: str, x: torch.Tensor, ws: Optional[torch.Tensor] = None) -> None:
    if not x.is_cuda or (ws is not None and ws.device != x.device):
        _refuse(where, "the tensors and the workspace have to be on one GPU")


def _room(ws: torch.Tensor, where: str) -> int:
    """The bytes of a workspace.  (An expanded one has more elements than memory.)"""
    if not ws.is_contiguous():
        _refuse(where, "the workspace has strides %s: it has to be contiguous" % (ws.stride(),))
    return ws.numel() * ws.element_size()


def _pair(a, b, rows, cols, like, where, names):
    """Addresses and common row stride of two tensors that are both there or both not."""
    if (a is None) != (b is None):
        _refuse(where, "%s and %s go together" % names)
    if a is None:
        return 0, 0, cols
    ld = _matrix(a, rows, cols, like, where, names[0])
    if _matrix(b, rows, cols, like, where, names[1]) != ld:
        _refuse(where, "%s and %s have different row strides" % names)
    return a.data_ptr(), b.data_ptr(), ld


# ---- dropout ---------------------------------------------------------------------
def zvc_dropout(x: torch.Tensor, y: torch.Tensor, p: float, seed: int, offset: int = 0,
                residual: Optional[torch.Tensor] = None, d_offset: Optional[torch.Tensor] = None,
                stream=None) -> None:
    """Enqueue y = drop(x), or residual + drop(x).  With dy for x it is the gradient."""
    where = "zvc_dropout"
    code = _type(x, where)
    tensors = [(t, name) for t, name in ((x, "x"), (y, "y"), (residual, "residual")) if t is not None]
    if all(t.is_contiguous() and t.shape == x.shape for t, _ in tensors):
        rows, cols = 1, x.numel()                      # of any shape: one long row
        lds = [cols] * 3
        for t, name in tensors[1:]:
            if t.dtype != x.dtype or t.device != x.device:
                _refuse(where, "%s is %s on %s, x is %s on %s" % (name, t.dtype, t.device, x.dtype, x.device))
    else:
        if x.dim() != 2:
            _refuse(where, "tensors of one shape, contiguous or 2-D, expected")
        rows, cols = x.shape
        lds = [_matrix(t, rows, cols, x, where, name) for t, name in tensors] + [cols]
    drop, word = _fraction(p, where), _word(d_offset, x, where)
    _on_gpu(where, x)
    _check(_native().zvc_dropout(x.data_ptr(), lds[0], 0 if residual is None else residual.data_ptr(), lds[2],
                                 y.data_ptr(), lds[1], rows, cols, code, drop, seed, offset, word,
                                 _stream_handle(stream)), where)


# ---- the gated block -----------------------------------------------------------------
def zvc_glu_workspace_bytes(m: int, n: int, k: int, dtype: torch.dtype, backward: bool = False,
                            loose: bool = False) -> int:
    code = TYPES.get(dtype)
    return 0 if code is None else int(_native().zvc_glu_workspace_bytes(m, n, k, code, int(backward), int(loose)))


def _loose(*tensors: torch.Tensor) -> bool:
    return any(t.data_ptr() % 16 or (t.shape[0] > 1 and (t.stride(0) * t.element_size()) % 16) for t in tensors)


def new_glu_workspace(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, backward: bool = False) -> torch.Tensor:
    """A workspace for the calls on these tensors; backward: for both passes."""
    m, k, n = x.shape[0], x.shape[1], w_gate.shape[0]
    loose = _loose(x, w_gate, w_up)
    need = max(zvc_glu_workspace_bytes(m, n, k, x.dtype, b, loose) for b in ((False, True) if backward else (False,)))
    return torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)


def _activation(name: str, where: str) -> int:
    code = ACTIVATIONS.get(name)
    if code is None:
        _refuse(where, "activation %r; there are %s" % (name, ", ".join(ACTIVATIONS)))
    return code


def zvc_glu_forward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, h: torch.Tensor, ws: torch.Tensor,
                    activation: str = "silu", gate: Optional[torch.Tensor] = None, up: Optional[torch.Tensor] = None,
                    p: float = 0.0, seed: int = 0, offset: int = 0, d_offset: Optional[torch.Tensor] = None,
                    stream=None) -> None:
    """Enqueue h = drop(act(x w_gate^T) * (x w_up^T)); gate and up receive what the backward pass needs."""
    where = "zvc_glu_forward"
    code, act = _type(x, where), _activation(activation, where)
    if x.dim() != 2 or w_gate.dim() != 2:
        _refuse(where, "x and the weights have to be 2-D")
    m, k, n = x.shape[0], x.shape[1], w_gate.shape[0]
    ldx = _matrix(x, m, k, x, where, "x")
    wg, wu, ldw = _pair(w_gate, w_up, n, k, x, where, ("w_gate", "w_up"))
    ldh = _matrix(h, m, n, x, where, "h")
    gate_at, up_at, ldp = _pair(gate, up, m, n, x, where, ("gate", "up"))
    drop, word = _fraction(p, where), _word(d_offset, x, where)
    room = _room(ws, where)
    _on_gpu(where, x, ws)
    _check(_native().zvc_glu_forward(x.data_ptr(), ldx, wg, wu, ldw, h.data_ptr(), ldh, gate_at, up_at, ldp, m, n, k,
                                     code, act, drop, seed, offset, word, ws.data_ptr(), room,
                                     _stream_handle(stream)), where)


def zvc_glu_backward(dh: torch.Tensor, x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor,
                     dx: Optional[torch.Tensor], dw_gate: Optional[torch.Tensor], dw_up: Optional[torch.Tensor],
                     ws: torch.Tensor, activation: str = "silu", gate: Optional[torch.Tensor] = None,
                     up: Optional[torch.Tensor] = None, p: float = 0.0, seed: int = 0, offset: int = 0,
                     d_offset: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue the gradients of x, w_gate and w_up (None: not wanted) from dh, from the kept gate and up or, without
    them, from x again."""
    where = "zvc_glu_backward"
    code, act = _type(x, where), _activation(activation, where)
    if x.dim() != 2 or w_gate.dim() != 2:
        _refuse(where, "x and the weights have to be 2-D")
    m, k, n = x.shape[0], x.shape[1], w_gate.shape[0]
    ldx = _matrix(x, m, k, x, where, "x")
    wg, wu, ldw = _pair(w_gate, w_up, n, k, x, where, ("w_gate", "w_up"))
    lddh = _matrix(dh, m, n, x, where, "dh")
    gate_at, up_at, ldp = _pair(gate, up, m, n, x, where, ("gate", "up"))
    lddx = k if dx is None else _matrix(dx, m, k, x, where, "dx")
    dwg, dwu, lddw = _pair(dw_gate, dw_up, n, k, x, where, ("dw_gate", "dw_up"))
    drop, word = _fraction(p, where), _word(d_offset, x, where)
    room = _room(ws, where)
    _on_gpu(where, x, ws)
    _check(_native().zvc_glu_backward(dh.data_ptr(), lddh, x.data_ptr(), ldx, wg, wu, ldw, gate_at, up_at, ldp,
                                      0 if dx is None else dx.data_ptr(), lddx, dwg, dwu, lddw, m, n, k, code, act,
                                      drop, seed, offset, word, ws.data_ptr(), room,
                                      _stream_handle(stream)), where)
