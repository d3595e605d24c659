"""Binding of libzvc_experts.so (C ABI in include/zvc_experts.h): the router of a mixture of experts, and the
experts' matrix products with their gradients.

    experts.zvc_route(logits, chosen, weights, offsets, order, place, ws)        # ws = new_route_workspace(logits, top)
    rows = x[order // top]                                                       # an expert's rows one behind the other
    experts.zvc_expert_product(rows, w, offsets, y, ews)                         # ews = new_expert_workspace(rows, w)

Argument marshalling only, in the manner of `zvc`: the caller owns every tensor, outputs included, and
work is enqueued on the given or the current stream.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import importlib
import os
import warnings
from typing import Optional, Tuple

import torch

from .ffn import TYPES, _matrix, _refuse, _room, _type
from .zvc import _check, _current_device, _stream_handle

_PKG = os.path.dirname(os.path.abspath(__file__))
LIBRARY = os.path.join(_PKG, "libzvc_experts.so")

MAX_EXPERTS, MAX_TOP = 1024, 16

# every symbol include/zvc_experts.h declares
EXPORTS = ("zvc_route_workspace_bytes", "zvc_route", "zvc_route_backward", "zvc_expert_workspace_bytes", "zvc_expert_product",
           "zvc_expert_gradients")

_lib = None
_calls = None       # the calls, see _native()


def load() -> ctypes.CDLL:
    """Load the built library (paper_1705_01626_amd/libzvc_experts.so) and declare signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIBRARY):
        raise ImportError("%s is not built: run `python -m paper_1705_01626_amd.build` (there is no CPU "
                          "fallback)" % LIBRARY)
    lib = ctypes.CDLL(LIBRARY)
    vp, sz, ci = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    lib.zvc_route_workspace_bytes.restype = sz
    lib.zvc_route_workspace_bytes.argtypes = [sz, sz, sz]
    lib.zvc_route.restype = ci
    lib.zvc_route.argtypes = [vp, sz, vp, vp, vp, vp, vp, sz, sz, sz, ci, ci, vp, sz, vp]
    lib.zvc_route_backward.restype = ci
    lib.zvc_route_backward.argtypes = [vp, vp, sz, vp, vp, sz, sz, sz, sz, ci, ci, vp]
    lib.zvc_expert_workspace_bytes.restype = sz
    lib.zvc_expert_workspace_bytes.argtypes = [sz, sz, sz, sz, ci, ci]
    lib.zvc_expert_product.restype = ci
    lib.zvc_expert_product.argtypes = [vp, sz, vp, sz, sz, vp, vp, sz, sz, sz, sz, sz, ci, vp, sz, vp]
    lib.zvc_expert_gradients.restype = ci
    lib.zvc_expert_gradients.argtypes = [vp, sz, vp, sz, vp, sz, sz, vp, vp, sz, vp, sz, sz, sz, sz, sz, sz, ci, vp, sz, vp]
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
        calls.open_experts(LIBRARY)
        _calls = calls
    return calls


# ---- arguments -------------------------------------------------------------------
def _stack(t: torch.Tensor, experts: int, n: int, k: int, like: torch.Tensor, where: str, name: str) -> Tuple[int, int]:
    """The row stride and the experts' stride of an experts x n x k tensor of like's type and device."""
    if t.dim() != 3 or t.shape != (experts, n, k):
        _refuse(where, "%s is %s, %d x %d x %d expected" % (name, tuple(t.shape), experts, n, k))
    if t.dtype != like.dtype or t.get_device() != like.get_device():
        _refuse(where, "%s is %s on %s, the first tensor is %s on %s" % (name, t.dtype, t.device, like.dtype, like.device))
    between, row, col = t.stride()
    if n <= 1:
        row = k
    if t.numel() and ((col != 1 and k > 1) or row < k or (experts > 1 and between < (n - 1) * row + k)):
        _refuse(where, "%s has strides %s: rows have to be contiguous, and rows and experts apart" % (name, t.stride()))
    return row, between if experts > 1 and n and k else n * row


def _plain(t: torch.Tensor, shape: tuple, dtype: torch.dtype, device: int, where: str, name: str) -> int:
    """The address of a contiguous tensor."""
    # (what nearly every call has, with few of the attribute lookups that a call's host time goes to)
    if t.dtype is dtype and t.shape == shape and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    if tuple(t.shape) != shape or t.dtype != dtype:
        _refuse(where, "%s is %s %s, %s %s expected" % (name, t.dtype, tuple(t.shape), dtype, shape))
    if t.get_device() != device:
        _refuse(where, "%s is on %s, the first tensor is on another device" % (name, t.device))
    _refuse(where, "%s has strides %s: it has to be contiguous" % (name, t.stride()))


def _here(where: str, device: int, ws: Optional[torch.Tensor] = None) -> None:
    if device < 0 or (ws is not None and ws.get_device() != device):
        _refuse(where, "the tensors and the workspace have to be on one GPU")
    if device != (torch.cuda.current_device() if _current_device is None else _current_device()):
        _refuse(where, "the tensors are on cuda:%d, the current device is cuda:%d" % (device, torch.cuda.current_device()))


# ---- the router -------------------------------------------------------------------
def zvc_route_workspace_bytes(m: int, experts: int, top: int) -> int:
    return int(load().zvc_route_workspace_bytes(m, experts, top))


def new_route_workspace(logits: torch.Tensor, top: int) -> torch.Tensor:
    """A workspace for zvc_route on these logits, or fewer rows."""
    need = zvc_route_workspace_bytes(logits.shape[0], logits.shape[1], top)
    return torch.empty(max(need, 256), dtype=torch.uint8, device=logits.device)


def zvc_route(logits: torch.Tensor, chosen: torch.Tensor, weights: torch.Tensor, offsets: torch.Tensor, order: torch.Tensor,
              place: torch.Tensor, ws: torch.Tensor, normalize: bool = True, stream=None) -> None:
    """Enqueue the choice of chosen.shape[1] experts for each row of logits: chosen (int32) and weights (float32), m x top; offsets
    (int64, experts + 1) of each expert's rows; order (int64, m * top), the entry of each row; place (int64, m x top), the row of each entry."""
    where = "zvc_route"
    code = _type(logits, where)
    if logits.dim() != 2 or chosen.dim() != 2:
        _refuse(where, "logits and chosen have to be 2-D")
    (m, experts), top = logits.shape, chosen.shape[1]
    ldl = _matrix(logits, m, experts, logits, where, "logits")
    device, entries = logits.get_device(), (m, top)
    at = (_plain(chosen, entries, torch.int32, device, where, "chosen"), _plain(weights, entries, torch.float32, device, where, "weights"),
          _plain(offsets, (experts + 1,), torch.int64, device, where, "offsets"),
          _plain(order, (m * top,), torch.int64, device, where, "order"), _plain(place, entries, torch.int64, device, where, "place"))
    room = _room(ws, where)
    _here(where, device, ws)
    _check(_native().zvc_route(logits.data_ptr(), ldl, *at, m, experts, top, code, int(normalize), ws.data_ptr(), room,
                               _stream_handle(stream)), where)


def zvc_route_backward(dweights: torch.Tensor, logits: torch.Tensor, chosen: torch.Tensor, dlogits: torch.Tensor,
                       normalize: bool = True, stream=None) -> None:
    """Enqueue the gradient of logits from dweights (float32, m x top), with zvc_route's chosen."""
    where = "zvc_route_backward"
    code = _type(logits, where)
    if logits.dim() != 2 or chosen.dim() != 2:
        _refuse(where, "logits and chosen have to be 2-D")
    (m, experts), top = logits.shape, chosen.shape[1]
    ldl = _matrix(logits, m, experts, logits, where, "logits")
    ldd = _matrix(dlogits, m, experts, logits, where, "dlogits")
    device = logits.get_device()
    dw = _plain(dweights, (m, top), torch.float32, device, where, "dweights")
    at = _plain(chosen, (m, top), torch.int32, device, where, "chosen")
    _here(where, device)
    _check(_native().zvc_route_backward(dw, logits.data_ptr(), ldl, at, dlogits.data_ptr(), ldd, m, experts, top, code, int(normalize),
                                        _stream_handle(stream)), where)


# ---- the experts' products ----------------------------------------------------------
def zvc_expert_workspace_bytes(m: int, experts: int, n: int, k: int, dtype: torch.dtype, backward: bool = False) -> int:
    code = TYPES.get(dtype)
    return 0 if code is None else int(load().zvc_expert_workspace_bytes(m, experts, n, k, code, int(backward)))


def new_expert_workspace(x: torch.Tensor, w: torch.Tensor, backward: bool = False) -> torch.Tensor:
    """A workspace for the calls on these tensors, or fewer rows; backward: for both passes."""
    m, (experts, n, k) = x.shape[0], w.shape
    need = max(zvc_expert_workspace_bytes(m, experts, n, k, x.dtype, b) for b in ((False, True) if backward else (False,)))
    return torch.empty(max(need, 256), dtype=torch.uint8, device=x.device)


def zvc_expert_product(x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, y: torch.Tensor, ws: torch.Tensor, stream=None) -> None:
    """Enqueue y[r] = x[r] w[e]^T for offsets[e] <= r < offsets[e+1]; other rows of y stay as they were.  w: experts x n x k."""
    where = "zvc_expert_product"
    code = _type(x, where)
    if x.dim() != 2 or w.dim() != 3:
        _refuse(where, "x has to be 2-D and w 3-D")
    m, (experts, n, k) = x.shape[0], w.shape
    ldx = _matrix(x, m, k, x, where, "x")
    ldw, sw = _stack(w, experts, n, k, x, where, "w")
    ldy = _matrix(y, m, n, x, where, "y")
    device = x.get_device()
    at = _plain(offsets, (experts + 1,), torch.int64, device, where, "offsets")
    room = _room(ws, where)
    _here(where, device, ws)
    _check(_native().zvc_expert_product(x.data_ptr(), ldx, w.data_ptr(), ldw, sw, at, y.data_ptr(), ldy, m, experts, n, k, code,
                                        ws.data_ptr(), room, _stream_handle(stream)), where)


def zvc_expert_gradients(dy: torch.Tensor, x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, dx: Optional[torch.Tensor],
                         dw: Optional[torch.Tensor], ws: torch.Tensor, stream=None) -> None:
    """Enqueue the gradients of x and w (None: not wanted) from dy; rows of dx that are no expert's stay as they were."""
    where = "zvc_expert_gradients"
    code = _type(x, where)
    if x.dim() != 2 or w.dim() != 3:
        _refuse(where, "x has to be 2-D and w 3-D")
    m, (experts, n, k) = x.shape[0], w.shape
    ldx = _matrix(x, m, k, x, where, "x")
    ldw, sw = _stack(w, experts, n, k, x, where, "w")
    lddy = _matrix(dy, m, n, x, where, "dy")
    lddx = k if dx is None else _matrix(dx, m, k, x, where, "dx")
    lddw, sdw = (k, n * k) if dw is None else _stack(dw, experts, n, k, x, where, "dw")
    device = x.get_device()
    at = _plain(offsets, (experts + 1,), torch.int64, device, where, "offsets")
    room = _room(ws, where)
    _here(where, device, ws)
    _check(_native().zvc_expert_gradients(dy.data_ptr(), lddy, x.data_ptr(), ldx, w.data_ptr(), ldw, sw, at,
                                          0 if dx is None else dx.data_ptr(), lddx, 0 if dw is None else dw.data_ptr(), lddw, sdw, m,
                                          experts, n, k, code, ws.data_ptr(), room, _stream_handle(stream)), where)
