"""Binding of libzvc_adamw.so (C ABI in include/zvc_adamw.h): an AdamW step over many tensors in one launch,
with states in 32 bits or in 8.

    state = adamw.new_adamw_state(w, bits=8)
    plan = adamw.new_plan([(w, grad, state, master), ...])          # once; master None where w itself is all there is
    adamw.zvc_adamw(plan, rate=3e-4, step=t)                        # t = 1, 2, ...

Argument marshalling only, in the manner of `zvc`: the caller owns every tensor, and work is enqueued
on the given or the current stream.  A plan keeps its tensors alive, and dropped behind a call it keeps their memory
until that step has run.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import importlib
import os
import warnings
from typing import Optional, Sequence, Tuple

import torch

from .ffn import TYPES, _refuse
from .zvc import _check, _stream_handle

_PKG = os.path.dirname(os.path.abspath(__file__))
LIBRARY = os.path.join(_PKG, "libzvc_adamw.so")

BLOCK = 128                       # elements of an 8-bit state that share a scale
CODES = torch.float8_e4m3fn       # what 8-bit states are held in

# every symbol include/zvc_adamw.h declares
EXPORTS = ("zvc_adamw_plan_bytes", "zvc_adamw_plan", "zvc_adamw")

_lib = None
_calls = None       # the calls, see _native()


class _Tensor(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in ("param", "master", "grad", "m", "v", "m_scale", "v_scale")] + [
        ("count", ctypes.c_uint64)] + [(name, ctypes.c_int32) for name in ("type", "grad_type", "state_bits", "decays")]


class _Now(ctypes.Structure):
    _fields_ = [(name, ctypes.c_double) for name in ("rate", "beta1", "beta2", "eps", "decay", "factor")] + [
        ("step", ctypes.c_uint64), ("seed", ctypes.c_uint64), ("d_step", ctypes.c_void_p), ("d_factors", ctypes.c_void_p)]


def load() -> ctypes.CDLL:
    """Load the built library (paper_1705_01626_amd/libzvc_adamw.so) and declare signatures."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIBRARY):
        raise ImportError("%s is not built: run `python -m paper_1705_01626_amd.build` (there is no CPU "
                          "fallback)" % LIBRARY)
    lib = ctypes.CDLL(LIBRARY)
    vp, sz, ci = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    lib.zvc_adamw_plan_bytes.restype = sz
    lib.zvc_adamw_plan_bytes.argtypes = [sz]
    lib.zvc_adamw_plan.restype = ci
    lib.zvc_adamw_plan.argtypes = [vp, sz, vp, sz]
    lib.zvc_adamw.restype = ci
    lib.zvc_adamw.argtypes = [vp, vp, vp, vp]
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
        calls.open_adamw(LIBRARY)
        _calls = calls
    return calls


def new_adamw_state(param: torch.Tensor, bits: int = 32) -> Tuple[torch.Tensor, ...]:
    """The state of a tensor before its first step: (m, v) in 32 bits, or in 8 (m, r, m_scale, r_scale) with r = sqrt(v)."""
    if bits == 32:
        return tuple(torch.zeros(param.shape, dtype=torch.float32, device=param.device) for _ in range(2))
    if bits != 8:
        _refuse("new_adamw_state", "bits = %r, 8 or 32 expected" % (bits,))
    scales = -(-param.numel() // BLOCK)
    return (*(torch.zeros(param.shape, dtype=CODES, device=param.device) for _ in range(2)),
            *(torch.zeros(scales, dtype=torch.float32, device=param.device) for _ in range(2)))


class Plan:
    """What new_plan() makes: the tensors of a step, and the bytes that describe them on the host and on their device."""

    def __init__(self, tensors, host, device_bytes):
        self.tensors, self.host, self.device_bytes = tensors, host, device_bytes
        self.device = device_bytes.device
        self.streams = set()                        # that the tensors' allocator knows to be used
        self.used_on(torch.cuda.current_stream(self.device))        # (most steps': here and not in the first of them; the tensors may have been made on another)

    def used_on(self, stream) -> None:
        """No memory of the plan's tensors, nor its own, goes to another tensor before what is on `stream` by then has run.  (Of the gradients
        and weights too: the plan may be the last to hold them.)"""
        for param, grad, state, master in self.tensors:
            for t in (param, grad, *state, master):
                if t is not None:
                    t.record_stream(stream)
        self.device_bytes.record_stream(stream)
        self.streams.add(int(stream.cuda_stream))


def _flat(t: torch.Tensor, count: int, types, device, where: str, name: str) -> int:
    """The address of a contiguous tensor of `count` elements."""
    if t.dtype not in types:
        _refuse(where, "%s is %s, %s expected" % (name, t.dtype, " or ".join(str(x) for x in types)))
    if t.numel() != count:
        _refuse(where, "%s has %d elements, %d expected" % (name, t.numel(), count))
    if t.device != device:
        _refuse(where, "%s is on %s, the first tensor is on %s" % (name, t.device, device))
    if not t.is_contiguous():
        _refuse(where, "%s has strides %s: it has to be contiguous" % (name, t.stride()))
    return t.data_ptr()


def new_plan(tensors: Sequence[tuple], decay: Optional[Sequence[bool]] = None) -> Plan:
    """A plan for a step over tensors, each (param, grad, state, master): state from new_adamw_state(), master
    a float32 tensor with the weights of a 16-bit param, or None.  decay: for each, whether weight decay applies (default: to all).
    The plan holds addresses: gradients are written into these tensors (a new tensor in `.grad` is not seen), none is resized, and a
    captured graph with a step of it needs the plan for as long as it is replayed."""
    where = "new_plan"
    tensors = [tuple(t) for t in tensors]
    if not tensors:
        _refuse(where, "no tensors")
    if decay is None:
        decay = [True] * len(tensors)
    if len(decay) != len(tensors):
        _refuse(where, "decay for %d tensors, there are %d" % (len(decay), len(tensors)))
    device = tensors[0][0].device
    table = (_Tensor * len(tensors))()
    for i, (param, grad, state, master) in enumerate(tensors):
        name, count = "tensor %d's " % i, param.numel()
        if param.dtype not in TYPES:
            _refuse(where, "%sparam is %s; fp32, fp16 and bf16 are taken" % (name, param.dtype))
        e = table[i]
        e.param = _flat(param, count, (param.dtype,), device, where, name + "param")
        e.grad = _flat(grad, count, (param.dtype, torch.float32), device, where, name + "grad")
        if master is not None:
            if param.dtype == torch.float32:
                _refuse(where, "%sparam is float32 and needs no master" % name)
            e.master = _flat(master, count, (torch.float32,), device, where, name + "master")
        if len(state) == 2:
            m, v = state
            e.m, e.v = (_flat(t, count, (torch.float32,), device, where, name + which) for t, which in ((m, "m"), (v, "v")))
            e.state_bits = 32
        elif len(state) == 4:
            m, r, m_scale, r_scale = state
            e.m, e.v = (_flat(t, count, (CODES,), device, where, name + which) for t, which in ((m, "m"), (r, "r")))
            e.m_scale, e.v_scale = (_flat(t, -(-count // BLOCK), (torch.float32,), device, where, name + which)
                                    for t, which in ((m_scale, "m_scale"), (r_scale, "r_scale")))
            e.state_bits = 8
        else:
            _refuse(where, "%sstate has %d parts, 2 or 4 expected" % (name, len(state)))
        e.count, e.type, e.grad_type, e.decays = count, TYPES[param.dtype], TYPES[grad.dtype], int(bool(decay[i]))
    if device.type != "cuda":
        _refuse(where, "the tensors have to be on one GPU")
    need = load().zvc_adamw_plan_bytes(len(tensors))
    host = torch.empty(max(need, 1), dtype=torch.uint8)
    _check(load().zvc_adamw_plan(ctypes.addressof(table), len(tensors), host.data_ptr(), need), where)
    return Plan(tensors, host, host.to(device))


def zvc_adamw(plan: Plan, rate: float, step: int, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
              decay: float = 0.0, factor: float = 1.0, seed: int = 0, d_step: Optional[torch.Tensor] = None,
              d_factors: Optional[torch.Tensor] = None, stream=None) -> None:
    """Enqueue step number `step` (from 1 on) of every tensor of the plan.  factor: what gradients are multiplied by; seed: of the
    8-bit states' rounding.  d_step (int64) is added to step, and rate and factor are multiplied by d_factors[0] and [1]
    (float32), when the work runs."""
    where = "zvc_adamw"
    if plan.device.index != torch.cuda.current_device():
        _refuse(where, "the plan is on %s, the current device is cuda:%d" % (plan.device, torch.cuda.current_device()))
    now = _Now(rate, beta1, beta2, eps, decay, factor, 0, 0, 0, 0)
    if not 0 <= step < 1 << 64:
        _refuse(where, "step = %r, a number from 1 on expected" % (step,))
    now.step, now.seed = step, seed & (1 << 64) - 1
    if d_step is not None:
        if d_step.dtype != torch.int64 or d_step.numel() < 1 or d_step.device != plan.device:
            _refuse(where, "d_step has to be an int64 tensor on the plan's device")
        now.d_step = d_step.data_ptr()
    if d_factors is not None:
        if (d_factors.dtype != torch.float32 or d_factors.numel() < 2 or d_factors.device != plan.device
                or not d_factors.is_contiguous()):
            _refuse(where, "d_factors has to be two contiguous floats on the plan's device")
        now.d_factors = d_factors.data_ptr()
    handle = _stream_handle(stream)
    if handle not in plan.streams:
        plan.used_on(torch.cuda.current_stream() if stream is None else stream)
    _check(_native().zvc_adamw(plan.host.data_ptr(), plan.device_bytes.data_ptr(), ctypes.addressof(now), handle), where)
