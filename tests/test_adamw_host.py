"""The host side of the optimizer's step: plans and refusals, all before any GPU call, and the reference that the GPU tests
use.  No GPU needed."""
import ctypes
import math
import os
import re
import sys

import numpy as np
import pytest
import torch

from paper_1705_01626_amd import adamw, zvc
from paper_1705_01626_amd import build as zvc_build
from tests import adamw_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FP32, FP16, BF16 = range(3)


@pytest.fixture(scope="module")
def lib():
    zvc_build.ensure_built()
    return adamw.load()


def test_exports_every_declared_symbol(lib):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "zvc_adamw.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(zvc_adamw(?:_plan(?:_bytes)?)?)\s*\(", header)) == set(adamw.EXPORTS)
    for name in adamw.EXPORTS:
        assert getattr(lib, name) is not None


def tensor(number=1, count=1000, type=BF16, grad_type=None, bits=32, kept=True, **other):
    """A tensor at addresses of its own."""
    at = [(number << 40) + (i << 36) for i in range(7)]
    t = adamw._Tensor(at[0], at[1] if kept else None, at[2], at[3], at[4], at[5] if bits == 8 else None, at[6] if bits == 8 else None, count, type,
                      type if grad_type is None else grad_type, bits, 1)
    for k, v in other.items():
        setattr(t, k, v)
    return t


def plan(lib, *tensors, room=None):
    table = (adamw._Tensor * max(len(tensors), 1))(*tensors)
    need = lib.zvc_adamw_plan_bytes(len(tensors)) if room is None else room
    host = np.zeros(max(need, 8) // 8 + 1, dtype=np.uint64)
    return lib.zvc_adamw_plan(ctypes.addressof(table), len(tensors), host.ctypes.data, need), host


@pytest.mark.parametrize("wrong,status", [
    ({"type": 3}, zvc.ZVC_E_ARG), ({"type": FP32}, zvc.ZVC_E_ARG), ({"grad_type": FP16}, zvc.ZVC_E_ARG), ({"grad_type": 5}, zvc.ZVC_E_ARG),
    ({"bits": 16}, zvc.ZVC_E_ARG), ({"count": (1 << 34) + 1}, zvc.ZVC_E_ARG), ({"param": 0}, zvc.ZVC_E_ARG), ({"grad": 0}, zvc.ZVC_E_ARG),
    ({"m": 0}, zvc.ZVC_E_ARG), ({"v": 0}, zvc.ZVC_E_ARG), ({"m_scale": 1 << 50}, zvc.ZVC_E_ARG), ({"bits": 8, "m_scale": 0}, zvc.ZVC_E_ARG),
    ({"bits": 8, "v_scale": 0}, zvc.ZVC_E_ARG), ({"param": (1 << 40) + 1}, zvc.ZVC_E_ALIGN), ({"grad": (1 << 50) + 1}, zvc.ZVC_E_ALIGN),
    ({"master": (1 << 50) + 2}, zvc.ZVC_E_ALIGN), ({"m": (1 << 50) + 2}, zvc.ZVC_E_ALIGN), ({"bits": 8, "v_scale": (1 << 50) + 2}, zvc.ZVC_E_ALIGN)])
def test_plan_refuses(lib, wrong, status):
    assert plan(lib, tensor(**wrong))[0] == status


def test_plan_refuses_what_overlaps(lib):
    """Whatever is written, against anything; gradients may share."""
    base = 1 << 40
    names = ("param", "master", "grad", "m", "v", "m_scale", "v_scale")
    for bits in (8, 32):
        for a in names if bits == 8 else names[:5]:
            for b in names if bits == 8 else names[:5]:
                one, two = tensor(1, bits=bits), tensor(2, bits=bits)
                setattr(two, a, getattr(one, b))
                want = zvc.ZVC_OK if a == b == "grad" else zvc.ZVC_E_ARG
                assert plan(lib, one, two)[0] == want, (bits, a, b)
    assert plan(lib, tensor(1), tensor(1))[0] == zvc.ZVC_E_ARG                               # the same tensor twice
    assert plan(lib, tensor(1), tensor(2, param=base + 1998))[0] == zvc.ZVC_E_ARG
    assert plan(lib, tensor(1), tensor(2, param=base + 2000))[0] == zvc.ZVC_OK               # back to back
    assert plan(lib, tensor(1, bits=8), tensor(2, bits=8, m_scale=base + (5 << 36) + 28))[0] == zvc.ZVC_E_ARG
    assert plan(lib, tensor(1, bits=8), tensor(2, bits=8, m_scale=base + (5 << 36) + 32))[0] == zvc.ZVC_OK
    assert plan(lib, tensor(1, m=2 ** 64 - 1000))[0] == zvc.ZVC_E_ARG                        # around the end of memory


def test_plans_of_no_and_of_many_tensors(lib):
    assert plan(lib)[0] == zvc.ZVC_OK
    assert plan(lib, tensor(count=0, param=0, grad=0, m=0, v=0, master=0))[0] == zvc.ZVC_OK
    assert plan(lib, tensor(), room=8)[0] == zvc.ZVC_E_CAPACITY
    assert lib.zvc_adamw_plan_bytes((1 << 20) + 1) == 0
    assert lib.zvc_adamw_plan(0, 1, 8, 1 << 20) == lib.zvc_adamw_plan(0, 0, 0, 1 << 20) == zvc.ZVC_E_ARG
    status, host = plan(lib, *[tensor(1 + i, count=2048 * i + 1) for i in range(100)])
    assert status == zvc.ZVC_OK and host[1] == 100 and host[2] == sum(i + 1 for i in range(100))
    # more pieces than a grid can have
    assert plan(lib, *[tensor(1 + i, count=1 << 33, param=(1 + 7 * i) << 44, master=(2 + 7 * i) << 44, grad=(3 + 7 * i) << 44, m=(4 + 7 * i) << 44,
                              v=(5 + 7 * i) << 44) for i in range(4)])[0] == zvc.ZVC_E_ARG


def step(lib, host, d_plan=1 << 50, **other):
    now = adamw._Now(1e-3, 0.9, 0.99, 1e-8, 0.1, 1.0, 1, 0, 0, 0)
    for k, v in other.items():
        setattr(now, k, v)
    return lib.zvc_adamw(host.ctypes.data, d_plan, ctypes.addressof(now), None)


@pytest.mark.parametrize("wrong,status", [
    ({"rate": math.nan}, zvc.ZVC_E_ARG), ({"rate": math.inf}, zvc.ZVC_E_ARG), ({"rate": 1e39}, zvc.ZVC_E_ARG), ({"beta1": 1.0}, zvc.ZVC_E_ARG), ({"beta2": -0.1}, zvc.ZVC_E_ARG),
    ({"beta2": math.nan}, zvc.ZVC_E_ARG), ({"eps": -1e-8}, zvc.ZVC_E_ARG), ({"decay": math.inf}, zvc.ZVC_E_ARG), ({"factor": math.nan}, zvc.ZVC_E_ARG),
    ({"step": 0}, zvc.ZVC_E_ARG), ({"d_step": (1 << 50) + 4}, zvc.ZVC_E_ALIGN), ({"d_factors": (1 << 50) + 2}, zvc.ZVC_E_ALIGN),
    ({"d_plan": 0}, zvc.ZVC_E_ARG), ({"d_plan": (1 << 50) + 8}, zvc.ZVC_E_ALIGN)])
def test_step_refuses(lib, wrong, status):
    assert step(lib, plan(lib, tensor())[1], **wrong) == status


def test_step_takes_plans_alone(lib):
    good = plan(lib, tensor())[1]
    for word in (0, 1, 3):
        bad = good.copy()
        bad[word] += 1
        assert step(lib, bad) == zvc.ZVC_E_ARG
    assert lib.zvc_adamw(0, 1 << 50, good.ctypes.data, None) == lib.zvc_adamw(good.ctypes.data, 1 << 50, 0, None) == zvc.ZVC_E_ARG
    assert step(lib, plan(lib)[1], d_plan=0) == step(lib, plan(lib, tensor(count=0))[1]) == zvc.ZVC_OK        # nothing to do: no GPU here


def test_python_refuses():
    p = torch.zeros(300)
    state, state8 = adamw.new_adamw_state(p), adamw.new_adamw_state(p, 8)
    assert [t.shape for t in state8] == [(300,), (300,), (3,), (3,)] and state8[0].dtype == torch.float8_e4m3fn

    def refused(match, *tensors, **kwargs):
        with pytest.raises(zvc.ZvcError, match=match) as error:
            adamw.new_plan(tensors, **kwargs)
        assert error.value.status == zvc.ZVC_E_ARG

    refused("no tensors")
    refused("param is torch.float64", (p.double(), p, state, None))
    refused("grad has 299", (p, p[:299], state, None))
    refused("grad is torch.float16", (p, p.half(), state, None))
    refused("needs no master", (p, p.clone(), state, p.clone()))
    refused("master is torch.bfloat16", (p.bfloat16(), p.clone(), state, p.bfloat16()))
    refused("state has 3 parts", (p, p.clone(), state8[:3], None))
    refused("m is torch.float8", (p, p.clone(), state8[:2], None))
    refused("m_scale has 2", (p, p.clone(), (*state8[:2], state8[2][:2], state8[3]), None))
    refused("strides", (torch.zeros(300, 2)[:, 0], p.clone(), state, None))
    refused("decay for 2", (p, p.clone(), state, None), decay=[True, False])
    refused("one GPU", (p, p.clone(), state, None))
    with pytest.raises(zvc.ZvcError, match="bits"):
        adamw.new_adamw_state(p, 4)


# ---- the reference ------------------------------------------------------------------
def test_calls_through_ctypes_give_the_same(lib, monkeypatch):
    want = adamw._native().zvc_adamw(0, 0, 0, 0)
    monkeypatch.setattr(adamw, "_calls", None)
    monkeypatch.setitem(sys.modules, "paper_1705_01626_amd._calls", None)
    with pytest.warns(RuntimeWarning, match="ctypes"):
        assert adamw._native().zvc_adamw(0, 0, 0, 0) == want == zvc.ZVC_E_ARG


def test_numbers_of_the_codes():
    """As torch reads e4m3."""
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(adamw_ref.NUMBERS, want, equal_nan=True)


def test_codes_are_right_on_the_average():
    """A value's code, over all random numbers, has the value as its mean; and a value that is a code's number is always that code."""
    random = np.arange(65536, dtype=np.float64)
    for value in (1.0, 0.73, 255.0, 200.3, 0.0033, 2.0 ** -9, 0.00011):
        for sign in (1, -1):
            values = np.full((65536, adamw_ref.BLOCK), 0.0, dtype=np.float32)
            values[:, 0], values[:, 1] = 255.5, sign * value             # (the first sets the scale, to 1)
            draws = np.zeros((65536, adamw_ref.BLOCK))
            draws[:, 1] = random
            codes, scales = adamw_ref.narrow(values.reshape(-1), draws.reshape(-1), False)
            assert (scales == 1).all()
            numbers = adamw_ref.NUMBERS[codes.reshape(-1, adamw_ref.BLOCK)[:, 1]]
            step = 2.0 ** (max(math.floor(math.log2(value)), -6) - 3)
            assert abs(numbers.mean() - sign * np.float32(value)) <= step * 2 ** -16
            assert len(set(numbers)) <= 2


def test_reference_step_against_the_formula():
    rng = np.random.default_rng(3)
    p, grad, m = (rng.standard_normal(500).astype(np.float32) for _ in range(3))
    v = rng.standard_normal(500).astype(np.float32) ** 2
    m1, v1 = adamw_ref.states(m, v, grad, 0.9, 0.99)
    assert np.allclose(m1, 0.9 * m + 0.1 * grad, rtol=1e-5, atol=1e-6) and np.allclose(v1, 0.99 * v + 0.01 * grad ** 2, rtol=1e-5)
    value, bound = adamw_ref.weights(p, m1, v1, 7, 1e-2, 0.9, 0.99, 1e-8, 0.1)
    t = torch.nn.Parameter(torch.from_numpy(p).double())
    opt = torch.optim.AdamW([t], lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    t.grad = torch.from_numpy(grad).double()
    opt.state[t] = {"step": torch.tensor(6.0), "exp_avg": torch.from_numpy(m).double(), "exp_avg_sq": torch.from_numpy(v).double()}
    opt.step()
    assert np.abs(t.detach().numpy() - value).max() < 1e-6 and (bound < 1e-5 * (1 + np.abs(p))).all()
