"""The host side of the training operators: exports, sizes, refusals before any GPU call, and the
reference that the GPU tests use.  No GPU needed."""
import math
import os
import re
import subprocess

import numpy as np
import pytest
import torch

from paper_1705_01626_amd import build as zvc_build
from paper_1705_01626_amd import ffn, zvc
from tests import ffn_ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
X, WG, WU, H, GATE, UP, WS, DH = ((i + 1) << 32 for i in range(8))
DX, DWG, DWU, Y, RES = ((i + 9) << 32 for i in range(5))
BIG = 1 << 31


@pytest.fixture(scope="module")
def lib():
    zvc_build.ensure_built()
    return ffn.load()


def test_exports_every_declared_symbol(lib):
    header = open(os.path.join(ROOT, "include", "zvc_ffn.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    assert set(re.findall(r"\b(zvc_[a-z_]+)\s*\(", header)) == set(ffn.EXPORTS)
    for name in ffn.EXPORTS:
        assert getattr(lib, name) is not None


def test_header_is_plain_c(tmp_path):
    source = tmp_path / "client.c"
    source.write_text('#include "zvc_ffn.h"\nint main(void) { return zvc_dropout_fraction(0.5) == (1ull << 31) ? 0 : 1; }\n')
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"),
                    "-I", zvc_build.ROCM_INCLUDE, "-c", str(source), "-o", str(tmp_path / "client.o")], check=True)


def test_fraction(lib):
    f = lib.zvc_dropout_fraction
    assert [f(p) for p in (0.0, 0.5, 1.0, 2.0 ** -32)] == [0, 1 << 31, 1 << 32, 1]
    assert f(0.1) == round(0.1 * 2 ** 32)
    assert all(f(p) > 1 << 32 for p in (-0.1, 1.0001, math.nan, math.inf))


def test_workspace_grows(lib):
    size = ffn.zvc_glu_workspace_bytes
    for dtype in ffn.TYPES:
        assert 0 < size(1, 8, 8, dtype) <= size(4096, 512, 512, dtype)
        assert size(4096, 512, 512, dtype, True) >= 2 * 4096 * 512 * torch.empty(0, dtype=dtype).element_size()
        assert size(100, 100, 100, dtype, True, True) >= size(100, 100, 100, dtype, True)
    assert size(1, 8, ffn.MAX_COLUMNS + 1, torch.float32) == 0
    assert size(1, 8, 8, torch.float64) == 0


def forward(lib, x=X, ldx=64, wg=WG, wu=WU, ldw=64, h=H, ldh=32, gate=0, up=0, ldp=32, m=16, n=32, k=64, type=2, act=1,
            drop=0, word=0, ws=WS, room=BIG):
    return lib.zvc_glu_forward(x, ldx, wg, wu, ldw, h, ldh, gate, up, ldp, m, n, k, type, act, drop, 1, 2, word, ws, room, None)


def backward(lib, dh=DH, lddh=32, x=X, ldx=64, wg=WG, wu=WU, ldw=64, gate=0, up=0, ldp=32, dx=DX, lddx=64, dwg=DWG, dwu=DWU,
             lddw=64, m=16, n=32, k=64, type=2, act=1, drop=0, word=0, ws=WS, room=BIG):
    return lib.zvc_glu_backward(dh, lddh, x, ldx, wg, wu, ldw, gate, up, ldp, dx, lddx, dwg, dwu, lddw, m, n, k, type, act,
                                drop, 1, 2, word, ws, room, None)


SHARED = [({"type": 3}, zvc.ZVC_E_ARG), ({"type": -1}, zvc.ZVC_E_ARG), ({"act": 4}, zvc.ZVC_E_ARG),
          ({"act": -1}, zvc.ZVC_E_ARG), ({"drop": (1 << 32) + 1}, zvc.ZVC_E_ARG), ({"word": 4}, zvc.ZVC_E_ALIGN),
          ({"ldx": 63}, zvc.ZVC_E_ARG), ({"ldw": 63}, zvc.ZVC_E_ARG), ({"ldx": (1 << 21) + 1}, zvc.ZVC_E_ARG),
          ({"k": (1 << 21) + 1, "ldx": 1 << 22, "ldw": 1 << 22}, zvc.ZVC_E_ARG), ({"m": (1 << 28) + 1}, zvc.ZVC_E_ARG),
          ({"m": 1 << 28, "n": 1 << 13, "ldh": 1 << 13, "lddh": 1 << 13}, zvc.ZVC_E_ARG),
          ({"gate": GATE}, zvc.ZVC_E_ARG), ({"up": UP}, zvc.ZVC_E_ARG),
          ({"gate": GATE, "up": UP, "ldp": 31}, zvc.ZVC_E_ARG), ({"x": 0}, zvc.ZVC_E_ARG), ({"wg": 0}, zvc.ZVC_E_ARG),
          ({"wu": 0}, zvc.ZVC_E_ARG), ({"ws": 0}, zvc.ZVC_E_ARG), ({"x": X + 1}, zvc.ZVC_E_ALIGN),
          ({"wu": WU + 2, "type": 0}, zvc.ZVC_E_ALIGN), ({"ws": WS + 128}, zvc.ZVC_E_ALIGN),
          ({"room": 0}, zvc.ZVC_E_WORKSPACE), ({"ws": X}, zvc.ZVC_E_ARG), ({"ws": WU - 256}, zvc.ZVC_E_ARG)]


def own(call, wrong):
    """The changes that this call has an argument for."""
    names = call.__code__.co_varnames[:call.__code__.co_argcount]
    return {k: v for k, v in wrong.items() if k in names}


@pytest.mark.parametrize("wrong,status", SHARED + [
    ({"h": 0}, zvc.ZVC_E_ARG), ({"h": H + 1}, zvc.ZVC_E_ALIGN), ({"ldh": 31}, zvc.ZVC_E_ARG), ({"h": X + 64}, zvc.ZVC_E_ARG),
    ({"h": WG}, zvc.ZVC_E_ARG), ({"gate": H, "up": UP}, zvc.ZVC_E_ARG), ({"gate": GATE, "up": GATE + 2}, zvc.ZVC_E_ARG),
    ({"h": X + 66, "ldh": 96, "ldx": 96}, zvc.ZVC_E_ARG)])
def test_forward_refuses(lib, wrong, status):
    assert forward(lib, **own(forward, wrong)) == status


@pytest.mark.parametrize("wrong,status", SHARED + [
    ({"dh": 0}, zvc.ZVC_E_ARG), ({"lddh": 31}, zvc.ZVC_E_ARG), ({"lddx": 63}, zvc.ZVC_E_ARG), ({"lddw": 63}, zvc.ZVC_E_ARG),
    ({"dwg": 0}, zvc.ZVC_E_ARG), ({"dwu": 0}, zvc.ZVC_E_ARG), ({"dx": X}, zvc.ZVC_E_ARG), ({"dwg": WG}, zvc.ZVC_E_ARG),
    ({"dwu": DWG + 64}, zvc.ZVC_E_ARG), ({"dx": DX + 1}, zvc.ZVC_E_ALIGN), ({"dh": DH + 1}, zvc.ZVC_E_ALIGN)])
def test_backward_refuses(lib, wrong, status):
    assert backward(lib, **own(backward, wrong)) == status


def dropout(lib, x=X, ldx=64, res=0, ldr=64, y=Y, ldy=64, rows=16, cols=64, type=2, drop=1 << 30, word=0):
    return lib.zvc_dropout(x, ldx, res, ldr, y, ldy, rows, cols, type, drop, 1, 2, word, None)


@pytest.mark.parametrize("wrong,status", [
    ({"type": 7}, zvc.ZVC_E_ARG), ({"drop": (1 << 32) + 1}, zvc.ZVC_E_ARG), ({"word": 12}, zvc.ZVC_E_ALIGN),
    ({"x": 0}, zvc.ZVC_E_ARG), ({"y": 0}, zvc.ZVC_E_ARG), ({"x": X + 1}, zvc.ZVC_E_ALIGN), ({"ldx": 63}, zvc.ZVC_E_ARG),
    ({"ldy": 10}, zvc.ZVC_E_ARG), ({"res": RES, "ldr": 5}, zvc.ZVC_E_ARG), ({"res": RES + 1}, zvc.ZVC_E_ALIGN),
    ({"y": X + 64}, zvc.ZVC_E_ARG), ({"y": X, "ldy": 80}, zvc.ZVC_E_ARG), ({"res": Y + 2}, zvc.ZVC_E_ARG),
    ({"rows": 1 << 40, "cols": 1 << 20, "ldx": 1 << 20, "ldy": 1 << 20}, zvc.ZVC_E_ARG),
    ({"rows": 1 << 63}, zvc.ZVC_E_ARG)])
def test_dropout_refuses(lib, wrong, status):
    assert dropout(lib, **wrong) == status


def test_empty_calls_do_nothing(lib):
    """No GPU here: a launch would be an error."""
    assert dropout(lib, rows=0) == dropout(lib, cols=0) == zvc.ZVC_OK
    assert forward(lib, m=0) == forward(lib, n=0) == zvc.ZVC_OK
    assert backward(lib, m=0, n=0) == backward(lib, k=0) == backward(lib, dx=0, dwg=0, dwu=0) == zvc.ZVC_OK


def test_python_refuses():
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    h, ws = torch.zeros(4, 6), torch.zeros(1024, dtype=torch.uint8)

    def refused(match, call, *args, **kwargs):
        with pytest.raises(zvc.ZvcError, match=match) as error:
            call(*args, **kwargs)
        assert error.value.status == zvc.ZVC_E_ARG

    refused("element type", ffn.zvc_glu_forward, x.double(), w, w, h, ws)
    refused("activation", ffn.zvc_glu_forward, x, w, w, h, ws, activation="tanh")
    refused("h is", ffn.zvc_glu_forward, x, w, w, h[:3], ws)
    refused("w_up is", ffn.zvc_glu_forward, x, w, w[:5], h, ws)
    refused("2-D", ffn.zvc_glu_forward, x[0], w, w, h, ws)
    refused("strides", ffn.zvc_glu_forward, torch.zeros(8, 4).t(), w, w, h, ws)
    refused("strides", ffn.zvc_glu_backward, torch.zeros(1, 6).expand(4, 6), x, w, w, None, None, None, ws)
    refused("go together", ffn.zvc_glu_forward, x, w, w, h, ws, gate=h.clone())
    refused("different row strides", ffn.zvc_glu_forward, x, w, torch.zeros(6, 9)[:, :8], h, ws)
    refused("torch.float16", ffn.zvc_glu_forward, x, w.half(), w, h, ws)
    refused("p = 1.5", ffn.zvc_glu_forward, x, w, w, h, ws, p=1.5)
    refused("p = nan", ffn.zvc_dropout, x, x, math.nan, 0)
    refused("int64", ffn.zvc_dropout, x, x, 0.5, 0, d_offset=torch.zeros(1))
    refused("y is", ffn.zvc_dropout, x, h, 0.5, 0)
    refused("contiguous or 2-D", ffn.zvc_dropout, torch.zeros(2, 3, 4).transpose(0, 1), torch.zeros(3, 2, 4), 0.5, 0)
    refused("one GPU", ffn.zvc_dropout, x, x.clone(), 0.5, 0)
    refused("one GPU", ffn.zvc_glu_forward, x, w, w, h, ws)
    refused("one GPU", ffn.zvc_glu_backward, h, x, w, w, x.clone(), w.clone(), w.clone(), ws)


def test_calls_through_ctypes_give_the_same(lib, monkeypatch):
    import sys
    args = (16, 32, 64, 2, 1, 0)
    want = ffn._native().zvc_glu_workspace_bytes(*args)
    monkeypatch.setattr(ffn, "_calls", None)
    monkeypatch.setitem(sys.modules, "paper_1705_01626_amd._calls", None)
    with pytest.warns(RuntimeWarning, match="ctypes"):
        assert ffn._native().zvc_glu_workspace_bytes(*args) == want > 0


# ---- the reference ------------------------------------------------------------------
@pytest.mark.parametrize("counter,key,want", [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))])
def test_generator_against_its_published_answers(counter, key, want):
    assert tuple(int(v[0]) for v in ffn_ref.philox(counter, key)) == want


@pytest.mark.parametrize("p", [0.001, 0.1, 0.5, 0.9])
def test_share_of_dropped_elements(p):
    """Within five standard deviations of p; and neighbours drop independently."""
    n = 1 << 18
    stays = ffn_ref.kept(1, n, p, 77, 5)[0].numpy()
    assert abs((~stays).mean() - p) < 5 * math.sqrt(p * (1 - p) / n)
    both = (~stays[1:] & ~stays[:-1]).mean()
    assert abs(both - p * p) < 5 * math.sqrt(p * p * (1 - p * p) / n) + 1e-9
    assert not np.array_equal(stays, ffn_ref.kept(1, n, p, 78, 5)[0].numpy())
    assert not np.array_equal(stays, ffn_ref.kept(1, n, p, 77, 6)[0].numpy())


@pytest.mark.parametrize("name", ["relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("p", [0.0, 0.4])
def test_reference_gradients_against_differences(name, p):
    gen = torch.Generator().manual_seed(4)
    make = lambda *shape: torch.randn(*shape, generator=gen, dtype=torch.float64)
    x, wg, wu, dh = make(5, 7), make(6, 7), make(6, 7), make(5, 6)
    ffn_ref.ROUND[torch.float64] = (2.0 ** -53, 0.0)

    def loss(x, wg, wu):
        return float((ffn_ref.forward(x, wg, wu, name, p, 3, 9)[0][0] * dh).sum())

    for t, (grad, _) in zip((x, wg, wu), ffn_ref.backward(dh, x, wg, wu, name, None, None, p, 3, 9)):
        for i in range(t.numel()):
            at, step = t.view(-1)[i].item(), 1e-6
            t.view(-1)[i] = at + step
            above = loss(x, wg, wu)
            t.view(-1)[i] = at - step
            below = loss(x, wg, wu)
            t.view(-1)[i] = at
            assert abs((above - below) / (2 * step) - grad.reshape(-1)[i].item()) < 1e-7
