"""The host side of the operators for mixtures of experts: exports, refusals before any GPU call, workspaces, which kernels are
launched, and the reference that the GPU tests use.  No GPU needed."""
import json
import math
import os
import re
import subprocess
import sys

import pytest
import torch

from paper_1705_01626_amd import build as zvc_build
from paper_1705_01626_amd import experts, zvc
from tests import experts_ref
from tests.experts_sizes import SIZES
from tests.test_ffn_launches import CHILD, fake  # noqa: F401 (a fixture)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
X, W, Y, DY, DX, DW, OFF, WS = ((i + 1) << 44 for i in range(8))
LOGITS, CHOSEN, WEIGHTS, ORDER, PLACE = ((i + 16) << 44 for i in range(5))
BIG = 1 << 43
FP32, FP16, BF16 = range(3)


@pytest.fixture(scope="module")
def lib():
    zvc_build.ensure_built()
    return experts.load()


def test_exports_every_declared_symbol(lib):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "zvc_experts.h")).read(), flags=re.S)
    assert set(re.findall(r"\b(zvc_[a-z_]+)\s*\(", header)) == set(experts.EXPORTS)
    for name in experts.EXPORTS:
        assert getattr(lib, name) is not None


@pytest.mark.parametrize("header", ["zvc_experts.h", "zvc_adamw.h"])
def test_header_is_plain_c(tmp_path, header):
    source = tmp_path / "client.c"
    source.write_text('#include "%s"\nint main(void) { return 0; }\n' % header)
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"),
                    "-I", zvc_build.ROCM_INCLUDE, "-c", str(source), "-o", str(tmp_path / "client.o")], check=True)


def route(lib, logits=LOGITS, ldl=64, chosen=CHOSEN, weights=WEIGHTS, offsets=OFF, order=ORDER, place=PLACE, m=100, e=64, top=4, type=2,
          norm=1, ws=WS, room=BIG):
    return lib.zvc_route(logits, ldl, chosen, weights, offsets, order, place, m, e, top, type, norm, ws, room, None)


@pytest.mark.parametrize("wrong,status", [
    ({"type": 3}, zvc.ZVC_E_ARG), ({"e": 0}, zvc.ZVC_E_ARG), ({"e": 1025, "ldl": 2000}, zvc.ZVC_E_ARG), ({"top": 0}, zvc.ZVC_E_ARG),
    ({"top": 17}, zvc.ZVC_E_ARG), ({"top": 4, "e": 3}, zvc.ZVC_E_ARG), ({"ldl": 63}, zvc.ZVC_E_ARG), ({"m": (1 << 25) + 1}, zvc.ZVC_E_ARG),
    ({"logits": 0}, zvc.ZVC_E_ARG), ({"chosen": 0}, zvc.ZVC_E_ARG), ({"weights": 0}, zvc.ZVC_E_ARG), ({"offsets": 0}, zvc.ZVC_E_ARG),
    ({"order": 0}, zvc.ZVC_E_ARG), ({"place": 0}, zvc.ZVC_E_ARG), ({"ws": 0}, zvc.ZVC_E_ARG), ({"logits": LOGITS + 1}, zvc.ZVC_E_ALIGN),
    ({"chosen": CHOSEN + 2}, zvc.ZVC_E_ALIGN), ({"weights": WEIGHTS + 2}, zvc.ZVC_E_ALIGN), ({"offsets": OFF + 4}, zvc.ZVC_E_ALIGN),
    ({"order": ORDER + 4}, zvc.ZVC_E_ALIGN), ({"place": PLACE + 4}, zvc.ZVC_E_ALIGN), ({"ws": WS + 128}, zvc.ZVC_E_ALIGN),
    ({"room": 0}, zvc.ZVC_E_WORKSPACE), ({"weights": CHOSEN}, zvc.ZVC_E_ARG), ({"order": LOGITS + 64}, zvc.ZVC_E_ARG), ({"place": WS + 8}, zvc.ZVC_E_ARG)])
def test_route_refuses(lib, wrong, status):
    assert route(lib, **wrong) == status


def route_backward(lib, dw=WEIGHTS, logits=LOGITS, ldl=64, chosen=CHOSEN, out=DX, ldd=64, m=100, e=64, top=4, type=2):
    return lib.zvc_route_backward(dw, logits, ldl, chosen, out, ldd, m, e, top, type, 1, None)


@pytest.mark.parametrize("wrong,status", [
    ({"type": -1}, zvc.ZVC_E_ARG), ({"top": 65}, zvc.ZVC_E_ARG), ({"ldd": 63}, zvc.ZVC_E_ARG), ({"dw": 0}, zvc.ZVC_E_ARG), ({"logits": 0}, zvc.ZVC_E_ARG),
    ({"chosen": 0}, zvc.ZVC_E_ARG), ({"out": 0}, zvc.ZVC_E_ARG), ({"out": LOGITS}, zvc.ZVC_E_ARG), ({"out": CHOSEN + 16}, zvc.ZVC_E_ARG),
    ({"out": DX + 1}, zvc.ZVC_E_ALIGN), ({"dw": WEIGHTS + 1}, zvc.ZVC_E_ALIGN)])
def test_route_backward_refuses(lib, wrong, status):
    assert route_backward(lib, **wrong) == status
    assert route_backward(lib, m=0) == zvc.ZVC_OK


def product(lib, x=X, ldx=64, w=W, ldw=64, sw=32 * 64, off=OFF, y=Y, ldy=32, m=16, e=5, n=32, k=64, type=2, ws=WS, room=BIG):
    return lib.zvc_expert_product(x, ldx, w, ldw, sw, off, y, ldy, m, e, n, k, type, ws, room, None)


def gradients(lib, dy=DY, lddy=32, x=X, ldx=64, w=W, ldw=64, sw=32 * 64, off=OFF, dx=DX, lddx=64, dw=DW, lddw=64, sdw=32 * 64, m=16, e=5, n=32, k=64,
              type=2, ws=WS, room=BIG):
    return lib.zvc_expert_gradients(dy, lddy, x, ldx, w, ldw, sw, off, dx, lddx, dw, lddw, sdw, m, e, n, k, type, ws, room, None)


SHARED = [({"type": 3}, zvc.ZVC_E_ARG), ({"e": 0}, zvc.ZVC_E_ARG), ({"e": 1025}, zvc.ZVC_E_ARG), ({"ldx": 63}, zvc.ZVC_E_ARG), ({"ldw": 63}, zvc.ZVC_E_ARG),
          ({"sw": 32 * 64 - 1}, zvc.ZVC_E_ARG), ({"ldx": (1 << 21) + 1}, zvc.ZVC_E_ARG), ({"m": (1 << 28) + 1}, zvc.ZVC_E_ARG),
          ({"k": (1 << 21) + 1, "ldx": 1 << 22, "ldw": 1 << 22}, zvc.ZVC_E_ARG), ({"x": 0}, zvc.ZVC_E_ARG), ({"w": 0}, zvc.ZVC_E_ARG), ({"off": 0}, zvc.ZVC_E_ARG),
          ({"ws": 0}, zvc.ZVC_E_ARG), ({"x": X + 1}, zvc.ZVC_E_ALIGN), ({"w": W + 2, "type": 0}, zvc.ZVC_E_ALIGN), ({"off": OFF + 4}, zvc.ZVC_E_ALIGN),
          ({"ws": WS + 128}, zvc.ZVC_E_ALIGN), ({"room": 0}, zvc.ZVC_E_WORKSPACE), ({"ws": W + 256}, zvc.ZVC_E_ARG)]


@pytest.mark.parametrize("wrong,status", SHARED + [
    ({"y": 0}, zvc.ZVC_E_ARG), ({"ldy": 31}, zvc.ZVC_E_ARG), ({"y": Y + 1}, zvc.ZVC_E_ALIGN), ({"y": X + 64}, zvc.ZVC_E_ARG), ({"y": W + 4 * 4096}, zvc.ZVC_E_ARG),
    ({"y": OFF + 8}, zvc.ZVC_E_ARG), ({"y": WS}, zvc.ZVC_E_ARG)])
def test_product_refuses(lib, wrong, status):
    assert product(lib, **wrong) == status


@pytest.mark.parametrize("wrong,status", SHARED + [
    ({"dy": 0}, zvc.ZVC_E_ARG), ({"lddy": 31}, zvc.ZVC_E_ARG), ({"lddx": 63}, zvc.ZVC_E_ARG), ({"lddw": 63}, zvc.ZVC_E_ARG), ({"sdw": 64}, zvc.ZVC_E_ARG),
    ({"dx": DX + 1}, zvc.ZVC_E_ALIGN), ({"dw": DW + 1}, zvc.ZVC_E_ALIGN), ({"dx": X}, zvc.ZVC_E_ARG), ({"dw": W + 2}, zvc.ZVC_E_ARG), ({"dw": DX + 64}, zvc.ZVC_E_ARG),
    ({"dx": OFF}, zvc.ZVC_E_ARG)])
def test_gradients_refuses(lib, wrong, status):
    assert gradients(lib, **wrong) == status


def test_empty_calls_do_nothing(lib):
    """No GPU here: a launch would be an error."""
    assert product(lib, m=0) == product(lib, n=0) == zvc.ZVC_OK
    assert gradients(lib, k=0) == gradients(lib, dx=0, dw=0) == gradients(lib, dw=0, m=0) == gradients(lib, dx=0, n=0) == zvc.ZVC_OK


def test_python_refuses():
    logits, ws = torch.zeros(4, 8), torch.zeros(4096, dtype=torch.uint8)
    chosen, weights, offsets = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(9, dtype=torch.int64)
    order, place = torch.zeros(8, dtype=torch.int64), torch.zeros(4, 2, dtype=torch.int64)

    def refused(match, call, *args, **kwargs):
        with pytest.raises(zvc.ZvcError, match=match) as error:
            call(*args, **kwargs)
        assert error.value.status == zvc.ZVC_E_ARG

    r = experts.zvc_route
    refused("element type", r, logits.double(), chosen, weights, offsets, order, place, ws)
    refused("2-D", r, logits[0], chosen, weights, offsets, order, place, ws)
    refused("chosen is", r, logits, chosen.long(), weights, offsets, order, place, ws)
    refused("weights is", r, logits, chosen, weights[:, :1], offsets, order, place, ws)
    refused("offsets is", r, logits, chosen, weights, offsets[:8], order, place, ws)
    refused("order is", r, logits, chosen, weights, offsets, place, place, ws)
    refused("strides", r, logits, chosen, weights, offsets, order, torch.zeros(2, 4, dtype=torch.int64).t(), ws)
    refused("workspace has strides", r, logits, chosen, weights, offsets, order, place, ws[::2])
    refused("one GPU", r, logits, chosen, weights, offsets, order, place, ws)
    refused("dlogits is", experts.zvc_route_backward, weights, logits, chosen, logits[:, :7])
    refused("dweights is", experts.zvc_route_backward, weights.half(), logits, chosen, logits.clone())
    refused("one GPU", experts.zvc_route_backward, weights, logits, chosen, logits.clone())
    x, w, y, off = torch.zeros(6, 16), torch.zeros(3, 10, 16), torch.zeros(6, 10), torch.zeros(4, dtype=torch.int64)
    refused("3-D", experts.zvc_expert_product, x, w[0], off, y, ws)
    refused("x is", experts.zvc_expert_product, x, w[:, :, :15], off, y, ws)
    refused("w has strides", experts.zvc_expert_product, x, torch.zeros(1, 10, 16).expand(3, 10, 16), off, y, ws)
    refused("w has strides", experts.zvc_expert_product, x, torch.zeros(3, 16, 10).transpose(1, 2), off, y, ws)
    refused("y is", experts.zvc_expert_product, x, w, off, y[:5], ws)
    refused("offsets is", experts.zvc_expert_product, x, w, off.int(), y, ws)
    refused("torch.float16", experts.zvc_expert_product, x, w.half(), off, y, ws)
    refused("one GPU", experts.zvc_expert_product, x, w, off, y, ws)
    refused("dy is", experts.zvc_expert_gradients, x, x, w, off, None, None, ws)
    refused("dw is", experts.zvc_expert_gradients, y, x, w, off, None, w[:2], ws)
    refused("dx has strides", experts.zvc_expert_gradients, y, x, w, off, torch.zeros(16, 6).t(), None, ws)
    refused("one GPU", experts.zvc_expert_gradients, y, x, w, off, x.clone(), w.clone(), ws)


def test_strides_of_a_stack():
    w = torch.zeros(3, 10, 24)
    assert experts._stack(w[:, :, :16], 3, 10, 16, w, "call", "w") == (24, 240)
    assert experts._stack(w[:, :4, :16], 3, 4, 16, w, "call", "w") == (24, 240)
    assert experts._stack(w[:1], 1, 10, 24, w, "call", "w") == (24, 240)
    assert experts._stack(w[:, :1], 3, 1, 24, w, "call", "w") == (24, 240)
    assert experts._stack(torch.zeros(3, 0, 24), 3, 0, 24, w, "call", "w")[0] >= 24
    far = torch.zeros(1 << 22).as_strided((3, 1, 8), (64, 1 << 21, 1))          # (one row has no next one)
    assert experts._stack(far, 3, 1, 8, far, "call", "w") == (8, 64)


def test_calls_through_ctypes_give_the_same(lib, monkeypatch):
    bad = [0] * 12
    want = experts._native().zvc_route_backward(*bad)
    monkeypatch.setattr(experts, "_calls", None)
    monkeypatch.setitem(sys.modules, "paper_1705_01626_amd._calls", None)
    with pytest.warns(RuntimeWarning, match="ctypes"):
        assert experts._native().zvc_route_backward(*bad) == want == zvc.ZVC_E_ARG


# ---- which kernels, and their workspace ------------------------------------------------
def aligned(x):
    return (x + 7) // 8 * 8


def calls_of(m, e, n, k, type, room, loose):
    """A forward and a backward call."""
    ldk, ldn = (k, n) if loose else (aligned(k), aligned(n))
    return [["zvc_expert_product", [X, ldk, W, ldk, n * ldk, OFF, Y, ldn, m, e, n, k, type, WS, room[0], 0]],
            ["zvc_expert_gradients", [DY, ldn, X, ldk, W, ldk, n * ldk, OFF, DX, ldk, DW, ldk, n * ldk, m, e, n, k, type, WS, room[1], 0]]]


def run(fake, calls):  # noqa: F811
    zvc_build.ensure_built()
    done = subprocess.run([sys.executable, "-c", CHILD.replace("lib.zvc_glu_workspace_bytes.restype = ctypes.c_size_t\n", ""), fake, zvc_build.EXPERTS_LIBRARY],
                          input=json.dumps(calls), capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
    return json.loads(done.stdout)


def test_every_kernel_is_launched(fake, lib, tmp_path):  # noqa: F811
    """And no kernel is in the library that no call launches; grids hold fewer than 2^32 lanes."""
    calls = [c for m, e, n, k in SIZES for type in (FP32, FP16, BF16) for loose in (False, True) for c in calls_of(m, e, n, k, type, (BIG, BIG), loose)]
    # (an odd address: every operand by way of registers)
    calls += [[name, [a + 4 if i in (0, 2, 4) and a >= X else a for i, a in enumerate(args)]] for m, e, n, k in SIZES for type in (FP32, FP16, BF16)
              for name, args in calls_of(m, e, n, k, type, (BIG, BIG), True)]
    calls += [["zvc_route", [LOGITS, e, CHOSEN, WEIGHTS, OFF, ORDER, PLACE, m, e, 2, type, 1, WS, BIG, 0]] for m in (32, 33) for e in (16, 100, 200, 300, 600, 1024)
              for type in (FP32, FP16, BF16)]
    calls += [["zvc_route_backward", [WEIGHTS, LOGITS, e, CHOSEN, DX, e, 33, e, 2, type, 1, 0]] for e in (16, 100, 200, 300, 600, 1024) for type in (FP32, FP16, BF16)]
    kernels, results = run(fake, calls)
    assert all(status == 0 and lines for status, lines in results)
    launched = {line.split()[0] for _, lines in results for line in lines}
    assert launched == set(kernels)
    from tests import test_ffn_launches
    with pytest.MonkeyPatch.context() as patch:
        patch.setattr(zvc_build, "FFN_LIBRARY", zvc_build.EXPERTS_LIBRARY)
        assert launched == test_ffn_launches.device_kernels(tmp_path)
    for _, lines in results:
        for line in lines:
            v = {k: int(n) for k, n in re.findall(r"(\w+)=(\d+)", line)}
            assert v["grid"] * v["block"] < 1 << 32 and v["rows"] == v["depth"] == 1
            if "expert_gradients_kernel" in line or "loose_kernel" in line:
                assert v["grid"] % 8 == 0                        # (dW's tiles are dealt to the XCDs)


def test_the_workspace_that_is_asked_for_is_enough(fake, lib):  # noqa: F811
    """And a byte less is refused."""
    torches = {FP32: torch.float32, FP16: torch.float16, BF16: torch.bfloat16}
    calls = []
    for m, e, n, k in SIZES:
        for type in torches:
            room = [experts.zvc_expert_workspace_bytes(m, e, n, k, torches[type], back) for back in (False, True)]
            assert min(room) >= 256
            calls += calls_of(m, e, n, k, type, room, True) + calls_of(m, e, n, k, type, [r - 1 for r in room], True)
    _, results = run(fake, calls)
    for i in range(0, len(results), 4):
        assert [status for status, _ in results[i:i + 4]] == [0, 0, zvc.ZVC_E_WORKSPACE, zvc.ZVC_E_WORKSPACE]
        assert results[i + 2][1] == results[i + 3][1] == []
    assert experts.zvc_expert_workspace_bytes(1, 1, 1, 1, torch.float64) == 0
    assert experts.zvc_expert_workspace_bytes(1, 1025, 1, 1, torch.float32) == 0
    assert experts.zvc_route_workspace_bytes(4, 8, 9) == 0
    assert 0 < experts.zvc_route_workspace_bytes(32, 64, 8) < experts.zvc_route_workspace_bytes(33, 64, 8) < experts.zvc_route_workspace_bytes(16384, 64, 8)


def test_the_largest_sizes_are_launched_within_a_grids_limits(fake, lib):  # noqa: F811
    most = 1 << 28
    sizes = [(most, 1, 1, 1), (most, 1024, 1, 4096), (most, 1024, 4096, 1), (1, 1024, 1 << 15, 1 << 15), (1 << 19, 1, 1 << 21, 1 << 19), (most, 7, 4096, 4096)]
    _, results = run(fake, [c for m, e, n, k in sizes for type in (FP32, BF16) for loose in (False, True) for c in calls_of(m, e, n, k, type, (BIG, BIG), loose)])
    for status, lines in results:
        assert status == 0 and lines
        for line in lines:
            v = {k: int(n) for k, n in re.findall(r"(\w+)=(\d+)", line)}
            assert v["grid"] * v["block"] < 1 << 32 and v["rows"] == v["depth"] == 1
    _, results = run(fake, [["zvc_route", [LOGITS, 1024, CHOSEN, WEIGHTS, OFF, ORDER, PLACE, 1 << 23, 1024, 16, BF16, 1, WS, BIG, 0]],
                            ["zvc_route_backward", [WEIGHTS, LOGITS, 1, CHOSEN, DX, 1, 1 << 27, 1, 1, FP32, 0, 0]]])
    for status, lines in results:
        assert status == 0
        for line in lines:
            v = {k: int(n) for k, n in re.findall(r"(\w+)=(\d+)", line)}
            assert v["grid"] * v["block"] < 1 << 32


# ---- the reference ------------------------------------------------------------------
def test_reference_of_the_router():
    inf, nan = math.inf, math.nan
    logits = torch.tensor([[1.0, 3.0, 3.0, -inf], [nan, -inf, -inf, nan], [0.0, 0.0, 0.0, 0.0], [-inf, -inf, 5.0, nan]])
    chosen, weights, offsets, order, place = experts_ref.route(logits, 2, True)
    assert chosen == [[1, 2], [-1, -1], [0, 1], [2, -1]]
    assert weights == [[0.5, 0.5], [0, 0], [0.5, 0.5], [1.0, 0]]
    assert offsets == [0, 1, 3, 5, 5] and order == [4, 0, 5, 1, 6, -1, -1, -1]
    assert place == [1, 3, -1, -1, 0, 2, 4, -1]
    weights = experts_ref.route(logits, 2, False)[1]
    assert weights[2] == [0.25, 0.25] and abs(sum(weights[0]) - 2 / (2 + math.exp(-2))) < 1e-15


@pytest.mark.parametrize("normalize", [True, False])
def test_reference_gradient_against_differences(normalize):
    gen = torch.Generator().manual_seed(5)
    logits, dw = torch.randn(4, 6, generator=gen, dtype=torch.float64), torch.randn(4, 3, generator=gen, dtype=torch.float64)
    logits[1, 2] = -math.inf
    logits[2] = -math.inf
    chosen = experts_ref.choose(logits, 3)
    from tests import ffn_ref
    ffn_ref.ROUND[torch.float64] = (2.0 ** -53, 0.0)
    grad = experts_ref.route_backward(dw, logits, chosen, normalize)[0]

    def loss(l):
        assert experts_ref.choose(l, 3) == chosen
        return float((torch.tensor(experts_ref.route(l, 3, normalize)[1], dtype=torch.float64) * dw).sum())

    for t in range(4):
        for e in range(6):
            if logits[t, e] == -math.inf:
                assert grad[t, e] == 0
                continue
            up, down = logits.clone(), logits.clone()
            up[t, e] += 1e-6
            down[t, e] -= 1e-6
            assert abs((loss(up) - loss(down)) / 2e-6 - float(grad[t, e])) < 1e-8
