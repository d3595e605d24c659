"""Which kernels the training operators launch for which sizes, written down by a stand-in for the HIP runtime
(fake_hip_launches.cpp) in a child process: that the sizes of the GPU tests launch the kernels that they are meant for,
and that no kernel is built that no call launches.  No GPU needed."""
import itertools
import json
import os
import re
import subprocess
import sys

import pytest

from paper_1705_01626_amd import build as zvc_build
from tests.ffn_routes import ROUTES
from tests.test_device_code import tool

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FP32, FP16, BF16 = range(3)
CHILD = """
import ctypes, json, sys
fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
fake.fake_log.restype = fake.fake_kernels.restype = ctypes.c_char_p
lib.zvc_glu_workspace_bytes.restype = ctypes.c_size_t
def call(name, args):
    fake.fake_clear()
    status = getattr(lib, name)(*[ctypes.c_size_t(a) for a in args])
    return [status, fake.fake_log().decode().splitlines()]
calls = json.loads(sys.stdin.read())
print(json.dumps([fake.fake_kernels().decode().split(), [call(*c) for c in calls]]))
"""
AT = [(i + 1) << 44 for i in range(10)]
ROOM = 1 << 43
SHAPES = {(4, 2, 4, 8, 2): "large", (2, 2, 4, 4, 2): "small", (2, 4, 4, 2, 2): "eights", (4, 1, 4, 2, 2): "thin",
          (2, 4, 4, 2, 4): "lone", (2, 2, 4, 2, 4): "half"}


@pytest.fixture(scope="module")
def fake(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("fake") / "libfake_hip_launches.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I", zvc_build.ROCM_INCLUDE,
                    "-o", out, os.path.join(ROOT, "tests", "fake_hip_launches.cpp")], check=True)
    return out


class Launch:
    def __init__(self, line):
        self.name = line.split()[0]
        self.values = {k: int(v) for k, v in re.findall(r"(\w+)=(\d+)", line)}
        self.kernel = re.search(r"\d+([a-z_]+_kernel)I", self.name).group(1)

    def cut(self, of):
        v = self.values
        return "whole" if v[of + "_parts"] == 1 else "mixed" if v[of + "_whole"] else "split"

    def route(self):
        if self.kernel == "token_kernel":
            return "tokens"
        numbers = re.search(r"5ShapeI((?:Li\d+E)+)", self.name).group(1)
        shape = SHAPES[tuple(int(i) for i in re.findall(r"\d+", numbers))]
        if self.kernel == "product_kernel":
            return "%s %s" % (shape, self.cut("p"))
        return "%s %s, %s%s" % (shape, self.cut("dx"), self.cut("dw"), ", ahead" if self.values["ahead"] else "")


def run(fake, calls):
    """The library's kernels, and (status, launches) of each call."""
    zvc_build.ensure_built()
    done = subprocess.run([sys.executable, "-c", CHILD, fake, zvc_build.FFN_LIBRARY], input=json.dumps(calls),
                          capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
    kernels, results = json.loads(done.stdout)
    return set(kernels), [(status, [Launch(line) for line in lines]) for status, lines in results]


def forward(m, n, k, dtype, keep=False, drop=0, room=ROOM, h=AT[3], ldh=0, gate=AT[4], ldp=0):
    return ["zvc_glu_forward", [AT[0], k, AT[1], AT[2], k, h, ldh or n, gate * keep, AT[5] * keep, ldp or n, m, n, k, dtype, 1, drop, 1,
                                2, 0, AT[9], room, 0]]


def backward(m, n, k, dtype, keep=False, drop=0, room=ROOM):
    return ["zvc_glu_backward", [AT[6], n, AT[0], k, AT[1], AT[2], k, AT[4] * keep, AT[5] * keep, n, AT[3], k, AT[7], AT[8], k,
                                 m, n, k, dtype, 1, drop, 1, 2, 0, AT[9], room, 0]]


def dropout(rows, cols, dtype, ld=None):
    ld = ld or cols
    return ["zvc_dropout", [AT[0], ld, 0, cols, AT[3], ld, rows, cols, dtype, 1 << 31, 1, 2, 0, 0]]


def test_sizes_launch_what_the_gpu_tests_are_for(fake):
    calls = [c for size in ROUTES for dtype in (BF16, FP16, FP32)
             for c in (forward(*size, dtype), backward(*size, dtype), backward(*size, dtype, True))]
    _, results = run(fake, calls)
    results = iter(results)
    for size, routes in ROUTES.items():
        for dtype in (BF16, FP16, FP32):
            projection, gradients = routes[2:] if dtype == FP32 else routes[:2]
            for again, keep in ((False, False), (True, False), (True, True)):
                status, launches = next(results)
                assert status == 0
                names = [x.kernel for x in launches if x.kernel not in ("join_kernel", "join_gradients_kernel", "align_kernel")]
                got = [x.route() for x in launches if x.kernel in ("product_kernel", "token_kernel", "gradients_kernel")]
                want = ([] if keep else [projection]) + ([gradients] if again else [])
                assert got == want and (names[0] == "slope_kernel") == keep, (size, dtype, got, want)


def test_every_cut_is_among_them():
    for column in range(4):
        seen = {r for size, routes in ROUTES.items() for r in [routes[column]]}
        if column % 2 == 0:
            shapes = ("large", "eights", "thin", "lone", "half") if column == 0 else ("eights", "thin")
            assert seen >= {"tokens", *(" ".join(c) for c in itertools.product(shapes, ("whole", "split", "mixed")))}
        else:
            for shape in ("large", "small", "thin") if column == 1 else ("small", "thin"):
                assert any(r.startswith(shape) and r.endswith("ahead") for r in seen)
                for place in (0, 1):
                    cuts = {r.split(" ", 1)[1].split(", ")[place] for r in seen if r.startswith(shape)}
                    assert cuts >= ({"whole", "split"} if (column, shape) == (1, "thin") else {"whole", "split", "mixed"})


def device_kernels(where):
    """The kernels of the library's code object: it can hold some that the host side never names."""
    fat, code = str(where / "fat"), str(where / "gfx950.co")
    subprocess.run([tool("llvm-objcopy"), "--dump-section", ".hip_fatbin=" + fat, zvc_build.FFN_LIBRARY, str(where / "rest.so")],
                   check=True)
    subprocess.run([tool("clang-offload-bundler"), "--unbundle", "--type=o", "--targets=hipv4-amdgcn-amd-amdhsa--gfx950",
                    "--input=" + fat, "--output=" + code], check=True)
    symbols = subprocess.run([tool("llvm-objdump"), "--syms", code], check=True, capture_output=True, text=True).stdout
    return set(re.findall(r"\b(\w+)\.kd$", symbols, flags=re.M))


def test_no_kernel_is_built_that_no_call_launches(fake, tmp_path):
    """The sizes above, some that take copies of unaligned inputs, numbers of tokens around each kernel for few, and dropout."""
    calls = [c for size in ROUTES for dtype in (BF16, FP16, FP32)
             for c in (forward(*size, dtype), backward(*size, dtype), backward(*size, dtype, True))]
    calls += [c for m in (1, 17, 33, 49, 65, 97) for dtype in (BF16, FP16, FP32) for c in (forward(m, 40, 33, dtype), backward(m, 40, 33, dtype))]
    calls += [dropout(rows, cols, dtype) for rows, cols in ((3, 100), (8192, 4096)) for dtype in (BF16, FP16, FP32)]
    kernels, results = run(fake, calls)
    assert all(status == 0 for status, _ in results)
    launched = {x.name for _, launches in results for x in launches}
    assert launched == kernels == device_kernels(tmp_path)


@pytest.mark.parametrize("dtype,each", [(BF16, 16), (FP32, 8)])
def test_a_dimension_of_dropouts_grid_holds_its_lanes(fake, dtype, each):
    """A dimension has fewer than 2^32 lanes; all of them together have every element."""
    sizes = [(1, 1), (1, 1 << 20), (1, (1 << 31) + 5), (1, (1 << 35) + 8), (1, 1 << 36), (1 << 20, (1 << 16) + 8), (1, 1 << 40)]
    _, results = run(fake, [dropout(rows, cols, dtype) for rows, cols in sizes])
    for (rows, cols), (status, launches) in zip(sizes, results):
        v = launches[0].values
        assert status == 0 and len(launches) == 1
        assert v["grid"] * v["block"] < 1 << 32 and v["rows"] < 1 << 16 and v["depth"] == 1
        assert v["rows"] == 1 or v["grid"] == 1 << 20             # (the kernel numbers workgroups by it)
        lanes = v["grid"] * v["rows"] * v["block"]
        assert rows * cols <= lanes * each and (v["rows"] - 1) * (1 << 20) * v["block"] * each < rows * cols


@pytest.mark.parametrize("past,call", [
    # as much as the caches hold, 256 MB, or more
    (1, {"m": 16384, "n": 8192, "k": 512}), (0, {"m": 16383, "n": 8192, "k": 512}), (1, {"m": 16384, "n": 11264, "k": 4096}),
    (1, {"m": 16384, "n": 2816, "k": 1024, "keep": True}), (0, {"m": 16384, "n": 2816, "k": 1024}),
    # behind long sums more than 32 MB of h
    (1, {"m": 4096, "n": 5632, "k": 2048}), (0, {"m": 4096, "n": 5632, "k": 2047, "keep": True}), (0, {"m": 4096, "n": 4096, "k": 2048}),
    (1, {"m": 4097, "n": 4096, "k": 4096}), (0, {"m": 1024, "n": 8192, "k": 128, "keep": True}), (0, {"m": 2000, "n": 2056, "k": 136}),
    # rows in whole halves of 128 bytes
    (1, {"m": 16384, "n": 11296, "k": 4096}), (0, {"m": 16384, "n": 11288, "k": 4096}), (0, {"m": 16384, "n": 11264, "k": 4096, "h": AT[3] + 32}),
    (0, {"m": 16384, "n": 11264, "k": 4096, "ldh": 11272}), (1, {"m": 16384, "n": 11264, "k": 4096, "ldh": 11296}),
    (0, {"m": 16384, "n": 11264, "k": 4096, "keep": True, "gate": AT[4] + 16}), (0, {"m": 16384, "n": 11264, "k": 4096, "keep": True, "ldp": 11265}),
    (1, {"m": 16384, "n": 11264, "k": 4096, "ldp": 11265})])
def test_what_goes_past_the_caches(fake, past, call):
    """A forward call's outputs where the caches do not hold them or the products take long, written in whole pieces; never dg and du,
    which are read next."""
    for dtype in (BF16, FP16):
        _, results = run(fake, [forward(dtype=dtype, **call), backward(call["m"], call["n"], call["k"], dtype)])
        (status, first), (_, again) = results
        product = [x for x in first if x.kernel == "product_kernel"]
        assert status == 0 and product[0].route().startswith("large") and product[0].values["p_past"] == past
        assert all(x.values.get(of + "_past", 0) == 0 for x in again for of in ("p", "dx", "dw"))
