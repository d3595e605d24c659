"""What the kernels of libzvc_experts.so and libzvc_adamw.so may rely on, read from their assembly (no GPU): the checks that
libzvc_ffn.so's have."""
import re

import pytest

from paper_1705_01626_amd import build as zvc_build
from tests import test_device_code, test_ffn_device_code, test_ffn_device_m0


def listing(tmp_path_factory, library):
    zvc_build.ensure_built()
    with pytest.MonkeyPatch.context() as patch:
        patch.setattr(zvc_build, "ensure_built", lambda: library)
        return test_device_code.assembly.__wrapped__(tmp_path_factory)


@pytest.fixture(scope="module")
def experts_assembly(tmp_path_factory):
    return listing(tmp_path_factory, zvc_build.EXPERTS_LIBRARY)


@pytest.fixture(scope="module")
def adamw_assembly(tmp_path_factory):
    return listing(tmp_path_factory, zvc_build.ADAMW_LIBRARY)


def test_no_packed_fp32_arithmetic(experts_assembly, adamw_assembly):
    test_ffn_device_code.test_no_packed_fp32_arithmetic(experts_assembly)
    test_ffn_device_code.test_no_packed_fp32_arithmetic(adamw_assembly)


def test_loads_past_an_operand_are_in_the_range_check(experts_assembly):
    test_ffn_device_code.test_loads_past_an_operand_are_in_the_range_check(experts_assembly)


def test_m0_is_only_written_for_the_load_behind_it(experts_assembly):
    test_ffn_device_m0.test_m0_is_only_written_for_the_load_behind_it(experts_assembly)


def test_large_tiles_keep_their_sums_in_registers(experts_assembly):
    """Between the first and the last matrix instruction of the large tiles' kernels nothing is spilled or read back."""
    parts = re.split(r"^[0-9a-f]+ <(\w+)>:$", experts_assembly, flags=re.M)
    kernels = {k: body for k, body in zip(parts[1::2], parts[2::2]) if re.search(r"expert_(product|gradients)_kernelIDF16b?_?N.*Li4ELi2ELi4ELi8E", k)}
    assert len(kernels) == 4
    for name, body in kernels.items():
        lines = body.splitlines()
        products = [i for i, line in enumerate(lines) if "v_mfma_f32_16x16x32" in line]
        assert len(products) >= 64
        inside = "\n".join(lines[products[0]:products[-1]])
        assert "scratch_load" not in inside and "scratch_store" not in inside, name


def test_the_steps_products_are_rounded_before_they_are_added(adamw_assembly):
    """m and v are sums of two rounded products each; the only fused instructions are those of the square root and of the powers."""
    body = adamw_assembly
    assert len(re.findall(r"\bv_sqrt_f32", body)) >= 100
    # (a correctly rounded square root takes two)
    assert len(re.findall(r"\bv_(?:fma|fmac|mad|mac)_f32", body)) <= 2 * len(re.findall(r"\bv_sqrt_f32", body))
