"""What the kernels of libzvc_ffn.so may rely on, read from their assembly (no GPU)."""
import re

import pytest

from paper_1705_01626_amd import build as zvc_build
from tests import test_device_code


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    zvc_build.ensure_built()
    with pytest.MonkeyPatch.context() as patch:
        patch.setattr(zvc_build, "ensure_built", lambda: zvc_build.FFN_LIBRARY)
        return test_device_code.assembly.__wrapped__(tmp_path_factory)


def test_loads_past_an_operand_are_in_the_range_check(assembly):
    """Lanes without an element read at an offset past the buffer's end.  The range check knows a load's vector
    and immediate offset alone."""
    loads = re.findall(r"buffer_load_\w+ +v\d+, s\[[\d:]+\], (\w+) offen lds", assembly)
    assert len(loads) == len(re.findall(r"\bbuffer_load_.* lds", assembly)) > 100
    assert set(loads) == {"0"}


def test_no_packed_fp32_arithmetic(assembly):
    assert not re.findall(r"\bv_pk_(?:add|mul|fma)_f32\b", assembly)


def test_16_bit_products_run_on_matrix_instructions_without_a_detour(assembly):
    """Between the first and the last one of the large tiles' kernels sums stay where they are: no spill is read back."""
    parts = re.split(r"^[0-9a-f]+ <(\w+)>:$", assembly, flags=re.M)
    kernels = {k: body for k, body in zip(parts[1::2], parts[2::2]) if re.search(r"(14product|\d16gradients)_kernelIDF16b?_?[LN].*Li4ELi2ELi4ELi8E", k)}
    assert len(kernels) == 6
    for name, body in kernels.items():
        lines = body.splitlines()
        products = [i for i, line in enumerate(lines) if "v_mfma_f32_16x16x32" in line]
        assert len(products) >= 64
        inside = "\n".join(lines[products[0]:products[-1]])
        assert "scratch_load" not in inside and "scratch_store" not in inside, name
