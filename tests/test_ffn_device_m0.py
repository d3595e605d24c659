"""The inline loads of libzvc_ffn.so write m0, which the compiler reserves and cannot be told of: that it is used by nothing
else, read from the assembly (no GPU)."""
import re

from tests.test_ffn_device_code import assembly  # noqa: F401 (a fixture)


def test_m0_is_only_written_for_the_load_behind_it(assembly):  # noqa: F811
    """Every load to LDS has its own write of m0 two instructions ahead, and nothing else in the library names the register."""
    lines = [line.split("//")[0].strip() for line in assembly.splitlines()]
    loads = [i for i, line in enumerate(lines) if re.match(r"buffer_load_.* lds$", line)]
    uses = [i for i, line in enumerate(lines) if re.search(r"\bm0\b", line)]
    assert len(loads) > 100
    assert uses == [i - 2 for i in loads]
    assert all(re.match(r"s_mov_b32 m0, s\d+$", lines[i]) and lines[i + 1] == "s_nop 0" for i in uses)
    # what uses m0 without naming it
    assert not re.findall(r"\b(?:ds_gws_\w+|s_movrel\w+|v_movrel\w+|s_sendmsg\w*|ds_\w*addtid\w*|global_load_lds_\w+|v_interp_\w+)\b", assembly)
