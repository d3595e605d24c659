"""Where the stores of libzvc_ffn.so's kernels go, read from their assembly (no GPU)."""
import re

from tests.test_device_code import functions
from tests.test_ffn_device_code import assembly  # noqa: F401 (a fixture)


def test_dropout_leaves_its_output_to_the_caches(assembly):  # noqa: F811
    """The next operation reads it: past the caches the call alone is faster and the two together slower."""
    kernels = functions(assembly, "dropout_kernel")
    assert len(kernels) == 3
    for name, body in kernels.items():
        stores = re.findall(r"^\s*(global_store_\w+ .*?)(?:\s*//.*)?$", body, flags=re.M)
        assert len(stores) >= 2 and not any(re.search(r"\bnt\b", x) for x in stores), name


def test_large_tiles_have_both_kinds_of_stores(assembly):  # noqa: F811
    """A call that asks for stores past the caches gets them, and one that does not does not: of two alike behind a branch the
    compiler would have made one."""
    kernels = {name: body for name, body in functions(assembly, "product_kernel").items()
               if "DoesE0E" in name and "Li4ELi2ELi4ELi8E" in name}
    assert len(kernels) == 2
    for name, body in kernels.items():
        stores = re.findall(r"^\s*(global_store_dwordx4 .*?)(?:\s*//.*)?$", body, flags=re.M)
        past = sum(bool(re.search(r"\bnt\b", x)) for x in stores)
        assert past >= 6 * 8 and len(stores) - past >= 6 * 8, name            # four activations, gate and up; eight rows a lane
