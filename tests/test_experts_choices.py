"""Which kernel the account takes for sizes at which it was measured, forced in turn: another fit of its rates that takes another one has to measure
them again (no GPU; launches are written down by a stand-in for the HIP runtime)."""
import re

import pytest

from tests.test_experts_host import BF16, BIG, FP16, FP32, calls_of, run
from tests.test_ffn_launches import SHAPES, fake  # noqa: F401 (a fixture)


def kernels(lines):
    """The launches in short: kernel and tile, or kernel, operation and rows."""
    out = []
    for line in lines:
        name = line.split()[0]
        kernel = re.search(r"\d+([a-z_]+)_kernelI", name).group(1)
        numbers = tuple(int(i) for i in re.findall(r"Li(\d+)E", name))
        if kernel in ("solo", "solo_join"):
            does = ("y", "dx", "dw")[int(re.search(r"DoesE(\d)E", name).group(1))]
            out.append("%s %s %d" % (kernel, does, 16 * numbers[-1]))
        else:
            out.append("%s %s" % (kernel, SHAPES[numbers]))
    return out


@pytest.mark.parametrize("size,type,forward,gradients", [
    # us by large tiles and by small ones: the product 217 and 251
    ((8192, 16, 5632, 2048), BF16, ["expert_product large"], None),
    # gradients of ragged rows 436 and 515
    ((8192, 16, 2048, 5632), BF16, ["expert_product large"], ["expert_gradients large"]),
    # 815 and 965
    ((16384, 32, 5632, 2048), BF16, ["expert_product large"], ["expert_gradients large"]),
    ((16384, 32, 5632, 2048), FP16, ["expert_product large"], ["expert_gradients large"]),
    ((8, 64, 2816, 1024), BF16, ["solo y 16"], None),
    ((1554, 13, 2730, 1000), FP16, ["expert_product eights"], None),
    # by tiles of 16 rows 43.6, of 64 81.9, of 128 132
    ((8 * 32, 8, 2048, 2048), FP32, ["solo y 16"], None),
    # 34.9, 24.6, 27.3
    ((8 * 128, 8, 2048, 2048), BF16, ["solo y 64"], None)])
def test_the_kernel_that_is_taken(fake, size, type, forward, gradients):  # noqa: F811
    _, results = run(fake, calls_of(*size, type, (BIG, BIG), False))
    assert results[0][0] == results[1][0] == 0
    assert kernels(results[0][1]) == forward
    assert gradients is None or kernels(results[1][1]) == gradients


def test_sizes_that_are_for_large_tiles(fake):  # noqa: F811
    """Those of the GPU test whose last round of large tiles goes in quarters."""
    for size in [(6165, 3, 2469, 416), (3884, 3, 3749, 496), (5424, 4, 2797, 456)]:
        for type in (FP16, BF16):
            _, results = run(fake, calls_of(*size, type, (BIG, BIG), False))
            assert kernels(results[0][1]) == ["expert_product large"]
