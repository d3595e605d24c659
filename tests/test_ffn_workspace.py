"""The gated block's workspace: what zvc_glu_workspace_bytes asks for is enough, is used and no more (no GPU; launches are written
down by a stand-in for the HIP runtime)."""
import re

import pytest

from paper_1705_01626_amd import ffn, zvc
from tests import test_ffn_launches as launches
from tests.ffn_routes import ROUTES
from tests.test_ffn_launches import BF16, FP16, FP32, fake  # noqa: F401 (a fixture)

TORCH = {code: dtype for dtype, code in ffn.TYPES.items()}
TYPES = (BF16, FP16, FP32)


def room(m, n, k, dtype, back=False):
    return ffn.zvc_glu_workspace_bytes(m, n, k, TORCH[dtype], back)


def tile_bytes(name):
    """Of one tile's sums."""
    wp, wq, pb, qb, _ = (int(i) for i in re.findall(r"Li(\d+)E", re.search(r"5ShapeI((?:Li\d+E)+)", name).group(1)))
    return 4 * wp * pb * 16 * wq * qb * 16


@pytest.mark.parametrize("m,n,k", [(1, 11264, 4096), (5, 2816, 1024), (48, 11264, 4096), (64, 4096, 4096)])
def test_few_tokens_need_no_sums(m, n, k):
    """Their kernel joins its sums on the compute unit."""
    for dtype in TYPES:
        assert room(m, n, k, dtype) <= 256


def test_sums_lie_in_the_workspace(fake):  # noqa: F811
    """With just the bytes that are asked for the calls are taken, and every part's sums lie inside; with a byte less they are refused."""
    sizes = [(m, n, k) for m, n, k in ROUTES if k % 8 == 0] + [(1, 11264, 4096), (64, 4096, 4096), (300, 4096, 4096)]
    calls, rooms = [], []
    for size in sizes:
        for dtype in TYPES:
            for make, back in ((launches.forward, False), (launches.backward, True)):
                rooms.append(room(*size, dtype, back))
                calls += [make(*size, dtype, room=rooms[-1]), make(*size, dtype, room=rooms[-1] - 1)]
    _, results = launches.run(fake, calls)
    ws, used = launches.AT[9], 0
    for i, bytes_there in enumerate(rooms):
        assert results[2 * i + 1] == (zvc.ZVC_E_WORKSPACE, [])
        status, made = results[2 * i]
        assert status == zvc.ZVC_OK
        for launch in made:
            for which in ("p", "dx", "dw"):
                v = launch.values
                if v.get(which + "_parts", 1) > 1:
                    sums = (v[which + "_tiles"] - v[which + "_whole"]) * v[which + "_parts"] * tile_bytes(launch.name)
                    assert ws <= v[which + "_sums"] and v[which + "_sums"] + sums <= ws + bytes_there
                    used += 1
    assert used > 100
