"""The gated block on the GPU at the sizes of ffn_routes, which launch every kind of tile and cut, against its formulas in 64 bits
(test_gpu_ffn's check and bounds)."""
import functools
import itertools

import pytest
import torch

from paper_1705_01626_amd import ffn
from tests import conftest, ffn_ref
from tests import test_gpu_ffn as blocks
from tests.ffn_routes import ROUTES

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
ACTS = list(ffn.ACTIVATIONS)


@pytest.fixture(autouse=True, scope="module")
def inputs():
    with conftest.repeatable_inputs(blocks), pytest.MonkeyPatch.context() as patch:
        patch.setattr(ffn_ref, "kept", functools.lru_cache(maxsize=8)(ffn_ref.kept))      # (seconds for the larger sizes)
        yield


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", list(ROUTES), ids=lambda size: "%dx%dx%d" % size)
def test_every_route(size, dtype):
    """Kept projections and computed again, with dropout and without; each size with two activations."""
    turn = list(ROUTES).index(size) + DTYPES.index(dtype)
    blocks.check_block(*size, dtype, ACTS[turn % 4], False, {"p": 0.0})
    blocks.check_block(*size, dtype, ACTS[(turn + 2) % 4], True, {"p": 0.1, "seed": turn, "offset": 5})
    if turn % 2:
        blocks.check_block(*size, dtype, ACTS[(turn + 1) % 4], False, {"p": 0.3, "seed": turn})
    else:
        blocks.check_block(*size, dtype, ACTS[(turn + 3) % 4], True, {"p": 0.0})


# a size for each shape of tile with ends inside a strip, a tile and eight columns, and one without any
SHAPES = {"half": (200, 331, 136), "lone": (517, 2051, 136), "eights": (4099, 2053, 72), "thin": (66, 8283, 88),
          "large": (3001, 2051, 136), "large whole tiles": (1024, 8192, 128)}


@pytest.mark.parametrize("keep,p", [(False, 0.0), (True, 0.0), (False, 0.25), (True, 0.1)])
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("shape", list(SHAPES))
def test_what_becomes_of_every_shape_of_tile(shape, name, keep, p):
    """Forward, and dg and du behind projections computed again (the gradients are sums over all of them)."""
    for dtype in DTYPES:
        blocks.check_block(*SHAPES[shape], dtype, name, keep, {"p": p, "seed": 2, "offset": 1 << 35})


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 1)])
@pytest.mark.parametrize("shape", ["half", "lone", "eights", "large"])
def test_strides_and_alignment_of_every_shape_of_tile(shape, pad, shift):
    for dtype in DTYPES:
        blocks.check_block(*SHAPES[shape], dtype, "gelu_tanh", True, {"p": 0.2, "seed": 4}, pad, shift)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(389, 8608, 16), (1040, 599, 1024), (777, 2730, 200), (512, 2056, 264), (152, 2816, 584)])
def test_projections_are_exact_on_a_grid(size, dtype):
    """Sums of grid numbers have no rounding, so the kept projections are the rounded true ones in every tile."""
    x, wg, wu, _ = blocks.problem(*size, dtype, "relu")
    _, gate, up = blocks.forward(x, wg, wu, "relu", True)
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    assert torch.equal(gate, g.clamp(min=0).to(dtype)) and torch.equal(up, torch.where(g > 0, u, 0.0).to(dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("size", [(405, 783, 7832), (1176, 6656, 976), (3370, 951, 1056), (133, 351, 8200)])
def test_gradients_that_go_ahead_repeat_bit_for_bit_and_alone(size, dtype):
    """The same bits again, and when only some of them are asked for."""
    assert ROUTES[size][1].endswith("ahead")
    x, wg, wu, dh = blocks.problem(*size, dtype, "silu")
    want = blocks.backward(dh, x, wg, wu, "silu", p=0.1, seed=2)
    ws = ffn.new_glu_workspace(x, wg, wu, backward=True)
    outs = [torch.empty_like(t) for t in (x, wg, wu)]
    for first, second in itertools.product((True, False), repeat=2):
        for t in outs:
            t.fill_(blocks.SENTINEL)
        ffn.zvc_glu_backward(dh, x, wg, wu, outs[0] if first else None, outs[1] if second else None, outs[2] if second else None,
                             ws, "silu", p=0.1, seed=2)
        for t, w, there in zip(outs, want, (first, second, second)):
            assert torch.equal(t, w) if there else bool((t == blocks.SENTINEL).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", [(3001, 2051, 264), (512, 2056, 264), (4096, 2056, 72), (152, 2816, 584)])
def test_what_is_no_number_stays_in_its_row(size, dtype):
    m, n, k = size
    x, wg, wu, dh = blocks.problem(m, n, k, dtype, "gelu")
    clean = blocks.forward(x, wg, wu, "gelu", True, p=0.2, seed=7)
    x[m - 2, k - 1] = float("nan")
    x[3, 0] = float("inf")
    rows = torch.ones(m, dtype=torch.bool, device=x.device)
    rows[m - 2] = rows[3] = False
    stays = ffn_ref.kept(m, n, 0.2, 7, 0).to(x.device)
    for got, want in zip(blocks.forward(x, wg, wu, "gelu", True, p=0.2, seed=7), clean):
        assert torch.equal(got[rows], want[rows])
        assert bool(torch.isnan(got[m - 2][stays[m - 2]]).all()) and not bool(got[~stays].any())
