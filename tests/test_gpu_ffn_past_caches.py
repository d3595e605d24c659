"""Outputs of 256 MB and more, which go past the caches, are those of calls whose rows' stride keeps them in."""
import pytest
import torch

from paper_1705_01626_amd import ffn
from tests import conftest
from tests import test_gpu_ffn as blocks

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("m,n,keep", [(16384, 8192, False), (16380, 11296, False), (8192, 5632, True)])
def test_the_same_bits(m, n, keep, dtype):
    k = 64
    for name in ffn.ACTIVATIONS:
        with conftest.repeatable_inputs(blocks):
            x, wg, wu, _ = blocks.problem(m, n, k, dtype, name)
        ws, results = ffn.new_glu_workspace(x, wg, wu), []
        for pad in (0, 8):
            outs = [torch.full((m, n + pad), blocks.SENTINEL, dtype=dtype, device=DEV) for _ in range(3 if keep else 1)]
            h, gate, up = ([t[:, :n] for t in outs] + [None, None])[:3]
            ffn.zvc_glu_forward(x, wg, wu, h, ws, name, gate, up, p=0.1, seed=3)
            assert all(bool((t[:, n:] == blocks.SENTINEL).all()) for t in outs)
            results.append([t[:, :n] for t in outs])
        for a, b in zip(*results):
            assert torch.equal(a, b), name
