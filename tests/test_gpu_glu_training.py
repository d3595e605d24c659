"""The example that trains a gated block with its kept projections on the host."""
import importlib.util
import os

import pytest
import torch

from paper_1705_01626_amd import ffn
from tests import ffn_ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("glu_training", os.path.join(ROOT, "examples", "glu_training.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_loss_falls(example):
    losses = example.train(12, 1024, 256, 704, say=lambda line: None)
    assert losses[-1] < 0.9 * losses[0] and all(a == a for a in losses)


def test_gradients_are_those_of_the_same_block_without_the_detour(example):
    """Bit for bit what zvc_glu_backward gives from projections that never left."""
    block = example.Block(300, 128, 264, 0.2, seed=5)
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(300, 128, generator=gen, device="cuda").to(torch.bfloat16)
    dy = torch.randn(300, 128, generator=gen, device="cuda").to(torch.bfloat16)
    block.forward(x)
    torch.cuda.synchronize()
    gate, up = block.gate.clone(), block.up.clone()
    block.gate.fill_(7.0), block.up.fill_(7.0)
    dx, dwg, dwu, _ = (t.clone() for t in block.backward(x, dy))
    assert torch.equal(block.gate, gate) and torch.equal(block.up, up)
    dout = torch.empty_like(dy)
    ffn.zvc_dropout(dy, dout, 0.2, 5, 1)
    want = [torch.empty_like(t) for t in (dx, dwg, dwu)]
    ffn.zvc_glu_backward(dout @ block.wd, x, block.wg, block.wu, *want, block.ws, "relu", gate, up, p=0.2, seed=5, offset=0)
    assert torch.equal(dx, want[0] + dy) and torch.equal(dwg, want[1]) and torch.equal(dwu, want[2])
    # no mask was kept: the generator says which elements are gone
    assert not bool(gate[~ffn_ref.kept(300, 264, 0.2, 5, 0).to("cuda")].any())
