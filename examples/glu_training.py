"""A gated feed-forward block trained with its kept projections away from GPU memory.

    y = x + drop(drop(relu(x Wg^T) * (x Wu^T)) Wd^T)

The forward pass keeps both projections (zero where the gate is closed or the element dropped), and each
leaves for pinned host memory as a compressed stream; before the backward pass they come back and the
gradients are computed from them.  No dropout mask is stored anywhere.  The products with Wd are plain
matrix products of torch.

    python examples/glu_training.py [--steps 20] [--tokens 4096] [--width 1024] [--inner 2816]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1705_01626_amd import ffn, zvc  # noqa: E402


class Kept:
    """A tensor of the forward pass in pinned host memory, as a compressed stream."""

    def __init__(self, like, stage, copy):
        n, w = like.numel(), like.element_size()
        self.ws, self.stage, self.copy = zvc.new_workspace(n, w, like.device), stage, copy
        self.pinned = torch.empty(zvc.zvc_max_compressed_bytes(n, w), dtype=torch.uint8, pin_memory=True)
        self.size = torch.zeros(1, dtype=torch.int64, pin_memory=True)
        self.nbytes = 0

    def leave(self, t):
        self.nbytes = zvc.zvc_offload(t, self.stage, self.pinned, self.size, self.ws, torch.cuda.current_stream(), self.copy)

    def come_back(self, out):
        zvc.zvc_prefetch(self.pinned, self.nbytes, self.stage, out, self.ws, self.copy, torch.cuda.current_stream())


class Block:
    """The block's weights and what its passes work in."""

    def __init__(self, tokens, width, inner, p, dtype=torch.bfloat16, device="cuda", seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        new = lambda *shape: torch.empty(*shape, dtype=dtype, device=device)
        weight = lambda rows, cols: (torch.randn(rows, cols, generator=gen, device=device) * cols ** -0.5).to(dtype)
        self.p, self.seed, self.step = p, seed, 0
        self.wg, self.wu, self.wd = weight(inner, width), weight(inner, width), weight(width, inner)
        self.h, self.gate, self.up = new(tokens, inner), new(tokens, inner), new(tokens, inner)
        self.dx, self.dwg, self.dwu = new(tokens, width), new(inner, width), new(inner, width)
        self.ws = ffn.new_glu_workspace(self.dx, self.wg, self.wu, backward=True)
        self.copy = torch.cuda.Stream()
        stages = [zvc.new_compressed_buffer(self.gate.numel(), self.gate.element_size(), device) for _ in range(2)]
        self.kept = [Kept(self.gate, stage, self.copy) for stage in stages]

    def forward(self, x):
        # one generator, and an offset of its own for each place and step
        self.drop = [{"p": self.p, "seed": self.seed, "offset": 2 * self.step + place} for place in (0, 1)]
        self.step += 1
        ffn.zvc_glu_forward(x, self.wg, self.wu, self.h, self.ws, "relu", self.gate, self.up, **self.drop[0])
        for kept, t in zip(self.kept, (self.gate, self.up)):
            kept.leave(t)
        out = self.h @ self.wd.t()
        y = torch.empty_like(x)
        ffn.zvc_dropout(out, y, residual=x, **self.drop[1])
        return y

    def backward(self, x, dy):
        """The gradients of x and the three weights."""
        torch.cuda.current_stream().wait_stream(self.copy)       # the streams are out, their buffers free
        self.copy.wait_stream(torch.cuda.current_stream())
        for kept, t in zip(self.kept, (self.gate, self.up)):
            kept.come_back(t)
        dout = torch.empty_like(dy)
        ffn.zvc_dropout(dy, dout, **self.drop[1])
        dwd, dh = dout.t() @ self.h, dout @ self.wd
        ffn.zvc_glu_backward(dh, x, self.wg, self.wu, self.dx, self.dwg, self.dwu, self.ws, "relu", self.gate, self.up,
                             **self.drop[0])
        return self.dx + dy, self.dwg, self.dwu, dwd


def train(steps, tokens, width, inner, p=0.1, rate=0.3, say=print):
    """Fits the block to a fixed linear map of its input; the losses."""
    block = Block(tokens, width, inner, p)
    gen = torch.Generator(device="cuda").manual_seed(1)
    target = (torch.randn(width, width, generator=gen, device="cuda") * width ** -0.5).to(torch.bfloat16)
    masters = [w.float() for w in (block.wg, block.wu, block.wd)]
    losses = []
    for step in range(steps):
        x = torch.randn(tokens, width, generator=gen, device="cuda").to(torch.bfloat16)
        y = block.forward(x)
        error = y.float() - (x @ target.t()).float()
        losses.append(float(error.square().mean()))
        grads = block.backward(x, (error * (2.0 / width)).to(torch.bfloat16))
        for master, w, g in zip(masters, (block.wg, block.wu, block.wd), grads[1:]):
            master -= rate / tokens * width ** 0.5 * g.float()
            w.copy_(master)
        raw = sum(t.numel() * t.element_size() for t in (block.gate, block.up))
        say("step %2d  loss %.4f  kept projections %.1f MB, %.2f of their size on the host" % (
            step, losses[-1], raw / 1e6, sum(k.nbytes for k in block.kept) / raw))
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    for name, value in (("steps", 20), ("tokens", 4096), ("width", 1024), ("inner", 2816)):
        parser.add_argument("--" + name, type=int, default=value)
    a = parser.parse_args()
    train(a.steps, a.tokens, a.width, a.inner)
