"""A mixture of experts trained with its hidden activations away from GPU memory and its optimizer's states in 8 bits.

    y = x + sum over a token's experts e of  weight_e relu(x W1_e^T) W2_e^T

A router gives each token two experts; their rows lie one expert behind the other, and the products go by the
router's offsets without the host ever knowing them.  The hidden activations, sparse by their ReLU, leave for pinned host
memory as a compressed stream and come back for the backward pass.  The step updates all weights in one launch, their masters
in 32 bits.  Gathering rows, the ReLU, the weighted sum and the router's own product are plain torch.

    python examples/moe_training.py [--steps 20] [--tokens 2048] [--width 512] [--inner 1024] [--experts 16]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.glu_training import Kept  # noqa: E402
from paper_1705_01626_amd import adamw, experts, zvc  # noqa: E402


class Mixture:
    """The weights, what the passes work in, and the optimizer's plan."""

    def __init__(self, tokens, width, inner, count, top=2, dtype=torch.bfloat16, device="cuda", seed=0, bits=8):
        gen = torch.Generator(device=device).manual_seed(seed)
        new = lambda *shape, dtype=dtype: torch.empty(*shape, dtype=dtype, device=device)
        weight = lambda *shape: torch.randn(*shape, generator=gen, device=device) * shape[-1] ** -0.5
        self.top, self.masters = top, [weight(count, inner, width), weight(count, width, inner), weight(count, width)]
        self.w1, self.w2, self.router = self.weights = [w.to(dtype) for w in self.masters]
        self.grads = self.dw1, self.dw2, self.drouter = [torch.empty_like(w) for w in self.weights]
        rows = tokens * top
        self.logits, self.dlogits = new(tokens, count, dtype=torch.float32), new(tokens, count, dtype=torch.float32)
        self.chosen, self.place = new(tokens, top, dtype=torch.int32), new(tokens, top, dtype=torch.int64)
        self.shares, self.offsets, self.order = new(tokens, top, dtype=torch.float32), new(count + 1, dtype=torch.int64), new(rows, dtype=torch.int64)
        # (rows of no expert stay as they are: zeros)
        self.hidden, self.out = torch.zeros_like(new(rows, inner)), torch.zeros_like(new(rows, width))
        self.dhidden, self.drows = torch.zeros_like(self.hidden), torch.zeros_like(self.out)
        self.route_ws = experts.new_route_workspace(self.logits, top)
        self.ws = [experts.new_expert_workspace(self.out, self.w1, backward=True), experts.new_expert_workspace(self.hidden, self.w2, backward=True)]
        self.copy = torch.cuda.Stream()
        self.kept = Kept(self.hidden, zvc.new_compressed_buffer(self.hidden.numel(), self.hidden.element_size(), device), self.copy)
        states = [adamw.new_adamw_state(w, bits) for w in self.weights]
        self.plan = adamw.new_plan(list(zip(self.weights, self.grads, states, self.masters)), decay=[True, True, False])
        self.step = 0

    def forward(self, x):
        self.logits.copy_(x.float() @ self.router.float().t())
        experts.zvc_route(self.logits, self.chosen, self.shares, self.offsets, self.order, self.place, self.route_ws)
        self.rows = x[self.order // self.top]
        experts.zvc_expert_product(self.rows, self.w1, self.offsets, self.hidden, self.ws[0])
        self.hidden.clamp_(min=0)
        self.kept.leave(self.hidden)
        experts.zvc_expert_product(self.hidden, self.w2, self.offsets, self.out, self.ws[1])
        # (an entry without a row has place -1: what lies in the last row is another token's, and of another step)
        self.there = (self.place >= 0)[..., None]
        self.picked = torch.where(self.there, self.out[self.place].float(), 0.0)     # tokens x top x width
        return x + (self.picked * self.shares[..., None]).sum(1).to(x.dtype)

    def backward(self, x, dy):
        """The gradient of x; those of the weights in self.grads."""
        torch.cuda.current_stream().wait_stream(self.copy)           # the stream is out, its buffer free
        self.copy.wait_stream(torch.cuda.current_stream())
        self.kept.come_back(self.hidden)
        dshares = (self.picked * dy.float()[:, None]).sum(2)
        dout = (dy.float()[:, None] * self.shares[..., None]).to(dy.dtype).flatten(0, 1)[self.order]
        experts.zvc_expert_gradients(dout, self.hidden, self.w2, self.offsets, self.dhidden, self.dw2, self.ws[1])
        self.dhidden.mul_(self.hidden > 0)
        experts.zvc_expert_gradients(self.dhidden, self.rows, self.w1, self.offsets, self.drows, self.dw1, self.ws[0])
        experts.zvc_route_backward(dshares, self.logits, self.chosen, self.dlogits)
        self.drouter.copy_(self.dlogits.t() @ x.float())
        drows = torch.where(self.there, self.drows[self.place].float(), 0.0)
        return (dy.float() + drows.sum(1) + self.dlogits @ self.router.float()).to(x.dtype)

    def update(self, rate):
        self.step += 1
        adamw.zvc_adamw(self.plan, rate, self.step, beta2=0.99, decay=0.01, seed=1)


def train(steps, tokens, width, inner, count, rate=2e-3, say=print):
    """Fits the mixture to a fixed map of its input; the losses."""
    block = Mixture(tokens, width, inner, count)
    gen = torch.Generator(device="cuda").manual_seed(1)
    target = (torch.randn(width, width, generator=gen, device="cuda") * width ** -0.5).to(torch.bfloat16)
    losses = []
    for step in range(steps):
        x = torch.randn(tokens, width, generator=gen, device="cuda").to(torch.bfloat16)
        y = block.forward(x)
        error = y.float() - (x @ target.t()).float()
        losses.append(float(error.square().mean()))
        block.backward(x, (error * (2.0 / error.numel())).to(torch.bfloat16))
        block.update(rate)
        raw = block.hidden.numel() * block.hidden.element_size()
        say("step %2d  loss %.4f  hidden activations %.1f MB, %.2f of their size on the host" % (step, losses[-1], raw / 1e6, block.kept.nbytes / raw))
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser()
    for name, value in (("steps", 20), ("tokens", 2048), ("width", 512), ("inner", 1024), ("experts", 16)):
        parser.add_argument("--" + name, type=int, default=value)
    a = parser.parse_args()
    train(a.steps, a.tokens, a.width, a.inner, a.experts)
