"""Router, experts' products, codec and optimizer together, as the example trains with them."""
import importlib.util
import os

import pytest
import torch

from paper_1705_01626_amd import adamw, experts
from tests.ffn_inputs import generator

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("moe_training", os.path.join(ROOT, "examples", "moe_training.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_runs(example):
    lines = []
    losses = example.train(4, 512, 128, 256, 8, say=lines.append)
    assert len(lines) == 4 and all(v == v and v < 1e6 for v in losses)


def test_gradients_against_autograd(example):
    """In 64 bits, with the experts that the router gave.

    Every rounding to bf16 between the products is at most 2^-8 of a number, at random about 2^-9.3 of a norm; the longest chain has five (hidden, dout, dhidden, drows, the
    sum), and the router's gradient is a difference of two dot products of rounded numbers.  2^-5 is above five times 2^-8 and that difference."""
    tokens, width, inner, count = 700, 136, 264, 6
    block = example.Mixture(tokens, width, inner, count, seed=3)
    gen = generator("moe")
    x = torch.randn(tokens, width, generator=gen, device="cuda").bfloat16()
    dy = torch.randn(tokens, width, generator=gen, device="cuda").bfloat16()
    y = block.forward(x)
    hidden = block.hidden.clone()
    block.hidden.fill_(7)
    dx = block.backward(x, dy)
    assert torch.equal(block.hidden, hidden)                         # what came back is what left
    leaves = [t.double().requires_grad_() for t in (x, block.w1, block.w2, block.router)]
    px, w1, w2, router = leaves
    logits = px @ router.t()
    chosen = block.chosen.long()
    shares = torch.softmax(logits.gather(1, chosen), 1)
    out = torch.zeros(tokens, width, dtype=torch.float64, device="cuda")
    for e in range(count):
        at = chosen == e
        rows = at.any(1)
        out[rows] = out[rows] + (shares * at).sum(1)[rows][:, None] * (torch.relu(px[rows] @ w1[e].t()) @ w2[e].t())
    want = px + out
    want.backward(dy.double())
    for got, exact in ((y, want), (dx, px.grad), (block.dw1, w1.grad), (block.dw2, w2.grad), (block.drouter, router.grad)):
        error = float((got.double() - exact.detach()).norm() / exact.detach().norm())
        assert error < 2.0 ** -5, error
    before = [w.clone() for w in block.masters]
    block.update(1e-2)
    for old, master, w in zip(before, block.masters, block.weights):
        assert torch.equal(master.to(w.dtype), w) and not torch.equal(old, master)
        assert float((old - master).abs().max()) < 1.1e-2 + 1e-4 * float(old.abs().max())      # the first step: rate times a sign, and decay


def test_a_step_of_padded_tokens_from_a_graph():
    """Router, products, gradients and AdamW in one captured graph; each replay has other tokens, some of them padding, and is compared with
    the same calls made one by one."""
    tokens, width, inner, count, top = 300, 64, 96, 5, 2
    gen = generator("padded")
    new = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device="cuda")
    logits, dshares = new(tokens, count, dtype=torch.float32), new(tokens, top, dtype=torch.float32)
    dout, x = new(tokens * top, inner), new(tokens, width)
    step = torch.ones(1, dtype=torch.int64, device="cuda")
    w = torch.randn(count, inner, width, generator=gen, device="cuda").bfloat16()

    class Side:
        def __init__(self):
            self.route = [new(tokens, top, dtype=torch.int32), new(tokens, top, dtype=torch.float32), new(count + 1, dtype=torch.int64),
                          new(tokens * top, dtype=torch.int64), new(tokens, top, dtype=torch.int64)]
            self.w, self.dw, self.y, self.drows, self.dlogits = w.clone(), new(count, inner, width), new(tokens * top, inner), new(tokens * top, width), new(tokens, count, dtype=torch.float32)
            self.state = adamw.new_adamw_state(w, 8)
            self.plan = adamw.new_plan([(self.w, self.dw, self.state, None)])
            self.rows = new(tokens * top, width)
            self.route_ws, self.ws = experts.new_route_workspace(logits, top), experts.new_expert_workspace(self.rows, w, backward=True)

        def run(self):
            experts.zvc_route(logits, *self.route, self.route_ws)
            torch.index_select(x, 0, (self.route[3] // top).clamp(min=0), out=self.rows)
            experts.zvc_expert_product(self.rows, self.w, self.route[2], self.y, self.ws)
            experts.zvc_expert_gradients(dout, self.rows, self.w, self.route[2], self.drows, self.dw, self.ws)
            experts.zvc_route_backward(dshares, logits, self.route[0], self.dlogits)
            adamw.zvc_adamw(self.plan, 1e-2, 0, d_step=step, seed=4)

        def results(self):
            return [*self.route, self.w, self.dw, self.y, self.drows, self.dlogits, self.state[0].view(torch.uint8), self.state[1].view(torch.uint8), *self.state[2:]]

    one, other = Side(), Side()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        (one.route[3] // top).clamp(min=0)                           # (what torch sets up at its first use)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.run()
    for turn in range(4):
        logits.copy_(torch.randn(tokens, count, generator=gen, device="cuda"))
        logits[torch.rand(tokens, generator=gen, device="cuda") < 0.3 * turn] = -float("inf")
        x.copy_(torch.randn(tokens, width, generator=gen, device="cuda"))
        dout.copy_(torch.randn(tokens * top, inner, generator=gen, device="cuda"))
        dshares.copy_(torch.randn(tokens, top, generator=gen, device="cuda"))
        step.fill_(turn + 1)
        graph.replay()
        other.run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(one.results(), other.results()))
        rows = int(one.route[2][-1])
        assert (one.route[3][rows:] == -1).all() and int((one.route[0] >= 0).sum()) == rows


def test_tokens_without_experts(example, monkeypatch):
    """They pass as they are in both directions, and what other tokens left in rows that are no expert's now reaches neither them nor any weight."""
    tokens, width, inner, count = 300, 72, 136, 5
    block = example.Mixture(tokens, width, inner, count, seed=5)
    gen = generator("without")
    draw = lambda: torch.randn(tokens, width, generator=gen, device="cuda").bfloat16()
    x, dy = draw(), draw()
    block.forward(x)
    block.backward(x, dy)
    away = torch.rand(tokens, generator=gen, device="cuda") < 0.4
    plain = example.experts.zvc_route

    def masked(logits, *args):
        logits[away] = -float("inf")
        plain(logits, *args)

    monkeypatch.setattr(example.experts, "zvc_route", masked)
    for stale in (None, float("nan")):
        x, dy = draw(), draw()
        rows = int((~away).sum()) * block.top
        if stale is not None:
            block.out[rows:], block.drows[rows:] = stale, stale
        y = block.forward(x)
        dx = block.backward(x, dy)
        assert int(block.offsets[-1]) == rows and (block.place[away] == -1).all()
        assert torch.equal(y[away], x[away]) and torch.equal(dx[away], dy[away])
        for t in (y, dx, *block.grads):
            assert torch.isfinite(t).all()
        assert not torch.equal(dx[~away], dy[~away]) and not torch.equal(y[~away], x[~away])


def test_the_first_step_goes_against_the_gradient(example):
    """m / (1 - beta1) is then the gradient and sqrt(v / (1 - beta2)) its size.  Weights lie below 8, where half a unit of 32 bits is 2^-22: three roundings of
    them and some ten of a change of 1e-2 are below 2^-20."""
    block = example.Mixture(256, 64, 128, 4, seed=9)
    gen = generator("against")
    x, dy = (torch.randn(256, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
    block.forward(x)
    block.backward(x, dy)
    before = [w.double() for w in block.masters]
    block.update(1e-2)
    for old, grad, new, decay in zip(before, block.grads, block.masters, (0.01, 0.01, 0.0)):
        g = grad.double()
        want = (1 - 1e-2 * decay) * old - 1e-2 * g / (g.abs() + 1e-8)
        assert float(old.abs().max()) < 8 and grad.any()
        assert float((new.double() - want).abs().max()) < 2.0 ** -20
