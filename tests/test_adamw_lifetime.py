"""Who keeps a step's memory until the step has run: a plan may be its tensors' only owner, and it may be dropped as soon as the call has
returned, whatever stream the step is on."""
import types

import pytest
import torch

from paper_1705_01626_amd import adamw
from tests.ffn_inputs import generator

HYPER = {"rate": 1e-2, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "decay": 0.1}


class Recorder:
    """Stands in for a tensor and writes down the streams that the allocator is told of."""

    def __init__(self):
        self.device, self.streams = torch.device("cuda", 0), []

    def data_ptr(self):
        return 1 << 40

    def record_stream(self, stream):
        self.streams.append(stream.cuda_stream)


def test_the_allocator_is_told_of_every_stream(monkeypatch):
    """Of all that a step reads or writes, once for each stream; the first is no exception, since a plan may be made on another stream than its tensors."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *device: types.SimpleNamespace(cuda_stream=0))
    monkeypatch.setattr(adamw, "_stream_handle", lambda stream: 0 if stream is None else stream.cuda_stream)
    monkeypatch.setattr(adamw, "_native", lambda: types.SimpleNamespace(zvc_adamw=lambda *args: 0))
    new = Recorder
    tensors = [(new(), new(), (new(), new()), None), (new(), new(), (new(), new(), new(), new()), new())]
    plan = adamw.Plan(tensors, new(), new())
    for stream in (None, 7, 7, None, 9, 7):
        adamw.zvc_adamw(plan, step=1, stream=None if stream is None else types.SimpleNamespace(cuda_stream=stream), **HYPER)
    for param, grad, state, master in tensors:
        for t in (param, grad, *state, *([] if master is None else [master]), plan.device_bytes):
            assert t.streams == [0, 7, 9]


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_what_a_dropped_plan_owned_is_not_given_away(bits):
    """The states are the plan's alone; no tensor gets their memory while a step on another stream has still to write it."""
    gen = generator("owner", bits)
    count = 300000
    weights = torch.randn(count, generator=gen, device="cuda")
    param, master, grad = weights.bfloat16(), weights.clone(), torch.randn(count, generator=gen, device="cuda").bfloat16()
    plan = adamw.new_plan([(param, grad, adamw.new_adamw_state(param, bits), master)])
    owned = [(t.data_ptr(), t.numel() * t.element_size()) for t in (*plan.tensors[0][2], plan.device_bytes)]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(200_000_000)
    adamw.zvc_adamw(plan, step=1, seed=1, stream=stream, **HYPER)
    del plan
    others = [torch.empty(size, dtype=torch.uint8, device="cuda") for _, size in owned for _ in range(20)]
    assert not stream.query()
    for t in others:
        for at, size in owned:
            assert t.data_ptr() + t.numel() <= at or at + size <= t.data_ptr()
    stream.synchronize()
    # the first step: m / (1 - beta1) is g and sqrt(v / (1 - beta2)) its size.  Weights lie below 8, where half a unit of 32 bits is 2^-22: three
    # roundings of them (shrinking, its factor, the difference), and some ten of a change of 1e-2, 2^-27 together, are below 2^-20.
    g = grad.double()
    want = 0.999 * weights.double() - 1e-2 * g / (g.abs() + 1e-8)
    assert float(weights.abs().max()) < 8
    assert float((master.double() - want).abs().max()) < 2.0 ** -20 and torch.equal(master.bfloat16(), param)
