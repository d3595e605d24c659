"""The optimizer's step on the GPU against its definition: m, v, codes and scales to the bit, weights within their roundings."""
import math

import numpy as np
import pytest
import torch

from paper_1705_01626_amd import adamw
from tests import adamw_ref
from tests.ffn_inputs import generator
from tests.ffn_ref import ROUND
from tests.gpu_util import say

pytestmark = pytest.mark.gpu
DEV = "cuda"
HYPER = {"rate": 1e-2, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "decay": 0.1}
KINDS = [(torch.float32, torch.float32, False), (torch.float16, torch.float16, True), (torch.float16, torch.float32, False), (torch.bfloat16, torch.bfloat16, True),
         (torch.bfloat16, torch.bfloat16, False), (torch.bfloat16, torch.float32, True), (torch.float16, torch.float16, False), (torch.float16, torch.float32, True),
         (torch.bfloat16, torch.float32, False)]


def within(values, at, dtype=None):
    """The values at element `at` of memory of their own, with 16 elements of 7 on either side that no step may change."""
    dtype = dtype or values.dtype
    base = torch.full((values.numel() + at + 32,), 7.0, device=DEV).to(dtype)
    t = base[16 + at:16 + at + values.numel()]
    t.copy_(values.to(dtype))
    return t


def make(count, kind, bits, at, gen, scale=1.0):
    """(param, grad, state, master) with a past."""
    dtype, grad_dtype, master = kind
    draw = lambda n=count: torch.randn(n, generator=gen, device=DEV)
    weights = draw()
    keep = (torch.rand(count, generator=gen, device=DEV) < 0.7)
    grad = draw() * scale * keep * torch.exp(2 * draw())
    if bits == 32:
        state = (within(draw() * scale, at), within((draw() * scale).square(), at))
    else:
        blocks = -(-count // adamw.BLOCK)
        codes = lambda: torch.randint(0, 0x7F, (count,), generator=gen, device=DEV, dtype=torch.uint8)
        sign = torch.randint(0, 2, (count,), generator=gen, device=DEV, dtype=torch.uint8) * 128
        scales = lambda: torch.exp2(torch.randint(-9, -6, (blocks,), generator=gen, device=DEV).float()) * scale
        state = (within((codes() | sign).view(adamw.CODES), at, adamw.CODES), within(codes().view(adamw.CODES), at, adamw.CODES), within(scales(), at), within(scales(), at))
    return within(weights, at, dtype), within(grad, at, grad_dtype), state, within(weights, at) if master else None


def host(t):
    return None if t is None else (t.view(torch.uint8) if t.dtype == adamw.CODES else t.float()).cpu().numpy().copy()


def snapshot(tensors):
    return [(host(p), host(g), [host(s) for s in state], host(m), p.dtype) for p, g, state, m in tensors]


def check(tensors, old, step, seed, decay=None, factor=1.0, **hyper):
    h = dict(HYPER, **hyper)
    for number, ((param, grad, state, master), (p0, g0, s0, m0, dtype)) in enumerate(zip(tensors, old)):
        name = "tensor %d, %d elements" % (number, p0.size)
        narrow = len(state) == 4
        with np.errstate(all="ignore"):
            m, v = (adamw_ref.widen(s0[0], s0[2]), adamw_ref.widen(s0[1], s0[3]) ** 2) if narrow else s0
            m, v = adamw_ref.states(m, v, g0, h["beta1"], h["beta2"], factor)
            if narrow:
                random = adamw_ref.halves(p0.size, number, step, seed)
                for values, least, codes, scales in ((m, False, state[0], state[2]), (np.sqrt(v), True, state[1], state[3])):
                    want = adamw_ref.narrow(values, random, least)
                    assert np.array_equal(host(scales), want[1]), name
                    got = host(codes)
                    at = ~np.isnan(values)                               # (a NaN's sign is nobody's)
                    assert np.array_equal(got[at], want[0][at]), name
                    assert ((got[~at] & 127) == 0x7E).all()
            else:
                assert np.array_equal(host(state[0]), m, equal_nan=True) and np.array_equal(host(state[1]), v, equal_nan=True), name
            before = p0 if m0 is None else m0
            value, bound = adamw_ref.weights(before, m, v, step, h["rate"], h["beta1"], h["beta2"], h["eps"], h["decay"] if decay is None or decay[number] else 0.0)
            fine = np.isfinite(value)
            for got, kind in ((param, dtype), (master, torch.float32)):
                if got is None:
                    continue
                rel, least = ROUND[kind]
                most = bound + (rel * (np.abs(value) + bound) + least)
                got = host(got).astype(np.float64)
                large = np.abs(value) > torch.finfo(kind).max * (1 - 2.0 ** -9)          # (fp16: where it becomes an infinity)
                assert (np.abs(got - value) <= most)[fine & ~large].all(), name
                assert not np.isfinite(got[~fine]).any(), name
            if master is not None:
                assert np.array_equal(host(master.to(dtype)), host(param), equal_nan=True)
        for t in (param, grad, master, *state):                              # what lies around them
            if t is not None:
                base = t._base
                first = t.storage_offset()
                rest = torch.cat([base[:first], base[first + t.numel():]]).float()
                assert (rest == 7).all(), name


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("kind", KINDS)
def test_a_step_over_tensors_of_all_sizes(kind, bits):
    gen = generator("sizes", str(kind), bits)
    counts = [1, 7, 8, 9, 127, 128, 129, 511, 2047, 2048, 2049, 4096, 5000, 70001]
    tensors = [make(c, kind, bits, i % 3 * (1 if i % 2 else 16), gen, 10.0 ** (i % 4 - 2)) for i, c in enumerate(counts)]
    plan = adamw.new_plan(tensors)
    for step in (1, 2, 1000):
        old = snapshot(tensors)
        say("adamw %s bits=%d step=%d" % (kind, bits, step))
        adamw.zvc_adamw(plan, step=step, seed=123456789012345, **HYPER)
        check(tensors, old, step, 123456789012345)


def test_mixed_tensors_and_empty_ones():
    """Types, state widths and decay by tensor; more tensors than a wave has lanes; the second search of many."""
    gen = generator("mixed")
    tensors = [make(1 + 37 * (i % 23) if i % 11 else 0, KINDS[i % len(KINDS)], 8 if i % 3 else 32, i % 5, gen) for i in range(200)]
    decay = [i % 4 != 0 for i in range(200)]
    plan = adamw.new_plan(tensors, decay=decay)
    old = snapshot(tensors)
    adamw.zvc_adamw(plan, step=3, seed=-1, **HYPER)
    check([t for t in tensors], old, 3, (1 << 64) - 1, decay)


def test_thousands_of_tensors():
    gen = generator("thousands")
    flat = [torch.randn(5000 * 3, generator=gen, device=DEV) for _ in range(4)]
    flat[3].square_()
    tensors = [(flat[0][3 * i:3 * i + 3], flat[1][3 * i:3 * i + 3], (flat[2][3 * i:3 * i + 3], flat[3][3 * i:3 * i + 3]), None) for i in range(5000)]
    old = [t.cpu().numpy().copy() for t in flat]
    adamw.zvc_adamw(adamw.new_plan(tensors), step=4, **HYPER)
    m, v = adamw_ref.states(old[2], old[3], old[1], HYPER["beta1"], HYPER["beta2"])
    assert np.array_equal(flat[2].cpu().numpy(), m) and np.array_equal(flat[3].cpu().numpy(), v)
    value, bound = adamw_ref.weights(old[0], m, v, 4, **HYPER)
    assert (np.abs(flat[0].cpu().numpy() - value) <= bound + 2.0 ** -24 * np.abs(value)).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_from_nothing(bits):
    """The first steps of a state that new_adamw_state made, gradients that are zero among them."""
    gen = generator("nothing", bits)
    p = within(torch.randn(3000, generator=gen, device=DEV), 0)
    g = within(torch.randn(3000, generator=gen, device=DEV), 0)
    g[500:1500] = 0
    state = tuple(within(t.float() if t.dtype == adamw.CODES else t, 0, t.dtype) for t in adamw.new_adamw_state(p, bits))
    tensors = [(p, g, state, None)]
    plan = adamw.new_plan(tensors)
    for step in (1, 2, 3):
        old = snapshot(tensors)
        adamw.zvc_adamw(plan, step=step, seed=9, **HYPER)
        check(tensors, old, step, 9)
    assert not state[0][500:1500].float().any() and not state[1][500:1500].float().any()


@pytest.mark.parametrize("bits", [8, 32])
def test_extremes(bits):
    """Infinities and NaNs stay in their elements; a block of zeros, the largest and the smallest numbers."""
    gen = generator("extremes", bits)
    tensors = [make(128 * 9, KINDS[0], bits, 0, gen)]
    p, g, state, _ = tensors[0]
    g[3], g[200], g[300] = math.nan, math.inf, -math.inf
    if bits == 32:
        state[0][384:512], state[1][384:512], g[384:512] = 0, 0, 0
        state[0][512:640], state[1][512:640], g[512:640] = 1e-30, 1e-38, 1e-25
        state[0][640:768], state[1][640:768], g[640:768] = 1e18, 1e37, 1e18
        state[0][770] = math.nan
    else:
        for i in (0, 1):
            state[i][384:512] = 0
        g[384:512] = 0
        for i in (2, 3):
            state[i][4], state[i][5] = 1e-33, 1e15
        g[512:640], g[640:768] = 1e-36, 1e16
    old = snapshot(tensors)
    adamw.zvc_adamw(adamw.new_plan(tensors), step=2, seed=5, **HYPER)
    check(tensors, old, 2, 5)
    assert torch.isfinite(p[[i for i in range(128 * 9) if i not in (3, 200, 300, 770)]]).all()


def test_what_the_device_adds_and_multiplies():
    """d_step and d_factors: the same bits as a call that has the numbers themselves, also from a captured graph."""
    gen = generator("device words")
    one = [make(5000, KINDS[3], 8, 0, gen), make(300, KINDS[0], 32, 1, gen)]
    clone = lambda t: None if t is None else within(t.float() if t.dtype == adamw.CODES else t, t.storage_offset() - 16, t.dtype)
    other = [(clone(p), clone(g), tuple(clone(s) for s in state), clone(m)) for p, g, state, m in one]
    plans = adamw.new_plan(one), adamw.new_plan(other)
    d_step, d_factors = torch.tensor([5], device=DEV), torch.tensor([0.5, 0.25], device=DEV)
    adamw.zvc_adamw(plans[0], step=10, seed=3, factor=2.0, **HYPER)
    adamw.zvc_adamw(plans[1], step=5, seed=3, factor=8.0, d_step=d_step, d_factors=d_factors, **dict(HYPER, rate=2e-2))
    same = lambda: all(np.array_equal(a, b) for x, y in zip(snapshot(one), snapshot(other)) for a, b in zip([x[0], *x[2], x[3]], [y[0], *y[2], y[3]]) if a is not None)
    torch.cuda.synchronize()
    assert same()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        adamw.zvc_adamw(plans[1], step=0, seed=3, d_step=d_step, d_factors=d_factors, **HYPER)
    for step in (11, 12, 13):
        d_step.fill_(step)
        d_factors.copy_(torch.tensor([1.0 / step, 2.0]))
        graph.replay()
        rate = float(np.float32(1.0 / step)) * HYPER["rate"]
        adamw.zvc_adamw(plans[0], step=step, seed=3, factor=2.0, **dict(HYPER, rate=rate))
        torch.cuda.synchronize()
        assert same()


def test_streams_and_a_plan_that_outlives_its_tensors_names():
    gen = generator("streams")
    tensors = [make(100000, KINDS[3], 8, 0, gen)]
    plan = adamw.new_plan([tensors[0]])
    old = snapshot(tensors)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    adamw.zvc_adamw(plan, step=1, seed=1, stream=stream, **HYPER)
    stream.synchronize()
    check(tensors, old, 1, 1)
    assert plan.tensors[0][0] is tensors[0][0]


def test_a_plan_that_is_dropped_before_its_step_has_run():
    """Its memory goes to no other tensor while a step on another stream has still to read it."""
    gen = generator("dropped")
    tensors = [make(5000, KINDS[3], 8, 0, gen)]
    old = snapshot(tensors)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    plan = adamw.new_plan(tensors)
    at, size = plan.device_bytes.data_ptr(), plan.device_bytes.numel()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(200_000_000)
    adamw.zvc_adamw(plan, step=1, seed=1, stream=stream, **HYPER)
    del plan
    others = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(50)]
    assert not stream.query() and at not in [t.data_ptr() for t in others]
    stream.synchronize()
    check(tensors, old, 1, 1)


def test_a_large_tensor():
    """More elements than 2^31 bytes of them; the last ones against the definition."""
    count = (1 << 30) + 1000
    p = torch.zeros(count, dtype=torch.bfloat16, device=DEV)
    g = torch.zeros(count, dtype=torch.bfloat16, device=DEV)
    state = adamw.new_adamw_state(p, 8)
    gen = generator("large")
    g[-3000:] = torch.randn(3000, generator=gen, device=DEV).bfloat16()
    adamw.zvc_adamw(adamw.new_plan([(p, g, state, None)]), step=1, seed=77, **HYPER)
    first = count // 8 * 8 - 2000
    m, v = adamw_ref.states(np.zeros(count - first, np.float32), np.zeros(count - first, np.float32), host(g[first:]), HYPER["beta1"], HYPER["beta2"])
    start = first // 128 * 128
    pad = np.zeros(first - start, np.float32)
    index = np.arange(start // 8, -(-count // 8), dtype=np.uint64)
    words = adamw_ref.philox((index, np.zeros_like(index), np.full_like(index, 1), np.zeros_like(index)), (77, 0))
    random = np.stack([words[j // 2] >> np.uint64(16 * (j % 2)) & np.uint64(0xFFFF) for j in range(8)], 1).reshape(-1)[:count - start].astype(np.float64)
    codes, scales = adamw_ref.narrow(np.concatenate([pad, m]), random, False)
    # (the first block holds gradients from before `first` too)
    assert np.array_equal(host(state[0][start:])[128:], codes[128:]) and np.array_equal(host(state[2][start // 128:])[1:], scales[1:])
    assert not p[:count - 3000].any() and p[-3000:].any()
