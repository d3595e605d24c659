"""The router and the experts' products on the GPU against their formulas in 64 bits."""
import math

import pytest
import torch

from paper_1705_01626_amd import experts, zvc
from tests import experts_ref
from tests.experts_sizes import SIZES
from tests.ffn_inputs import generator
from tests.gpu_util import say

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.float32, torch.float16, torch.bfloat16]
NAN = math.nan


# ---- the router -------------------------------------------------------------------
def route(logits, top, normalize, ws=None, stream=None):
    m, e = logits.shape
    out = [torch.full((m, top), 77, dtype=torch.int32, device=DEV), torch.full((m, top), NAN, device=DEV), torch.full((e + 1,), 77, dtype=torch.int64, device=DEV),
           torch.full((m * top,), 77, dtype=torch.int64, device=DEV), torch.full((m, top), 77, dtype=torch.int64, device=DEV)]
    experts.zvc_route(logits, *out, ws if ws is not None else experts.new_route_workspace(logits, top), normalize=normalize, stream=stream)
    return out


def check_route(logits, top, normalize, got):
    chosen, weights, offsets, order, place = experts_ref.route(logits.cpu(), top, normalize)
    assert got[0].tolist() == chosen and got[2].tolist() == offsets and got[3].tolist() == order
    assert got[4].view(-1).tolist() == place
    want = torch.tensor(weights, dtype=torch.float64).view(len(weights), top)
    assert ((got[1].cpu().double() - want).abs() <= want * experts_ref.EXP + experts_ref.LEAST).all()


def draw_logits(m, e, dtype, pad=0, masked=0.0, spread=1.0):
    gen = generator("logits", m, e, str(dtype), pad, masked)
    t = torch.randn(m, e + pad, generator=gen, device=DEV) * spread
    if masked:
        t.masked_fill_(torch.rand(m, e + pad, generator=gen, device=DEV) < masked, -math.inf)
        t[:, e // 2].masked_fill_(torch.rand(m, generator=gen, device=DEV) < 0.3, NAN)
        t[torch.rand(m, generator=gen, device=DEV) < 0.2] = -math.inf
    return t.to(dtype)[:, :e]


@pytest.mark.parametrize("m", [1, 3, 31, 32, 33, 700])
@pytest.mark.parametrize("e,top", [(1, 1), (2, 2), (7, 3), (16, 16), (64, 8), (65, 2), (128, 4), (129, 5), (255, 8), (300, 1), (513, 16), (1024, 16)])
def test_route(m, e, top):
    dtype = DTYPES[(m + e) % 3]
    for normalize, masked, pad in ((True, 0.0, 0), (False, 0.4, 3), (True, 0.9, 1)):
        say("route m=%d e=%d top=%d %s %s %s" % (m, e, top, dtype, normalize, masked))
        logits = draw_logits(m, e, dtype, pad, masked, spread=4.0)
        check_route(logits, top, normalize, route(logits, top, normalize))


@pytest.mark.parametrize("dtype", DTYPES)
def test_route_ties_and_extremes(dtype):
    """Equal logits by rising number, across the lanes' borders; the type's lowest value is a logit like others, minus infinity is none."""
    low = torch.finfo(dtype).min
    rows = [[0.0] * 100, [low] * 100, [-math.inf] * 99 + [low], [NAN] * 100, [-math.inf] * 100, [float(i % 5) for i in range(100)],
            [NAN if i % 2 else -0.0 for i in range(100)], [0.0 if i % 3 else -0.0 for i in range(100)], [30.0 - i for i in range(100)], [float(i) for i in range(100)],
            [torch.finfo(dtype).max] * 3 + [low] * 97, [-80.0] * 50 + [0.0] + [-85.0] * 49]
    logits = torch.tensor(rows, dtype=torch.float32).clamp(min=-math.inf, max=torch.finfo(dtype).max).to(dtype).to(DEV)
    for top in (1, 7, 16):
        for normalize in (True, False):
            check_route(logits, top, normalize, route(logits, top, normalize))


def test_route_of_an_infinity():
    """NaNs as the formula gives, and the choice is made all the same."""
    logits = torch.zeros(2, 10, device=DEV)
    logits[0, 4] = math.inf
    for normalize in (True, False):
        got = route(logits, 2, normalize)
        assert got[0].tolist() == [[4, 0], [0, 1]] and got[1][0].isnan().all() and not got[1][1].isnan().any()


def test_route_of_no_tokens():
    got = route(torch.zeros(0, 5, device=DEV), 2, True)
    assert got[2].tolist() == [0] * 6


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,e,top", [(1, 1, 1), (5, 3, 2), (16, 64, 8), (17, 130, 4), (100, 257, 16), (40, 1024, 6)])
def test_route_backward(dtype, m, e, top):
    for normalize, masked, pad in ((True, 0.0, 0), (False, 0.0, 3), (True, 0.5, 1), (False, 0.5, 0)):
        say("route_backward m=%d e=%d top=%d %s" % (m, e, top, dtype))
        logits = draw_logits(m, e, dtype, pad, masked, spread=3.0)
        chosen = torch.tensor(experts_ref.choose(logits.cpu(), top), dtype=torch.int32)
        if top > 2 and m > 2:                    # an expert twice, and numbers that are no expert's
            chosen[1, 1] = chosen[1, 0]
            chosen[2, 0], chosen[2, 1] = e, -5
        dw = torch.randn(m, top, generator=generator("dw", m, e, top), device=DEV)
        out = torch.full((m, e + pad), 77.0, dtype=dtype, device=DEV)
        experts.zvc_route_backward(dw, logits, chosen.to(DEV), out[:, :e], normalize=normalize)
        value, bound = experts_ref.route_backward(dw.cpu(), logits.cpu(), chosen.tolist(), normalize)
        assert ((out[:, :e].cpu().double() - value).abs() <= bound).all()
        assert (out[:, e:] == 77).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("e", [5, 16, 130, 1024])
def test_route_backward_of_what_is_not_finite(dtype, e):
    """An expert that is out gets 0 whatever the others' gradients are, and an infinity or a NaN stays in its token."""
    gen = generator("not finite", e, str(dtype))
    m, top = 12, 2
    logits = torch.randn(m, e, generator=gen, device=DEV).to(dtype)
    out = torch.rand(m, e, generator=gen, device=DEV) < 0.4
    out[:, :3], out[:, 3] = False, True
    logits[out] = -math.inf
    logits[:, 3] = NAN
    chosen = torch.tensor([[1, 0]] * m, dtype=torch.int32, device=DEV)
    dw = torch.randn(m, top, generator=gen, device=DEV)
    dw[1, 0], dw[3, 1], dw[5, 0] = math.inf, -math.inf, NAN
    logits[7, 2] = math.inf                       # (not a chosen one: a softmax over all is NaN)
    for normalize in (True, False):
        got = torch.full((m, e), 77.0, dtype=dtype, device=DEV)
        experts.zvc_route_backward(dw, logits, chosen, got, normalize=normalize)
        assert (got[out] == 0).all()
        odd = [1, 3, 5] if normalize else [1, 3, 5, 7]
        fine = [t for t in range(m) if t not in odd]
        assert torch.isfinite(got[fine]).all() and (got[fine][:, :2] != 0).all()
        assert not torch.isfinite(got[odd][:, :2]).any()
        if not normalize:
            assert not torch.isfinite(got[[1, 3, 5]][:, 2]).any() and got[7].isnan().logical_or(out[7]).all()


# ---- the products -----------------------------------------------------------------
def offsets_of(m, experts_, how, gen):
    """Where the experts' rows begin: dealt unevenly, all to one, evenly, with rows of no expert at both ends, or out of order."""
    if how == "one":
        at = [0] * (experts_ // 2 + 1) + [m] * (experts_ - experts_ // 2)
    elif how == "even":
        at = [m * e // experts_ for e in range(experts_ + 1)]
    elif how == "wild":
        at = (torch.randint(-m // 4 - 1, m + m // 4 + 2, (experts_ + 1,), generator=gen, device=DEV)).tolist()
        at[0], at[-1] = min(at[0], m // 3), (1 << 62 if experts_ % 2 else -(1 << 62))
    else:
        at = sorted(torch.randint(0, m + 1, (experts_ + 1,), generator=gen, device=DEV).tolist())
        if how == "all":
            at[0], at[-1] = 0, m
    return at


def draw(rows, cols, dtype, gen, std=1.0, ld=None, at=0, fill=NAN):
    """rows x cols normal draws within `fill`, at element `at` of their memory."""
    ld = ld or cols
    base = torch.full((at + rows * ld + 16,), fill, dtype=dtype, device=DEV)
    t = base[at:at + rows * ld].view(rows, ld)[:, :cols]
    t.copy_(torch.randn(rows, cols, generator=gen, device=DEV) * std)
    return t


def stack(experts_, n, k, dtype, gen, std, ld, at=0, extra=0, fill=NAN):
    base = torch.full((at + experts_ * (n * ld + extra) + 16,), fill, dtype=dtype, device=DEV)
    w = base.as_strided((experts_, n, k), (n * ld + extra, ld, 1), at)
    for e in range(experts_):
        w[e] = torch.randn(n, k, generator=gen, device=DEV) * std
    return w


def run_products(m, experts_, n, k, dtype, how, loose, part="both"):
    """Both calls on operands within NaNs; nothing beside the rows that the header names may change."""
    gen = generator("products", m, experts_, n, k, str(dtype), how, loose)
    up = lambda x: x if loose else (x + 7) // 8 * 8
    at = 1 if loose == 2 else 0
    x = draw(m, k, dtype, gen, 1.0, up(k) + (0 if loose else 8), at)
    dy = draw(m, n, dtype, gen, 1.0, up(n), at)
    w = stack(experts_, n, k, dtype, gen, max(k, 1) ** -0.5, up(k), at, 0 if loose else 64)
    offsets = offsets_of(m, experts_, how, gen)
    rows = experts_ref.starts(offsets, m)
    x[:rows[0]], x[rows[-1]:], dy[:rows[0]], dy[rows[-1]:] = NAN, NAN, NAN, NAN        # rows of no expert
    for e in range(experts_):
        if rows[e] == rows[e + 1]:
            w[e] = NAN                                                                   # an expert without rows
    off = torch.tensor(offsets, dtype=torch.int64, device=DEV)
    y, dx = draw(m, n, dtype, gen, 1.0, up(n) + 3 * bool(loose), at, 5.0), draw(m, k, dtype, gen, 1.0, up(k), at, 5.0)
    dw = stack(experts_, n, k, dtype, gen, 1.0, up(k), at, 0 if loose else 32, 5.0)
    before = y.clone(), dx.clone()
    ws = experts.new_expert_workspace(x, w, backward=True)
    say("products m=%d e=%d n=%d k=%d %s %s loose=%s" % (m, experts_, n, k, dtype, how, loose))
    experts.zvc_expert_product(x, w, off, y, ws)
    experts.zvc_expert_gradients(dy, x, w, off, dx, dw, ws)
    torch.cuda.synchronize()
    value, bound = experts_ref.product(x, w, offsets, before[0])
    close(y, value, bound, "y")
    wants = experts_ref.gradients(dy, x, w, offsets, before[1])
    for got, (value, bound), name in zip((dx, dw), wants, ("dx", "dw")):
        close(got, value, bound, name)
    for t in (y, dx, dw):                                                                # the gaps
        whole = t._base if t._base is not None else t
        flat = torch.empty(0, dtype=dtype, device=DEV).set_(whole.untyped_storage())
        mask = torch.ones(flat.numel(), dtype=torch.bool, device=DEV)
        mask.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(False)
        assert (flat[mask] == 5).all()


def close(got, value, bound, name):
    off = (got.double() - value).abs() - bound
    assert not got.isnan().any(), name
    assert float(off.max() if off.numel() else 0) <= 0, "%s is off by %g more than it may be" % (name, float(off.max()))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("size", SIZES)
def test_products(size, dtype):
    hows = ("all", "even") if size[0] * size[2] * size[3] > 2e10 else ("all", "some", "one", "wild")
    for i, how in enumerate(hows):
        for loose in ((0, 1, 2) if i == 0 else (i % 2,)):
            run_products(*size, dtype, how, loose)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("how", ["even", "all", "some", "wild"])
@pytest.mark.parametrize("size", [(6165, 3, 2469, 416), (3884, 3, 3749, 496), (5424, 4, 2797, 456)])
def test_a_part_of_a_round_of_large_tiles(size, how, dtype):
    """Even: 270 and 264 tiles of 256 x 256 for 256 workgroups, the last ones in quarters, at a ragged right and lower edge."""
    run_products(*size, dtype, how, 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("n,k", [(1, 1), (3, 5), (8, 8), (15, 17), (64, 64), (65, 33), (129, 250)])
@pytest.mark.parametrize("m,e", [(1, 1), (1, 5), (2, 1), (17, 3), (64, 64), (65, 1024), (130, 2), (513, 5)])
def test_small_products(m, e, n, k, dtype):
    for loose, how in ((0, "some"), (1, "all"), (2, "wild")):
        run_products(m, e, n, k, dtype, how, loose)


@pytest.mark.parametrize("dtype", DTYPES)
def test_products_of_nothing(dtype):
    """Sums over nothing are 0 in the rows that experts have."""
    off = torch.tensor([1, 3, 3], dtype=torch.int64, device=DEV)
    new = lambda *shape, v=3.0: torch.full(shape, v, dtype=dtype, device=DEV)
    y, ws = new(5, 7), torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    experts.zvc_expert_product(new(5, 0), new(2, 7, 0), off, y, ws)
    assert (y[1:3] == 0).all() and (y[:1] == 3).all() and (y[3:] == 3).all()
    dx, dw = new(5, 4), new(2, 0, 4)
    experts.zvc_expert_gradients(new(5, 0), new(5, 4), dw.clone(), off, dx, dw, ws)
    assert (dx[1:3] == 0).all() and (dx[:1] == 3).all() and (dx[3:] == 3).all()
    dw = new(2, 7, 4)
    experts.zvc_expert_gradients(new(0, 7), new(0, 4), new(2, 7, 4), off, new(0, 4), dw, ws)
    assert (dw == 0).all()


@pytest.mark.parametrize("size", [(600, 5, 700, 520), (40, 8, 256, 512), (5000, 2, 1024, 768), (777, 7, 1000, 682)])
def test_the_same_bits_however_they_are_asked_for(size):
    """Twice, one gradient alone, in a stream of its own and from a captured graph, whose replays see what is in the operands then."""
    m, e, n, k = size
    dtype = torch.bfloat16
    gen = generator("bits", *size)
    x, dy, w = draw(m, k, dtype, gen), draw(m, n, dtype, gen), stack(e, n, k, dtype, gen, k ** -0.5, k)
    off = torch.tensor(offsets_of(m, e, "all", gen), dtype=torch.int64, device=DEV)
    ws, other_ws = (experts.new_expert_workspace(x, w, backward=True) for _ in range(2))
    new = lambda: (torch.zeros(m, n, dtype=dtype, device=DEV), torch.zeros(m, k, dtype=dtype, device=DEV), torch.zeros(e, n, k, dtype=dtype, device=DEV))

    def both(out, ws, stream=None):
        experts.zvc_expert_product(x, w, off, out[0], ws, stream=stream)
        experts.zvc_expert_gradients(dy, x, w, off, out[1], out[2], ws, stream=stream)

    first, second, alone, aside, captured = (new() for _ in range(5))
    both(first, ws)
    both(second, ws)
    experts.zvc_expert_product(x, w, off, alone[0], ws)
    experts.zvc_expert_gradients(dy, x, w, off, alone[1], None, ws)
    experts.zvc_expert_gradients(dy, x, w, off, None, alone[2], ws)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    both(aside, other_ws, stream)
    torch.cuda.synchronize()
    for other in (second, aside):
        assert all(torch.equal(a, b) for a, b in zip(first, other))
    for got, want in zip(alone, first):         # (one gradient alone may be cut otherwise than both: its own bits, and near)
        assert float((got.double() - want.double()).norm() / want.double().norm()) < 2.0 ** -8
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(captured, ws)
    for turn in range(3):
        x.copy_(torch.randn(m, k, generator=gen, device=DEV))
        off.copy_(torch.tensor(offsets_of(m, e, "all", gen), dtype=torch.int64, device=DEV))
        for t in captured:
            t.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        want = new()
        for t in want:
            t.fill_(9)
        both(want, other_ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want))


def test_weights_beyond_32_bit_offsets():
    """A stack of 9 GB, and rows of the first and the last experts."""
    e, n, k = 70, 8192, 8192
    w = torch.zeros(e, n, k, dtype=torch.bfloat16, device=DEV)
    gen = generator("beyond")
    for i in (0, 33, 69):
        w[i] = torch.randn(n, k, generator=gen, device=DEV) / 64
    counts = [3 if i in (0, 33, 69) else 0 for i in range(e)]
    off = torch.tensor([sum(counts[:i]) for i in range(e + 1)], dtype=torch.int64, device=DEV)
    x, dy = draw(9, k, torch.bfloat16, gen), draw(9, n, torch.bfloat16, gen)
    y, dx = torch.zeros(9, n, dtype=torch.bfloat16, device=DEV), torch.zeros(9, k, dtype=torch.bfloat16, device=DEV)
    dw = torch.full_like(w, 3.0)
    ws = experts.new_expert_workspace(x, w, backward=True)
    experts.zvc_expert_product(x, w, off, y, ws)
    experts.zvc_expert_gradients(dy, x, w, off, dx, dw, ws)
    for j, i in enumerate((0, 33, 69)):
        rows = slice(3 * j, 3 * j + 3)
        for got, want in ((y[rows], x[rows].double() @ w[i].double().t()), (dx[rows], dy[rows].double() @ w[i].double()),
                          (dw[i], dy[rows].double().t() @ x[rows].double())):
            assert float((got.double() - want).norm() / want.norm()) < 2.0 ** -8
    for i in range(e):
        if counts[i] == 0:
            assert not dw[i].any()


def test_non_finite_numbers_stay_in_their_rows():
    """An infinity or a NaN of one expert's row, or weight, reaches no other row."""
    m, e, n, k = 200, 4, 136, 200
    for dtype in DTYPES:
        gen = generator("finite", str(dtype))
        x, w = draw(m, k, dtype, gen), stack(e, n, k, dtype, gen, 0.1, k)
        x[57, 3], x[120, 199], w[2, 5, 0] = NAN, math.inf, NAN
        off = torch.tensor([0, 50, 100, 150, 200], dtype=torch.int64, device=DEV)
        y = torch.zeros(m, n, dtype=dtype, device=DEV)
        experts.zvc_expert_product(x, w, off, y, experts.new_expert_workspace(x, w))
        odd = ~torch.isfinite(y)
        assert odd[57].all() and odd[120].all() and odd[100:150, 5].all()
        odd[57], odd[120], odd[100:150, 5] = False, False, False
        assert not odd.any()


def test_tensors_elsewhere_are_refused():
    x = torch.zeros(4, 8, device=DEV)
    with pytest.raises(zvc.ZvcError, match="device|one GPU"):
        experts.zvc_expert_product(x, torch.zeros(2, 8, 8, device=DEV), torch.zeros(3, dtype=torch.int64), x.clone(), torch.empty(256, dtype=torch.uint8, device=DEV))


def test_two_calls_at_once():
    """On streams of their own, with workspaces of their own, both of kernels that split their sums; and a router beside them."""
    m, e, n, k = 40, 8, 256, 4096
    gen = generator("at once")
    sets = []
    for _ in range(2):
        x, dy, w = draw(m, k, torch.bfloat16, gen), draw(m, n, torch.bfloat16, gen), stack(e, n, k, torch.bfloat16, gen, k ** -0.5, k)
        off = torch.tensor(offsets_of(m, e, "all", gen), dtype=torch.int64, device=DEV)
        logits = draw(3000, 65, torch.float32, gen)
        sets.append((x, dy, w, off, logits, experts.new_expert_workspace(x, w, backward=True), experts.new_route_workspace(logits, 4)))

    def run(s, stream):
        x, dy, w, off, logits, ws, rws = s
        new = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device=DEV)
        with torch.cuda.stream(stream):
            y, dx, dw = new(m, n), new(m, k), new(e, n, k)
            chosen, weights, offsets, order, place = (new(3000, 4, dtype=torch.int32), new(3000, 4, dtype=torch.float32), new(66, dtype=torch.int64),
                                                      new(12000, dtype=torch.int64), new(3000, 4, dtype=torch.int64))
            for _ in range(20):
                experts.zvc_expert_product(x, w, off, y, ws)
                experts.zvc_expert_gradients(dy, x, w, off, dx, dw, ws)
                experts.zvc_route(logits, chosen, weights, offsets, order, place, rws)
        return y, dx, dw, chosen, weights, offsets, order, place

    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    together = [run(s, stream) for s, stream in zip(sets, streams)]
    torch.cuda.synchronize()
    for s, got in zip(sets, together):
        alone = run(s, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, alone))
