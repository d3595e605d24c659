"""The training operators on the GPU against their formulas in 64 bits (ffn_ref), within bounds that
follow from the types and the lengths of the sums."""
import itertools

import pytest
import torch

from paper_1705_01626_amd import ffn, zvc
from tests import ffn_ref
from tests.gpu_util import say

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
ACTS = list(ffn.ACTIVATIONS)
SENTINEL = -77.0


def generator(*key):
    return torch.Generator(device=DEV).manual_seed(hash(key) % (1 << 31))


class Out:
    """A rows x cols output inside a larger buffer: `pad` elements behind each row, `shift` before the first."""

    def __init__(self, rows, cols, dtype, pad=0, shift=0):
        self.base = torch.full((shift + rows * (cols + pad) + 64,), SENTINEL, dtype=dtype, device=DEV)
        self.t = self.base.as_strided((rows, cols), (cols + pad, 1), shift)

    def untouched(self):
        """Everything around the output still holds what it held."""
        inside = torch.zeros_like(self.base, dtype=torch.bool)
        inside.as_strided(self.t.shape, self.t.stride(), self.t.storage_offset()).fill_(True)
        return bool((self.base[~inside] == SENTINEL).all())


def strided(t, pad=0, shift=0):
    base = torch.full((shift + t.shape[0] * (t.shape[1] + pad) + 64,), float("nan"), dtype=t.dtype, device=DEV)
    out = base.as_strided(t.shape, (t.shape[1] + pad, 1), shift)
    out.copy_(t)
    return out


def check(got, want, name):
    value, bound = want
    error = (got.to(torch.float64) - value).abs()
    bad = ~(error <= bound)
    if bool(bad.any()):
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError("%s: %d of %d elements too far, first at %s: %r, %r wanted, bound %.3g" % (
            name, int(bad.sum()), bad.numel(), at, float(got[at]), float(value[at]), float(bound[at])))


# ---- dropout -------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (1, 7, 0, 0), (3, 8, 0, 0), (5, 13, 0, 1), (64, 4096, 0, 0),
                                                 (33, 72, 8, 0), (33, 72, 5, 0), (7, 1000, 0, 3), (1, 100003, 0, 0),
                                                 (129, 31, 1, 0)])
@pytest.mark.parametrize("residual", [False, True])
def test_dropout(dtype, rows, cols, pad, shift, residual):
    gen = generator(rows, cols, pad, str(dtype))
    x = torch.randn(rows, cols, generator=gen, device=DEV).to(dtype)
    r = torch.randn(rows, cols, generator=gen, device=DEV).to(dtype)
    for p, seed, offset in ((0.0, 1, 2), (0.1, 3, 4), (0.5, (1 << 63) + 5, 1 << 40), (1.0, 7, 8), (2.0 ** -20, 9, 10)):
        say("dropout %s %dx%d pad %d shift %d p %g" % (dtype, rows, cols, pad, shift, p))
        y = Out(rows, cols, dtype, pad, shift)
        ffn.zvc_dropout(strided(x, pad, shift), y.t, p, seed, offset, residual=strided(r, pad, shift) if residual else None)
        want = ffn_ref.drop(x.to(torch.float64), p, seed, offset) + (r.to(torch.float64) if residual else 0)
        check(y.t, (want, ffn_ref.rounded(want, dtype) + 2.0 ** -22 * (want.abs() + r.abs().to(torch.float64))), "y")
        stays = ffn_ref.kept(rows, cols, p, seed, offset).to(DEV)
        assert torch.equal(y.t[~stays], (r if residual else torch.zeros_like(r))[~stays])
        assert y.untouched()


def test_dropout_where_sixteen_bits_do_not_decide():
    """p just above and just below a multiple of 2^-16: elements whose upper 16 bits equal p's are decided by the lower."""
    n = 1 << 21
    x = torch.ones(n, device=DEV)
    drops = []
    for low in (0, 1, 0x8000, 0xFFFF):
        p = (0x4000 * 65536 + low) / 2.0 ** 32
        y = torch.empty_like(x)
        ffn.zvc_dropout(x, y, p, 11, 12)
        drops.append(y == 0)
        assert torch.equal(~drops[-1].cpu(), ffn_ref.kept(1, n, p, 11, 12)[0])
    tied = int((drops[-1] & ~drops[0]).sum())
    assert 8 < tied < 80                                  # 32 expected
    assert not bool((drops[0] & ~drops[1]).any() | (drops[1] & ~drops[2]).any() | (drops[2] & ~drops[3]).any())


def test_dropout_of_any_shape_in_place_and_of_what_is_no_number():
    x = torch.randn(3, 5, 7, 4, device=DEV, dtype=torch.float16)
    stays = ffn_ref.kept(1, x.numel(), 0.5, 1, 0).view(x.shape).to(DEV)
    x[~stays] = float("inf")
    x[0, 0, 0, 0] = float("nan")
    y = torch.empty_like(x)
    ffn.zvc_dropout(x, y, 0.5, 1)
    assert torch.equal(y[~stays], torch.zeros_like(y[~stays]))
    assert bool(torch.isnan(y[0, 0, 0, 0])) == bool(stays[0, 0, 0, 0])
    assert torch.equal(y[stays][1:], (x * 2)[stays][1:])
    ffn.zvc_dropout(x, x, 0.5, 1)
    assert torch.equal(torch.nan_to_num(x), torch.nan_to_num(y))
    r = torch.randn_like(x)
    want = torch.empty_like(r)
    z = torch.randn_like(x)
    ffn.zvc_dropout(z, want, 0.25, 5, residual=r)
    ffn.zvc_dropout(z, r, 0.25, 5, residual=r)
    assert torch.equal(r, want)


def test_dropout_gradient_is_the_same_call():
    """<drop(x), v> = <x, drop(v)>, with numbers whose products and sums are exact."""
    gen = generator("adjoint")
    x = torch.randint(-8, 9, (100, 333), generator=gen, device=DEV).float()
    v = torch.randint(-8, 9, (100, 333), generator=gen, device=DEV).float()
    y, g = torch.empty_like(x), torch.empty_like(x)
    ffn.zvc_dropout(x, y, 0.5, 21, 3)
    ffn.zvc_dropout(v, g, 0.5, 21, 3)
    assert float((y.double() * v.double()).sum()) == float((x.double() * g.double()).sum())


def test_dropout_beyond_32_bit_offsets():
    """A tensor of more than 2^32 elements: its last ones are what the generator says."""
    rows, cols = (1 << 20) + 3, 4104
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device=DEV)
    ffn.zvc_dropout(x, x, 0.5, 5, 6)
    for row in (0, 1 << 19, (1 << 20) - 1, rows - 1):
        first = row * cols
        assert first % 8 == 0
        import numpy as np
        index = np.arange(first // 8, (first + cols) // 8, dtype=np.uint64)
        words = ffn_ref.philox((index & np.uint64(0xFFFFFFFF), index >> np.uint64(32), np.full_like(index, 6),
                                np.zeros_like(index)), (5, 0))
        halves = np.stack([(words[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF) for j in range(8)], 1).reshape(-1)
        assert torch.equal((x[row] != 0).cpu(), torch.from_numpy(halves >= 0x8000))
    assert abs(float((x == 0).float().mean(dim=1).mean()) - 0.5) < 1e-3


# ---- the gated block ------------------------------------------------------------------
SIZES = [(1, 8, 8), (1, 130, 64), (3, 37, 33), (5, 512, 200), (16, 64, 256), (17, 33, 40), (64, 256, 128), (65, 129, 72),
         (130, 264, 96), (257, 136, 65), (300, 520, 264), (1, 1, 1), (2, 3000, 1000)]


def problem(m, n, k, dtype, name, *key):
    gen = generator(m, n, k, str(dtype), *key)
    if name == "relu":
        make = lambda rows, cols, std: ffn_ref.grid(rows, cols, std, gen, dtype, DEV)
    else:
        make = lambda rows, cols, std: (torch.randn(rows, cols, generator=gen, device=DEV) * std).to(dtype)
    return make(m, k, 1.0), make(n, k, k ** -0.5), make(n, k, k ** -0.5), torch.randn(m, n, generator=gen, device=DEV).to(dtype)


def forward(x, wg, wu, name, keep=False, pad=0, shift=0, **drop):
    m, n = x.shape[0], wg.shape[0]
    outs = [Out(m, n, x.dtype, pad, shift) for _ in range(3 if keep else 1)]
    ws = ffn.new_glu_workspace(x, wg, wu)
    ws.fill_(0xFF)                                        # NaNs in every type
    ffn.zvc_glu_forward(x, wg, wu, outs[0].t, ws, name, outs[1].t if keep else None, outs[2].t if keep else None, **drop)
    assert all(o.untouched() for o in outs)
    return [o.t for o in outs]


def backward(dh, x, wg, wu, name, gate=None, up=None, pad=0, shift=0, **drop):
    m, n, k = x.shape[0], wg.shape[0], x.shape[1]
    outs = [Out(m, k, x.dtype, pad, shift), Out(n, k, x.dtype, pad, shift), Out(n, k, x.dtype, pad, shift)]
    ws = ffn.new_glu_workspace(x, wg, wu, backward=True)
    ws.fill_(0xFF)
    ffn.zvc_glu_backward(dh, x, wg, wu, outs[0].t, outs[1].t, outs[2].t, ws, name, gate, up, **drop)
    assert all(o.untouched() for o in outs)
    return [o.t for o in outs]


def check_block(m, n, k, dtype, name, keep, drop, pad=0, shift=0):
    say("glu %dx%dx%d %s %s keep %s %s pad %d shift %d" % (m, n, k, dtype, name, keep, drop, pad, shift))
    x, wg, wu, dh = problem(m, n, k, dtype, name)
    exact = name == "relu"
    want = ffn_ref.forward(x, wg, wu, name, exact_sums=exact, **drop)
    x, wg, wu, dh = (strided(t, pad, shift) for t in (x, wg, wu, dh))
    got = forward(x, wg, wu, name, keep, pad, shift, **drop)
    for g, w, label in zip(got, want, ("h", "gate", "up")):
        check(g, w, label)
    gate, up = got[1:] if keep else (None, None)
    for g, w, label in zip(backward(dh, x, wg, wu, name, gate, up, pad, shift, **drop),
                           ffn_ref.backward(dh, x, wg, wu, name, gate, up, exact_sums=exact, **drop), ("dx", "dwg", "dwu")):
        check(g, w, label)


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", DTYPES)
def test_block_sizes(m, n, k, dtype):
    for name, keep, p in (("silu", False, 0.0), ("relu", True, 0.3)):
        check_block(m, n, k, dtype, name, keep, {"p": p, "seed": 3, "offset": 4})


@pytest.mark.parametrize("m", [1, 16, 17, 32, 33, 48, 49, 64, 65, 96, 97, 128, 129])
@pytest.mark.parametrize("dtype", DTYPES)
def test_block_few_tokens(m, dtype):
    """Around every number of tokens at which another kernel takes over; sums of less than 128 bytes, of a few times that and
    of many, with and without a rest; more columns than a workgroup for each compute unit takes."""
    for n, k in ((24, 8), (40, 136), (264, 1032), (4104, 72)):
        check_block(m, n, k, dtype, "silu", m % 2 == 0, {"p": 0.1, "seed": m})
        if k <= 136:
            check_block(m, n, k, dtype, "relu", m % 2 == 1, {"p": 0.0})


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("p", [0.0, 0.25, 0.1, 1.0])
def test_block_activations_and_dropout(name, keep, p):
    for dtype in DTYPES:
        check_block(70, 136, 96, dtype, name, keep, {"p": p, "seed": (1 << 40) + 3, "offset": 1 << 33})
        check_block(9, 75, 48, dtype, name, keep, {"p": p, "seed": 1, "offset": 0})


@pytest.mark.parametrize("pad,shift", [(8, 0), (3, 0), (0, 1), (8, 8), (5, 7)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_block_strides_and_alignment(pad, shift, dtype):
    for m, n, k in ((66, 136, 64), (4, 64, 128), (200, 300, 96)):
        check_block(m, n, k, dtype, "gelu", True, {"p": 0.2, "seed": 5}, pad, shift)


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (7, 2048, 1024), (40, 1536, 2048), (128, 1024, 4096), (513, 1032, 520),
                                   (1024, 1024, 1024), (2050, 264, 328), (4096, 72, 64), (100, 128, 8200), (64, 8200, 128)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_block_larger_and_long_sums(m, n, k, dtype):
    check_block(m, n, k, dtype, "silu", m % 2 == 0, {"p": 0.1, "seed": 8})


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,n,k", [(1, 40, 64), (20, 264, 512), (300, 512, 256)])
def test_projections_are_exact_on_a_grid(m, n, k, dtype):
    """Sums of grid numbers have no rounding at all, so the kept projections are the rounded true ones."""
    x, wg, wu, _ = problem(m, n, k, dtype, "relu")
    _, gate, up = forward(x, wg, wu, "relu", True)
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    assert torch.equal(gate, g.clamp(min=0).to(dtype)) and torch.equal(up, torch.where(g > 0, u, 0.0).to(dtype))


def test_dropout_inside_is_dropout_behind():
    """Zeros in the same places as zvc_dropout puts them, also where a row's length is no multiple of eight."""
    for n in (64, 75):
        x, wg, wu, _ = problem(50, n, 64, torch.bfloat16, "silu")
        plain = forward(x, wg, wu, "silu")[0].contiguous()
        dropped = forward(x, wg, wu, "silu", p=0.3, seed=9, offset=2)[0]
        behind = torch.empty_like(plain)
        ffn.zvc_dropout(plain, behind, 0.3, 9, 2)
        assert torch.equal(dropped == 0, behind == 0)


def test_kept_projections_leave_through_the_codec_and_come_back():
    x, wg, wu, dh = problem(256, 512, 128, torch.bfloat16, "relu")
    drop = {"p": 0.2, "seed": 3}
    _, gate, up = (t.contiguous() for t in forward(x, wg, wu, "relu", True, **drop))
    want = backward(dh, x, wg, wu, "relu", gate, up, **drop)
    back = []
    for t in (gate, up):
        comp, nbytes = zvc.compress_tensor(t)
        assert nbytes < 0.55 * t.numel() * 2              # half of g is positive, a fifth dropped, 1/16 for masks
        out = torch.empty_like(t)
        zvc.zvc_decompress(comp, nbytes, out, zvc.new_workspace(t.numel(), 2))
        back.append(out)
    for a, b in zip(backward(dh, x, wg, wu, "relu", *back, **drop), want):
        assert torch.equal(a, b)


def test_rows_that_dropout_leaves_nothing_of_ignore_what_is_there():
    """p = 1: gradients are zero whatever dh holds; a NaN of x reaches its own row of h only."""
    x, wg, wu, dh = problem(70, 72, 64, torch.float16, "silu")
    dh[3] = float("nan")
    dh[4] = float("inf")
    for keep in (False, True):
        h, gate, up = forward(x, wg, wu, "silu", True, p=1.0)
        assert not bool(h.any() | gate.any() | up.any())
        for t in backward(dh, x, wg, wu, "silu", gate if keep else None, up if keep else None, p=1.0):
            assert not bool(t.any())
    x[5, 1] = float("nan")
    h = forward(x, wg, wu, "silu")[0]
    assert bool(torch.isnan(h[5]).all()) and not bool(torch.isnan(h[:5]).any() | torch.isnan(h[6:]).any())


@pytest.mark.parametrize("dtype", DTYPES)
def test_parts_of_the_gradient(dtype):
    x, wg, wu, dh = problem(130, 136, 72, dtype, "gelu")
    ws = ffn.new_glu_workspace(x, wg, wu, backward=True)
    want = backward(dh, x, wg, wu, "gelu")
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    ffn.zvc_glu_backward(dh, x, wg, wu, dx, None, None, ws, "gelu")
    ffn.zvc_glu_backward(dh, x, wg, wu, None, dwg, dwu, ws, "gelu")
    for a, b in zip((dx, dwg, dwu), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", DTYPES)
def test_sums_over_nothing(dtype):
    new = lambda *shape: torch.full(shape, SENTINEL, dtype=dtype, device=DEV)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    h, gate, up = new(5, 6), new(5, 6), new(5, 6)
    ffn.zvc_glu_forward(new(5, 0), new(6, 0), new(6, 0), h, ws, "gelu", gate, up)
    assert not bool(h.any() | gate.any() | up.any())
    dwg, dwu = new(6, 8), new(6, 8)
    ffn.zvc_glu_backward(new(0, 6), new(0, 8), new(6, 8), new(6, 8), new(0, 8), dwg, dwu, ws)
    assert not bool(dwg.any() | dwu.any())
    dx = new(5, 8)
    ffn.zvc_glu_backward(new(5, 0), new(5, 8), new(0, 8), new(0, 8), dx, new(0, 8), new(0, 8), ws)
    assert not bool(dx.any())


def test_halves_of_wider_buffers():
    """gate | up and dwg | dwu as halves of one buffer each, side by side and one after the other."""
    x, wg, wu, dh = problem(40, 48, 64, torch.bfloat16, "silu")
    _, gate, up = forward(x, wg, wu, "silu", True)
    both, h = torch.zeros(40, 96, dtype=x.dtype, device=DEV), torch.empty_like(dh)
    w = torch.cat([wg, wu])
    ws = ffn.new_glu_workspace(x, wg, wu, backward=True)
    ffn.zvc_glu_forward(x, w[:48], w[48:], h, ws, "silu", both[:, :48], both[:, 48:])
    assert torch.equal(both, torch.cat([gate, up], dim=1))
    dw, dx = torch.zeros_like(w), torch.empty_like(x)
    ffn.zvc_glu_backward(dh, x, w[:48], w[48:], dx, dw[:48], dw[48:], ws, "silu", both[:, :48], both[:, 48:])
    want = backward(dh, x, wg, wu, "silu", gate, up)
    assert torch.equal(dx, want[0]) and torch.equal(dw, torch.cat(want[1:]))


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_against_differences(dtype):
    """<dx, v> against (f(x + v) - f(x - v)) / 2 with f = <h, dh> by the kernels themselves; a curvature of order one and
    steps of 1/64 leave 2^-12 of the sum's size, and h's roundings sqrt(elements) of their own size each."""
    m, n, k = 24, 40, 64
    x, wg, wu, dh = problem(m, n, k, dtype, "gelu_tanh", "differences")
    gen = generator("directions")
    dx, dwg, dwu = backward(dh, x, wg, wu, "gelu_tanh")
    f = lambda x, wg, wu: float((forward(x, wg, wu, "gelu_tanh")[0].double() * dh.double()).sum())
    for which, grad in enumerate((dx, dwg, dwu)):
        args = [x, wg, wu]
        v = torch.randn(grad.shape, generator=gen, device=DEV) * (2.0 ** -6 if which == 0 else 2.0 ** -6 * k ** -0.5)
        ends, moved = [], []
        for sign in (1, -1):
            moved.append((args[which].float() + sign * v).to(dtype))
            ends.append(f(*[moved[-1] if i == which else a for i, a in enumerate(args)]))
        step = (moved[0].double() - moved[1].double()) / 2
        slope = float((grad.double() * step).sum())
        h = forward(x, wg, wu, "gelu_tanh")[0].double()
        rounding = ffn_ref.ROUND[dtype][0] * float((h * dh.double()).norm()) * 6 + 2.0 ** -18
        assert abs((ends[0] - ends[1]) / 2 - slope) < rounding + 2.0 ** -10 * float(grad.double().norm() * step.norm())


def test_another_stream_and_one_workspace_after_the_other():
    x, wg, wu, dh = problem(200, 264, 128, torch.bfloat16, "silu")
    want = forward(x, wg, wu, "silu")[0].clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    h, ws = torch.empty_like(dh), ffn.new_glu_workspace(x, wg, wu)
    ffn.zvc_glu_forward(x, wg, wu, h, ws, "silu", stream=side)
    y = torch.empty_like(h)
    ffn.zvc_dropout(h, y, 0.5, 1, stream=side)
    side.synchronize()
    assert torch.equal(h, want)
    assert torch.equal(y == 0, (~ffn_ref.kept(200, 264, 0.5, 1, 0)).to(DEV) | (h == 0))


def test_captured_step_drops_other_elements_at_each_replay():
    """A graph of forward, backward and dropout whose offset lies in device memory, against eager calls."""
    x, wg, wu, dh = problem(48, 136, 64, torch.float16, "silu")
    ws = ffn.new_glu_workspace(x, wg, wu, backward=True)
    word = torch.zeros(1, dtype=torch.int64, device=DEV)

    def step(offset, d_offset):
        out = [torch.empty_like(dh), torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu), torch.empty_like(x)]
        drop = {"p": 0.5, "seed": 6, "offset": offset, "d_offset": d_offset}
        ffn.zvc_glu_forward(x, wg, wu, out[0], ws, "silu", **drop)
        ffn.zvc_glu_backward(dh, x, wg, wu, out[1], out[2], out[3], ws, "silu", **drop)
        ffn.zvc_dropout(x, out[4], **drop)
        return out

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(0, word)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(10, word)
    seen = []
    for replay in range(4):
        word.fill_(replay * 3)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, step(10 + replay * 3, None)):
            assert torch.equal(a, b), replay
        seen.append(captured[0].clone())
    assert all(not torch.equal(a, b) for a, b in itertools.combinations(seen, 2))


def test_calls_repeat_bit_for_bit():
    x, wg, wu, dh = problem(333, 520, 264, torch.bfloat16, "gelu")
    first = backward(dh, x, wg, wu, "gelu", p=0.1, seed=2)
    for _ in range(3):
        for a, b in zip(backward(dh, x, wg, wu, "gelu", p=0.1, seed=2), first):
            assert torch.equal(a, b)


def test_rows_beyond_32_bit_offsets():
    """x and h of more than 4 GB each: the last rows are what they are alone."""
    m, n, k = (1 << 22) + 5, 520, 520
    x = torch.empty(m, k, dtype=torch.bfloat16, device=DEV)
    gen = generator("far")
    tail = torch.randn(300, k, generator=gen, device=DEV).to(x.dtype)
    x[:1024] = 0
    x[1024:] = tail[0]
    x[-300:] = tail
    wg = (torch.randn(n, k, generator=gen, device=DEV) * k ** -0.5).to(x.dtype)
    wu = (torch.randn(n, k, generator=gen, device=DEV) * k ** -0.5).to(x.dtype)
    h = torch.empty(m, n, dtype=x.dtype, device=DEV)
    ffn.zvc_glu_forward(x, wg, wu, h, ffn.new_glu_workspace(x, wg, wu), "silu")
    check(h[-300:], ffn_ref.forward(tail, wg, wu, "silu")[0], "h")
    assert not bool(h[:1024].any())


def test_gradients_of_rows_beyond_32_bit_offsets():
    """x, dh, dg and du of more than 4 GB each; only the last rows of dh are not zero, so the gradients are theirs alone."""
    m, n, k, rows = (1 << 22) + 5, 520, 520, 300
    gen = generator("far back")
    make = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)
    x = make(1, k).to(torch.bfloat16).expand(m, k).contiguous()
    x[-rows:] = make(rows, k).to(x.dtype)
    dh = torch.zeros(m, n, dtype=x.dtype, device=DEV)
    dh[-rows:] = make(rows, n).to(x.dtype)
    wg, wu = ((make(n, k) * k ** -0.5).to(x.dtype) for _ in range(2))
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    ffn.zvc_glu_backward(dh, x, wg, wu, dx, dwg, dwu, ffn.new_glu_workspace(x, wg, wu, backward=True), "silu")
    want = ffn_ref.backward(dh[-rows:], x[-rows:], wg, wu, "silu")
    check(dx[-rows:], want[0], "dx")
    assert not bool(dx[:1 << 20].any()) and not bool(dx[-rows - (1 << 20):-rows].any())
    for got, expected, label in zip((dwg, dwu), want[1:], ("dwg", "dwu")):
        check(got, expected, label)                       # (adding zeros rounds nothing)


@pytest.mark.parametrize("m,n,k", [(33, 48, 64), (129, 1032, 264), (600, 72, 2056)])
def test_gradients_ignore_what_lies_behind_the_rows(m, n, k):
    """Rows with gaps full of NaNs, odd tokens and columns in a stage, and a workspace full of NaNs: nothing of it gets in."""
    x, wg, wu, dh = problem(m, n, k, torch.bfloat16, "relu")
    want = backward(dh, x, wg, wu, "relu")
    got = backward(strided(dh, 8), strided(x, 16), strided(wg, 8), strided(wu, 8), "relu")
    for a, b in zip(got, want):
        assert torch.equal(a, b)
