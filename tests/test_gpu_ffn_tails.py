"""act(g) and act'(g) of the kernels over the whole range of g, relative to the value itself: far below 0 it is small, and a bound
on the absolute error says nothing there.

One token a value, g = x[0] and u = x[1] = 1 by weights that are 0 and 1, so both projections are exact; dh = 1, so that
dx[0] = act'(g) and dx[1] = act(g).

What the results may be off by, relative: half a unit in the last place of the type; exp's argument z, which up to nine roundings of
2^-24 leave 9 |z| x 2^-24 away; 16 x 2^-24 for what else is computed; and 2^-15 where gelu is computed for 16-bit types, a
quarter of fp16's rounding."""
import math

import pytest
import torch

from paper_1705_01626_amd import ffn
from tests import ffn_ref
from tests import test_gpu_ffn as blocks

pytestmark = pytest.mark.gpu
DEV = "cuda"
DTYPES = [torch.bfloat16, torch.float16, torch.float32]
F64 = torch.float64


def activations(g, name, rows=64):
    """act(g) from the forward pass, act(g) and act'(g) from the backward pass, for a vector g."""
    dtype = g.dtype
    pad = -g.numel() % rows
    g = torch.cat([g, torch.ones(pad, dtype=dtype, device=DEV)])
    m = g.numel()
    x = torch.zeros(m, 8, dtype=dtype, device=DEV)
    x[:, 0], x[:, 1] = g, 1
    wg, wu = torch.zeros(1, 8, dtype=dtype, device=DEV), torch.zeros(1, 8, dtype=dtype, device=DEV)
    wg[0, 0], wu[0, 1] = 1, 1
    h, dx, dwg, dwu = torch.empty(m, 1, dtype=dtype, device=DEV), torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    ws = ffn.new_glu_workspace(x, wg, wu, backward=True)
    ffn.zvc_glu_forward(x, wg, wu, h, ws, name)
    ffn.zvc_glu_backward(torch.ones_like(h), x, wg, wu, dx, dwg, dwu, ws, name)
    return [t[:m - pad].contiguous() for t in (h[:, 0], dx[:, 1], dx[:, 0])]


def argument(g, name):
    """exp's argument."""
    if name == "silu":
        return g.abs()
    return g * g / 2 if name == "gelu" else (2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)).abs()


def grid_of(dtype, least, most, count=40000):
    return torch.linspace(least, most, count, dtype=F64, device=DEV).to(dtype).unique()


def off(name, dtype, g):
    z = argument(g.to(F64), name)
    return (16 + 9 * z) * 2.0 ** -24 + (2.0 ** -15 if name == "gelu" and dtype != torch.float32 else 0)


# as far as results are normal numbers in 32 bits
RANGE = {"silu": (-80, 80), "gelu": (-12, 12), "gelu_tanh": (-9.5, 9.5)}


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", list(RANGE))
@pytest.mark.parametrize("tokens", [64, 40000])
def test_values_relative_to_themselves(name, dtype, tokens):
    """Few tokens, where each kernel is called for itself, and many."""
    g = grid_of(dtype, *RANGE[name], count=tokens)
    value = ffn_ref.act(g.to(F64), name)[0] if name != "gelu_tanh" else g.to(F64) * torch.sigmoid(
        2 * math.sqrt(2 / math.pi) * (g.to(F64) + 0.044715 * g.to(F64) ** 3))
    bound = off(name, dtype, g) * value.abs()
    bound = bound + ffn_ref.rounded(value.abs() + bound, dtype)
    h, du, _ = activations(g, name)
    blocks.check(h, (value, bound), "h")
    blocks.check(du, (value, bound), "du")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", list(RANGE))
def test_slopes_relative_to_their_terms(name, dtype):
    """act' is a sum of two terms of different signs below 0: relative to the larger one."""
    g = grid_of(dtype, *RANGE[name])
    x = g.to(F64)
    if name == "silu":
        s = torch.sigmoid(x)
        terms = s, x * s * torch.sigmoid(-x)
    elif name == "gelu":
        terms = 0.5 * torch.erfc(-x / math.sqrt(2)), x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    else:
        c = 2 * math.sqrt(2 / math.pi)
        s = torch.sigmoid(c * (x + 0.044715 * x ** 3))
        terms = s, x * s * torch.sigmoid(-c * (x + 0.044715 * x ** 3)) * c * (1 + 0.134145 * x * x)
    value = terms[0] + terms[1]
    # (1 - s at s near 1 has the rounding of s: 2^-24 of the factors that it is multiplied by)
    bound = off(name, dtype, g) * (terms[0].abs() + terms[1].abs()) + 2.0 ** -23 * (x > 0) * (1 + x.abs()) * (1 + x * x)
    bound = bound + ffn_ref.rounded(value.abs() + bound, dtype)
    blocks.check(activations(g, name)[2], (value, bound), "slope")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", ["relu", *RANGE])
def test_large_numbers_have_the_limits(name, dtype):
    """act(g) = g and act' = 1 far above 0, 0 and 0 far below it, up to the largest number of the type."""
    g = torch.tensor([s * v for s in (1.0, -1.0) for v in (200.0, 1e5, 1e13, 1e18, 3e19, 1e20, 1e30, 3e38)], device=DEV).to(dtype)
    h, du, slope = activations(g, name)
    zero = torch.zeros_like(g)
    assert torch.equal(h, torch.where(g > 0, g, zero)) and torch.equal(du, h)
    assert torch.equal(slope, (g > 0).to(dtype))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("name", ["relu", *RANGE])
@pytest.mark.parametrize("rows", [3, 700])
def test_a_nan_stays_one(name, dtype, rows):
    """In each type and activation, few tokens and many."""
    g = torch.randn(rows, device=DEV).to(dtype)
    g[1] = float("nan")
    there = torch.arange(rows, device=DEV) == 1
    for t, label in zip(activations(g, name, rows), ("h", "du", "slope")):
        assert torch.equal(torch.isnan(t), there), label


def test_silu_in_32_bits():
    """To a few units in the last place wherever it is a normal number: 8 x 2^-24."""
    g = grid_of(torch.float32, -87, 88)
    value = g.to(F64) * torch.sigmoid(g.to(F64))
    bound = 2.0 ** -21 * value.abs() + 2.0 ** -125
    for t in activations(g, "silu")[:2]:
        blocks.check(t, (value, bound), "silu")
