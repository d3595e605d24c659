"""AdamW with states in 32 bits or in 8 (include/zvc_adamw.h), from the header's text and with nothing of the GPU path: 32-bit steps as numpy
computes them, each multiplication and addition rounded, and codes from their definition."""
import math

import numpy as np

from tests.ffn_ref import philox

BLOCK = 128


def numbers():
    """The number of each of the 256 codes."""
    code = np.arange(256)
    exponent, significand = code >> 3 & 15, code & 7
    size = np.where(exponent == 0, significand * 2.0 ** -9, (1 + significand / 8) * 2.0 ** (exponent - 7.0))
    size[(code & 127) == 127] = math.nan
    return np.where(code & 128, -size, size)


NUMBERS = numbers()


def halves(count, tensor, step, seed):
    """The 16-bit number that decides each element's rounding."""
    index = np.arange(-(-count // 8), dtype=np.uint64)
    word = (1 << 32) - 1
    words = philox((index, np.full_like(index, tensor), np.full_like(index, step & word), np.full_like(index, step >> 32)),
                   (seed & word, seed >> 32 & word))
    out = np.empty((index.size, 8), dtype=np.uint64)
    for j in range(8):
        out[:, j] = words[j // 2] >> np.uint64(16 * (j % 2)) & np.uint64(0xFFFF)
    return out.reshape(-1)[:count].astype(np.float64)


def widen(codes, scales):
    return (NUMBERS[codes] * np.repeat(scales.astype(np.float64), BLOCK)[:codes.size]).astype(np.float32)


def narrow(values, random, least):
    """Codes and scales of float32 values.  All steps are exact in 64 bits but the rounding down itself."""
    size = np.abs(values.astype(np.float64))
    finite = np.where(np.isfinite(size), size, 0.0)
    blocks = np.pad(finite, (0, -size.size % BLOCK)).reshape(-1, BLOCK).max(axis=1)
    exponent = np.maximum(np.floor(np.log2(np.maximum(blocks, 2.0 ** -95))), -95)
    scales = 2.0 ** (exponent - 7)
    units = finite / np.repeat(scales, BLOCK)[:size.size]
    step = 2.0 ** (np.maximum(np.floor(np.log2(np.maximum(units, 2.0 ** -6))), -6) - 3)
    # what is below the scaled number's 23 bits of fraction at e4m3's smallest exponent is rounded to the nearest first
    fine = np.where(units < 2.0 ** -6, np.round(units / step * 2 ** 20) / 2 ** 20, units / step)
    up = np.floor(fine + random / 65536) * step
    up = np.minimum(up, 448.0)
    if least:
        up = np.where(size > 0, np.maximum(up, 2.0 ** -9), up)
    up = np.where(np.isfinite(size), up, 448.0)
    codes = np.searchsorted(NUMBERS[:127], up)
    assert (NUMBERS[codes] == up).all()
    return (codes | np.signbit(values) * 128).astype(np.uint8), scales.astype(np.float32)


def states(m, v, grad, beta1, beta2, factor=1.0):
    """m and v after a step, in float32."""
    f = np.float32
    with np.errstate(all="ignore"):
        g = grad.astype(f) * f(factor)
        return f(beta1) * m + f(1 - beta1) * g, f(beta2) * v + f(1 - beta2) * (g * g)


def weights(p, m, v, t, rate, beta1, beta2, eps, decay):
    """(value, bound) of the weights after a step, from the new m and v, in 64 bits."""
    p, m, v = (x.astype(np.float64) for x in (p, m, v))
    with np.errstate(all="ignore"):
        change = rate / (1 - beta1 ** t) * m / (np.sqrt(v / (1 - beta2 ** t)) + eps)
        value = (1 - rate * decay) * p - change
        # in 32 bits: two roundings of p's term, some ten of the other (1/x is one of them, within a unit), one of their difference
        return value, 2.0 ** -22 * np.abs(p) + 2.0 ** -19 * np.abs(change) + 2.0 ** -23 * np.abs(value) + 2.0 ** -126
