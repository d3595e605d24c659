"""The training operators written from their formulas in 64 bits (include/zvc_ffn.h), and how far a
result in 32-bit sums may lie from them.  Shares no code with the GPU path."""
import math

import numpy as np
import torch

F64 = torch.float64
# half a unit in the last place, relative (2^-bits of the significand: 24, 11, 8), and what rounding below the normal numbers costs
ROUND = {torch.float32: (2.0 ** -24, 2.0 ** -149), torch.float16: (2.0 ** -11, 2.0 ** -25),
         torch.bfloat16: (2.0 ** -8, 2.0 ** -134)}
SUM = 2.0 ** -24              # relative error of one addition in 32 bits
# act() and act'() in 32 bits, by exp of an argument of some ten: 2^-24 x |argument| and a few roundings more
ACT = 2.0 ** -18
STEEP = 1.2                   # most of |act'| and of |act''| for silu, gelu and gelu_tanh


def philox(counter, key):
    """Philox4x32-10 for a counter of four 32-bit words and a key of two, numpy arrays or integers."""
    c = [np.atleast_1d(np.asarray(v, dtype=np.uint64)) for v in counter]
    k = [np.uint64(int(v)) for v in key]
    word = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k[0], b & word, (a >> np.uint64(32)) ^ c[3] ^ k[1], a & word]
        k = [np.uint64((int(k[0]) + 0x9E3779B9) & 0xFFFFFFFF), np.uint64((int(k[1]) + 0xBB67AE85) & 0xFFFFFFFF)]
    return c


def numbers(count, seed, offset):
    """The 32-bit number of each element."""
    index = np.arange(-(-count // 8), dtype=np.uint64)
    low, high = index & np.uint64(0xFFFFFFFF), index >> np.uint64(32)
    tail = (offset & 0xFFFFFFFF, offset >> 32 & 0xFFFFFFFF)
    key = (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF)
    out = np.empty((index.size, 8), dtype=np.uint64)
    blocks = [philox((low, high | np.uint64(flag), np.full_like(low, tail[0]), np.full_like(low, tail[1])), key)
              for flag in (0, 0x80000000)]
    for j in range(8):
        upper, lower = ((b[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF) for b in blocks)
        out[:, j] = upper * np.uint64(65536) + lower
    return out.reshape(-1)[:count]


def kept(rows, cols, p, seed, offset):
    if p == 0:
        return torch.ones(rows, cols, dtype=torch.bool)
    return torch.from_numpy(numbers(rows * cols, seed, offset) >= np.uint64(round(p * 2 ** 32))).view(rows, cols)


def drop(t, p, seed, offset):
    stays = kept(t.shape[0], t.shape[1], p, seed, offset).to(t.device)
    return torch.where(stays, t / (1 - p) if p < 1 else t, torch.zeros((), dtype=F64, device=t.device))


def act(g, name):
    """act(g) and act'(g)."""
    if name == "relu":
        return torch.where(g <= 0, 0 * torch.ones_like(g), g), torch.where(g <= 0, 0.0, 1.0).to(F64)
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    if name == "gelu":
        cdf = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return g * (1 + t) / 2, (1 + t) / 2 + g * (1 - t * t) / 2 * c * (1 + 3 * 0.044715 * g ** 2)


def project(x, wg, wu):
    """g, u and how far sums in 32 bits may lie from them."""
    x, wg, wu = x.to(F64), wg.to(F64), wu.to(F64)
    k = x.shape[1]
    return [x @ wg.t(), x @ wu.t(), k * SUM * (x.abs() @ wg.abs().t()), k * SUM * (x.abs() @ wu.abs().t())]


def rounded(value, dtype):
    """What rounding to `dtype` may change."""
    rel, least = ROUND[dtype]
    return rel * value.abs() + least


def forward(x, wg, wu, name, p=0.0, seed=0, offset=0, exact_sums=False):
    """[(value, bound)] of h, gate and up."""
    g, u, dg, du = project(x, wg, wu)
    if exact_sums:
        dg, du = 0 * dg, 0 * du
    a, _ = act(g, name)
    da = STEEP * dg + ACT * g.abs()
    scale = 1 / (1 - p) if p < 1 else 1.0
    stays = kept(*g.shape, p, seed, offset).to(g.device).to(F64)
    h = a * u * scale * stays
    bound = (da * u.abs() + a.abs() * du + da * du) * scale + 2.0 ** -21 * h.abs()
    relu = name == "relu"
    gate, up = (a, torch.where(g <= 0, 0.0, u)) if relu else (g, u)
    out = [(h, bound), (gate * stays, da if relu else dg), (up * stays, du)]
    return [(v, (b + rounded(v.abs() + b, x.dtype)) * stays) for v, b in out]


def backward(dh, x, wg, wu, name, gate=None, up=None, p=0.0, seed=0, offset=0, exact_sums=False):
    """[(value, bound)] of dx, dwg and dwu."""
    dtype = x.dtype
    if gate is None:
        g, u, eg, eu = project(x, wg, wu)
        if exact_sums:
            eg, eu = 0 * eg, 0 * eu
    else:
        g, u = gate.to(F64), up.to(F64)
        eg = eu = torch.zeros_like(g)
    d = drop(dh.to(F64), p, seed, offset)
    a, slope = act(g, name)
    relu = name == "relu"
    ea = STEEP * eg + (0 if relu else ACT) * g.abs()
    eslope = 0 * eg if relu else STEEP * eg + ACT * (1 + g.abs())
    du, dg = d * a, d * u * slope
    bu, bg = d.abs() * ea + 2.0 ** -21 * du.abs(), d.abs() * (eu * slope.abs() + u.abs() * eslope + eu * eslope) + 2.0 ** -21 * dg.abs()
    bu, bg = bu + rounded(du.abs() + bu, dtype), bg + rounded(dg.abs() + bg, dtype)
    x, wg, wu = x.to(F64), wg.to(F64), wu.to(F64)
    m, n = dg.shape
    mags = [(dg.abs() + bg) @ wg.abs() + (du.abs() + bu) @ wu.abs(), (dg.abs() + bg).t() @ x.abs(), (du.abs() + bu).t() @ x.abs()]
    out = [(dg @ wg + du @ wu, bg @ wg.abs() + bu @ wu.abs() + 2 * n * SUM * mags[0]),
           (dg.t() @ x, bg.t() @ x.abs() + m * SUM * mags[1]), (du.t() @ x, bu.t() @ x.abs() + m * SUM * mags[2])]
    return [(v, b + rounded(v.abs() + b, dtype)) for v, b in out]


def grid(rows, cols, std, gen, dtype, device):
    """Draws on a uniform grid of 8-bit numbers: sums of their products are exact in 32 bits."""
    unit = 2.0 ** round(math.log2(std / 32))
    t = torch.randn(rows, cols, generator=gen, device=device) * std
    return ((t / unit).round().clamp(-127, 127) * unit).to(dtype)
