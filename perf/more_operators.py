"""What the operators of mixtures of experts and the optimizer's step are measured by.

A case is one pass through a public entry point of paper_1705_01626_amd.experts or .adamw on buffers that a
training or serving program keeps:

  route            each token's `top` largest logits among the experts, their softmax weights, and the order of all
                   (token, choice) entries by expert: what the products and the gathering of their rows go by
  route_backward   the gradient of the logits from that of the weights
  product          y[r] = x[r] W_e^T for the rows r of expert e, which lie one expert behind the other
  gradients        dx[r] = dy[r] W_e and dW_e = dy_e^T x_e
  adamw            one AdamW step over many tensors: weights and, for 16-bit ones, their 32-bit masters; states in 32 bits or
                   in 8 (e4m3, a scale that is a power of two for each block of 128 elements, stochastic rounding)

An expert's logit of minus infinity (or a NaN) takes the expert out of a token's choice; a token without
any is padding and takes no row.  Rows behind the last expert's stay as they were.

The 8-bit states' stochastic rounding takes its random numbers from a counter-based generator, a function of
(seed, step, tensor, element), so that every implementation rounds alike.
"""
import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}
LARGEST_FLOPS = 4 * 16384 * 5632 * 2048
LARGEST_WEIGHTS = 32 * 5632 * 2048
LARGEST_STEP = 8 * 3 * 2816 * 2048 * 28             # bytes
BLOCK = 128                                         # elements that share a scale
SMALL = 4096                                        # tensors below keep their states in 32 bits


# ------------------------------------------------------------------------------- cases
def _route(name, op, dtype, m, experts, top, normalize, masked=0.0, pad=0):
    """m tokens; masked: share of tokens that are padding, and of experts' logits that are taken out."""
    case = {"op": op, "dtype": dtype, "m": int(m), "experts": int(experts), "top": int(top), "normalize": bool(normalize),
            "masked": float(masked), "pad": int(pad)}
    return dict(case, name=name) if name else case


def _product(name, op, dtype, m, experts, n, k, skew=0.3, spare=0, pad=0):
    """m rows over the experts, the more unevenly the larger `skew`; spare: rows behind the last; pad: elements between rows of x."""
    case = {"op": op, "dtype": dtype, "m": int(m), "experts": int(experts), "n": int(n), "k": int(k), "skew": float(skew),
            "spare": int(spare), "pad": int(pad)}
    return dict(case, name=name) if name else case


def _adamw(name, dtype, grad, bits, blocks, width, inner, odd=0, master=True, shapes=0):
    """blocks: gated blocks (three inner x width matrices and two vectors each); odd: that many tensors of any small size besides,
    everything back to back at odd elements."""
    case = {"op": "adamw", "dtype": dtype, "grad": grad, "bits": int(bits), "blocks": int(blocks), "width": int(width),
            "inner": int(inner), "odd": int(odd), "master": bool(master and dtype != "fp32"), "shapes": int(shapes)}
    return dict(case, name=name) if name else case


def listed():
    return [
        # Eight tokens of a decoding batch choose among 64 experts: the smallest call, a matter of latency.
        _route("route_decode_bf16", "route", "bf16", 8, 64, 8, True),
        # A long prompt's tokens among many experts, a part of them padding.
        _route("route_prompt_fp32", "route", "fp32", 16384, 256, 8, False, masked=0.1),
        # The training step's router, two of 64 experts.
        _route("route_backward_train_fp32", "route_backward", "fp32", 4096, 64, 2, True),
        # A long batch, weights from the softmax over all experts.
        _route("route_backward_long_bf16", "route_backward", "bf16", 16384, 256, 8, False, masked=0.1),
        # One token through eight of 64 small experts: eight weights read once for a row each.
        _product("product_token_bf16", "product", "bf16", 8, 64, 2816, 1024, skew=0.0),
        # An ordinary training forward: 4096 tokens, two of 16 experts each.
        _product("product_train_bf16", "product", "bf16", 8192, 16, 5632, 2048),
        # A ragged one: odd rows and widths, some experts without a row, room behind the last.
        _product("product_ragged_fp16", "product", "fp16", 1554, 13, 2730, 1000, skew=1.2, spare=100, pad=24),
        # Both gradients of a long batch: the largest.
        _product("gradients_train_bf16", "gradients", "bf16", 16384, 32, 5632, 2048),
        # Ragged gradients in 32 bits.
        _product("gradients_ragged_fp32", "gradients", "fp32", 777, 7, 1000, 682, skew=1.2, spare=23),
        # A step over many small tensors (biases, norms, a few matrices) at odd addresses.
        _adamw("adamw_odd_bf16", "bf16", "bf16", 32, 1, 256, 512, odd=200, shapes=1),
        # A model of eight blocks in 32 bits, states in 32 bits.
        _adamw("adamw_blocks_fp32", "fp32", "fp32", 32, 8, 2048, 2816),
        # Two larger blocks in mixed precision, states in 8 bits.
        _adamw("adamw_8bit_bf16", "bf16", "bf16", 8, 2, 4096, 5632, odd=7, shapes=2),
    ]


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))


def draw(rng):
    op = rng.choice(("route", "route_backward", "product", "product", "gradients", "gradients", "adamw", "adamw"))
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    if op.startswith("route"):
        experts = _log_uniform(rng, 2, 512)
        top = min(experts, rng.choice((1, 2, 4, 6, 8)))
        most = 16384 * 256 // max(64, experts)
        return _route(None, op, dtype, _log_uniform(rng, 1 if op == "route" else 16, min(16384, most)), experts, top,
                      rng.random() < 0.5, rng.choice((0.0, 0.0, 0.1, 0.5)), rng.choice((0, 0, 3)))
    if op != "adamw":
        n, k = _log_uniform(rng, 128, 8192), _log_uniform(rng, 128, 4096)
        if rng.random() < 0.6:
            n, k = n // 64 * 64, k // 64 * 64
        elif rng.random() < 0.6:
            n, k = n // 2 * 2, k // 8 * 8
        experts = _log_uniform(rng, 1, max(1, min(128, LARGEST_WEIGHTS // (n * k))))
        flops = LARGEST_FLOPS // 16 if dtype == "fp32" else LARGEST_FLOPS
        m = _log_uniform(rng, 1, max(1, min(16384, flops // ((2 if op == "product" else 4) * n * k))))
        return _product(None, op, dtype, m, experts, n, k, rng.choice((0.0, 0.3, 1.2)), rng.choice((0, 0, 77)),
                        rng.choice((0, 0, 0, 8, 3)))
    width, inner = _log_uniform(rng, 64, 4096) // 8 * 8, _log_uniform(rng, 128, 8192)
    most = max(1, min(16, LARGEST_STEP // (28 * 3 * width * inner)))
    return _adamw(None, dtype, rng.choice((dtype, dtype, "fp32")), rng.choice((8, 32)), _log_uniform(rng, 1, most), width, inner,
                  rng.choice((0, 0, 5, 40)), rng.random() < 0.7, rng.randrange(1000))


# ------------------------------------------------------------------------------- inputs
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 31)
    return gen


def _route_inputs(case, seed):
    gen, m, experts = _generator(seed), case["m"], case["experts"]
    logits = torch.randn(m, experts + case["pad"], generator=gen, device="cuda")
    logits += 0.5 * torch.randn(experts + case["pad"], generator=gen, device="cuda")       # some experts are liked more
    if case["masked"]:
        drop = torch.rand(m, 1, generator=gen, device="cuda") < case["masked"]
        out = torch.rand(m, experts + case["pad"], generator=gen, device="cuda") < case["masked"]
        logits.masked_fill_(drop | out, -math.inf)
    s = {"logits": logits.to(DTYPES[case["dtype"]])[:, :experts]}
    if case["op"] == "route_backward":
        s["dweights"] = torch.randn(m, case["top"], generator=gen, device="cuda")
        s["chosen"] = _choose(s["logits"], case["top"])
    return s


def _bounds(case, seed):
    """Where each expert's rows begin, and the end of the last's."""
    rng, experts = random.Random(int(seed) * 7919 + 5), case["experts"]
    likes = [math.exp(2 * case["skew"] * rng.gauss(0, 1)) for _ in range(experts)]
    if case["skew"] > 1 and experts > 3:
        likes[rng.randrange(experts)] = 0.0
    counts = [0] * experts
    if case["m"] <= experts and case["skew"] == 0:       # one token's choices: an expert is chosen once
        for e in rng.sample(range(experts), case["m"]):
            counts[e] = 1
    elif case["m"] <= 4096:
        for e in rng.choices(range(experts), likes, k=case["m"]):
            counts[e] += 1
    else:
        total = sum(likes)
        counts = [int(case["m"] * v / total) for v in likes]
        counts[max(range(experts), key=likes.__getitem__)] += case["m"] - sum(counts)
    out = [0]
    for c in counts:
        out.append(out[-1] + c)
    return out


def _product_inputs(case, seed):
    gen, dtype = _generator(seed), DTYPES[case["dtype"]]
    m, experts, n, k = case["m"] + case["spare"], case["experts"], case["n"], case["k"]

    def draws(rows, cols, std, pad=0):
        t = torch.empty(rows, cols + pad, dtype=dtype, device="cuda")
        step = max(1, (1 << 26) // (cols + pad))
        for at in range(0, rows, step):
            t[at:at + step] = std * torch.randn(min(step, rows - at), cols + pad, generator=gen, device="cuda")
        return t[:, :cols]

    s = {"bounds": _bounds(case, seed), "x": draws(m, k, 1.0, case["pad"]),
         "w": draws(experts * n, k, k ** -0.5).view(experts, n, k)}
    s["offsets"] = torch.tensor(s["bounds"], dtype=torch.int64, device="cuda")
    if case["op"] == "gradients":
        s["dy"] = draws(m, n, 1.0)
    return s


def _shapes(case):
    shapes = []
    for _ in range(case["blocks"]):
        shapes += [(case["inner"], case["width"])] * 2 + [(case["width"], case["inner"]), (case["width"],), (case["inner"],)]
    rng = random.Random(case["shapes"])
    shapes += [(_log_uniform(rng, 1, 20000),) for _ in range(case["odd"])]
    return shapes


def _adamw_inputs(case, seed):
    """One arena for each kind of buffer, and each tensor's views into them."""
    gen, rng, shapes = _generator(seed), random.Random(int(seed)), _shapes(case)
    sizes = [math.prod(shape) for shape in shapes]
    narrow = [case["bits"] == 8 and size >= SMALL for size in sizes]
    align = 1 if case["odd"] else 16

    def places(counts):
        at, out = 1 if case["odd"] else 0, []
        for c in counts:
            out.append(at)
            at += -(-c // align) * align
        return out, max(at, 1)

    def normal(count, std):
        t = torch.empty(count, device="cuda")
        for at in range(0, count, 1 << 26):
            t[at:at + (1 << 26)] = std * torch.randn(min(1 << 26, count - at), generator=gen, device="cuda")
        return t

    def cut(arena, counts, at):
        return [arena[a:a + c] for a, c in zip(at, counts)]

    at, total = places(sizes)
    weights = normal(total, 0.02)
    s = {"step": 1 + rng.randrange(1000), "seed": rng.randrange(1 << 62), "shapes": shapes,
         "param": weights.to(DTYPES[case["dtype"]])}
    params = cut(s["param"], sizes, at)
    masters = [None] * len(sizes)
    if case["master"]:
        s["master"] = weights
        masters = cut(weights, sizes, at)
    # gradients differ by tensor and by column, and half of those behind a closed gate are zero
    grads = normal(total, 1e-3)
    grads *= torch.rand(total, generator=gen, device="cuda") < 0.75
    grads = cut(grads.to(DTYPES[case["grad"]]), sizes, at)
    wide = [0 if n else size for n, size in zip(narrow, sizes)]
    few = [size if n else 0 for n, size in zip(narrow, sizes)]
    blocks = [-(-size // BLOCK) for size in few]
    (at32, total32), (at8, total8), (at_scale, total_scale) = places(wide), places(few), places(blocks)
    s["m"], s["v"] = normal(total32, 3e-4), normal(total32, 1e-3).square_()
    for name, std in (("m8", 50.0), ("r8", 60.0)):
        t = torch.empty(total8, dtype=torch.float8_e4m3fn, device="cuda")
        for a in range(0, total8, 1 << 26):
            part = std * torch.randn(min(1 << 26, total8 - a), generator=gen, device="cuda")
            t[a:a + (1 << 26)] = (part if name == "m8" else part.abs() + 1).clamp_(-255, 255).to(torch.float8_e4m3fn)
        s[name] = t
        s[name + "_scale"] = torch.exp2(torch.randint(-20, -16, (total_scale,), generator=gen, device="cuda").float())
    m32, v32 = cut(s["m"], wide, at32), cut(s["v"], wide, at32)
    m8, r8 = cut(s["m8"], few, at8), cut(s["r8"], few, at8)
    ms, rs = cut(s["m8_scale"], blocks, at_scale), cut(s["r8_scale"], blocks, at_scale)
    s["tensors"] = [(params[i], grads[i], (m8[i], r8[i], ms[i], rs[i]) if narrow[i] else (m32[i], v32[i]), masters[i])
                    for i in range(len(sizes))]
    return s


HYPER = {"rate": 3e-4, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "decay": 0.1}


def _inputs(case, seed):
    if case["op"].startswith("route"):
        return _route_inputs(case, seed)
    return _adamw_inputs(case, seed) if case["op"] == "adamw" else _product_inputs(case, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    dtype = DTYPES[case["dtype"]]
    new = lambda *shape, dtype=dtype: torch.zeros(*shape, dtype=dtype, device="cuda")
    if case["op"] == "route":
        m, top = case["m"], case["top"]
        s["chosen"], s["weights"] = new(m, top, dtype=torch.int32), new(m, top, dtype=torch.float32)
        s["offsets"] = new(case["experts"] + 1, dtype=torch.int64)
        s["order"], s["place"] = new(m * top, dtype=torch.int64), new(m, top, dtype=torch.int64)
    elif case["op"] == "route_backward":
        s["dlogits"] = new(case["m"], case["experts"])
    elif case["op"] == "product":
        s["y"] = new(case["m"] + case["spare"], case["n"])
    elif case["op"] == "gradients":
        s["dx"], s["dw"] = new(case["m"] + case["spare"], case["k"]), new(case["experts"], case["n"], case["k"])
    if own:
        from paper_1705_01626_amd import adamw, experts
        s["experts"], s["adamw"] = experts, adamw
        if case["op"] == "route":
            s["ws"] = experts.new_route_workspace(s["logits"], case["top"])
        elif case["op"] in ("product", "gradients"):
            s["ws"] = experts.new_expert_workspace(s["x"], s["w"], backward=case["op"] == "gradients")
        elif case["op"] == "adamw":
            s["plan"] = adamw.new_plan(s["tensors"])
    torch.cuda.synchronize()
    return s


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _adamw_outputs(s):
    return {name: s[name] for name in ("param", "master", "m", "v", "m8", "r8", "m8_scale", "r8_scale") if name in s}


def _run_own(s):
    case, experts = s["case"], s["experts"]
    if case["op"] == "route":
        experts.zvc_route(s["logits"], s["chosen"], s["weights"], s["offsets"], s["order"], s["place"], s["ws"],
                          normalize=case["normalize"])
        return [s["chosen"], s["weights"], s["offsets"], s["order"], s["place"]]
    if case["op"] == "route_backward":
        experts.zvc_route_backward(s["dweights"], s["logits"], s["chosen"], s["dlogits"], normalize=case["normalize"])
        return s["dlogits"]
    if case["op"] == "product":
        experts.zvc_expert_product(s["x"], s["w"], s["offsets"], s["y"], s["ws"])
        return s["y"]
    if case["op"] == "gradients":
        experts.zvc_expert_gradients(s["dy"], s["x"], s["w"], s["offsets"], s["dx"], s["dw"], s["ws"])
        return [s["dx"], s["dw"]]
    s["adamw"].zvc_adamw(s["plan"], step=s["step"], seed=s["seed"], **HYPER)
    s["step"] += 1
    return _adamw_outputs(s)


# ------------------------------------------------------------------------------- the same in plain torch
def _choose(logits, top):
    """The `top` largest logits of each row, ties to the lowest index; -1 where there is none left."""
    left = torch.where(logits > -math.inf, logits.float(), -math.inf)
    columns = torch.arange(logits.shape[1], dtype=torch.int32, device=logits.device)
    chosen = []
    for _ in range(top):
        best = left.amax(1, keepdim=True)
        at = torch.where(left == best, columns, logits.shape[1]).amin(1, keepdim=True)
        chosen.append(torch.where(best > -math.inf, at, -1))
        left = torch.where(columns == at, -math.inf, left)
    return torch.cat(chosen, 1).to(torch.int32)


def _softmax(logits, live):
    top = torch.where(live, logits, -math.inf).amax(1, keepdim=True)
    e = torch.where(live, torch.exp(logits - torch.where(top > -math.inf, top, 0.0)), 0.0)
    return e / e.sum(1, keepdim=True).clamp(min=1e-30)


def _run_plain(s):
    case = s["case"]
    if case["op"] == "adamw":
        for number in range(len(s["tensors"])):
            _step_plain(s, number)
        s["step"] += 1
        return _adamw_outputs(s)
    if case["op"] in ("product", "gradients"):
        return _product_plain(s)
    logits, top = s["logits"], case["top"]
    live, wide = logits > -math.inf, logits.float()
    if case["op"] == "route":
        chosen = _choose(logits, top)
        there, at = chosen >= 0, chosen.clamp(min=0).long()
        if case["normalize"]:
            weights = _softmax(wide.gather(1, at), there)
        else:
            weights = torch.where(there, _softmax(wide, live).gather(1, at), 0.0)
        flat = chosen.view(-1)
        member = flat[:, None] == torch.arange(case["experts"], dtype=torch.int32, device=flat.device)
        running = member.cumsum(0)
        offsets = torch.zeros(case["experts"] + 1, dtype=torch.int64, device=flat.device)
        offsets[1:] = running[-1].cumsum(0)
        expert = flat.clamp(min=0).long()
        place = torch.where(flat >= 0, offsets[expert] + running.gather(1, expert[:, None])[:, 0] - 1, -1)
        order = torch.full_like(place, -1)
        entries = torch.arange(flat.numel(), device=flat.device)
        # (entries without an expert go behind the last, where nothing is read: one place more than there is)
        order = torch.cat([order, order[:1]]).index_copy_(0, torch.where(place >= 0, place, flat.numel()), entries)[:-1]
        return [chosen, weights, offsets, order, place.view_as(chosen)]
    chosen, dw = s["chosen"], s["dweights"]
    there, at = chosen >= 0, chosen.clamp(min=0).long()
    dw = torch.where(there, dw, 0.0)
    zeros = torch.zeros_like(wide)
    if case["normalize"]:
        w = _softmax(wide.gather(1, at), there)
        grad = w * (dw - (w * dw).sum(1, keepdim=True))
        return zeros.scatter_add_(1, at, grad).to(logits.dtype)
    p = _softmax(wide, live)
    dense = zeros.scatter_add_(1, at, dw)
    return (p * (dense - (p * dense).sum(1, keepdim=True))).to(logits.dtype)


def _product_plain(s):
    bounds, x, w = s["bounds"], s["x"], s["w"]
    for e in range(len(bounds) - 1):
        rows = slice(bounds[e], bounds[e + 1])
        if s["case"]["op"] == "product":
            s["y"][rows] = x[rows].float() @ w[e].float().t()
        else:
            dy = s["dy"][rows].float()
            s["dx"][rows] = dy @ w[e].float()
            s["dw"][e] = dy.t() @ x[rows].float()
    return s["y"] if s["case"]["op"] == "product" else [s["dx"], s["dw"]]


def _random_halves(count, tensor, step, seed, device):
    """Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) under the key `seed`: element i
    takes the 16-bit half i % 8 of counter (i / 8, tensor in the upper word; step), the low half of each word first."""
    word = 0xFFFFFFFF
    c0 = torch.arange(-(-count // 8), dtype=torch.int64, device=device)
    c1, c2, c3 = torch.full_like(c0, tensor), torch.full_like(c0, step & word), torch.full_like(c0, step >> 32 & word)
    k0, k1 = seed & word, seed >> 32 & word
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57            # 64-bit products, modulo 2^64
        c0, c1, c2, c3 = ((b >> 32) & word) ^ c1 ^ k0, b & word, ((a >> 32) & word) ^ c3 ^ k1, a & word
        k0, k1 = (k0 + 0x9E3779B9) & word, (k1 + 0xBB67AE85) & word
    return torch.stack([h for c in (c0, c1, c2, c3) for h in (c & 0xFFFF, c >> 16)], 1).view(-1)[:count].int()


def _widen(codes, scale):
    """The values of 8-bit codes."""
    return codes.float() * scale.repeat_interleave(BLOCK)[:codes.numel()]


def _narrow(value, halves, least):
    """Codes and scales of 32-bit values: the largest of a block comes to lie in [128, 256); rounded up where the random half carries."""
    size = value.abs()
    blocks = torch.nn.functional.pad(torch.where(size < math.inf, size, 0.0), (0, -value.numel() % BLOCK)).view(-1, BLOCK).amax(1)
    exponent = (blocks.view(torch.int32) >> 23).clamp(min=32)
    scale, inverse = ((exponent - 7) << 23).view(torch.float32), ((261 - exponent) << 23).view(torch.float32)
    bits = (size * inverse.repeat_interleave(BLOCK)[:value.numel()] * 2.0 ** -120).view(torch.int32)
    bits = torch.where(size < math.inf, bits, 0x7E << 20)
    codes = torch.minimum((bits + (halves << 4)) >> 20, torch.full_like(bits, 0x7E))
    if least:
        codes = torch.where(size > 0, codes.clamp(min=1), codes)
    codes = codes | (value.view(torch.int32) >> 24 & 0x80)
    return codes.to(torch.uint8).view(torch.float8_e4m3fn), scale


def _step_plain(s, number):
    param, grad, state, master = s["tensors"][number]
    narrow = len(state) == 4
    h = HYPER
    m, v = (_widen(state[0], state[2]), _widen(state[1], state[3]).square_()) if narrow else state
    g = grad.float()
    m = h["beta1"] * m + (1 - h["beta1"]) * g
    v = h["beta2"] * v + (1 - h["beta2"]) * (g * g)
    root = torch.sqrt(v)
    p = (param if master is None else master).float()
    correct1, correct2 = 1 - h["beta1"] ** s["step"], 1 - h["beta2"] ** s["step"]
    p = p * (1 - h["rate"] * h["decay"]) - (h["rate"] / correct1) * (m / (root / math.sqrt(correct2) + h["eps"]))
    if master is not None:
        master.copy_(p)
    param.copy_(p)
    if narrow:
        halves = _random_halves(grad.numel(), number, s["step"], s["seed"], grad.device)
        for i, (value, least) in enumerate(((m, False), (root, True))):
            codes, scale = _narrow(value, halves, least)
            state[i].copy_(codes)
            state[2 + i].copy_(scale)
    else:
        state[0].copy_(m)
        state[1].copy_(v)


# ------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] == "adamw":
        return _adamw_exact(case, s)
    if case["op"] in ("product", "gradients"):
        return _product_exact(case, s)
    return _route_exact(case, s)


def _route_exact(case, s):
    raw = s["logits"].to(torch.float64)
    raw = torch.where(torch.isnan(raw), torch.full_like(raw, -math.inf), raw)
    values, index = torch.sort(raw, dim=1, descending=True, stable=True)
    values, index = values[:, :case["top"]], index[:, :case["top"]]
    there = torch.isfinite(values)
    dead = torch.isneginf(raw).all(1, keepdim=True)
    over = torch.where(dead, torch.zeros_like(raw), raw) if not case["normalize"] else None
    if case["normalize"]:
        w = torch.softmax(torch.where(dead, torch.zeros_like(values), values), 1)
    else:
        w = torch.softmax(over, 1).gather(1, index)
    w = torch.where(there, w, torch.zeros_like(w))
    if case["op"] == "route":
        return [None, w, None, None, None]
    dw = torch.where(there, s["dweights"].to(torch.float64), torch.zeros_like(w))
    out = torch.zeros_like(raw)
    mean = (w * dw).sum(1, keepdim=True)
    if case["normalize"]:
        return out.scatter_(1, index, torch.where(there, w * (dw - mean), torch.zeros_like(w)))
    out = -torch.softmax(over, 1) * mean
    out = out.scatter_add_(1, index, w * dw)
    return torch.where(torch.isneginf(raw), torch.zeros_like(out), out)


def _product_exact(case, s):
    f64 = torch.float64
    rows, n, k = case["m"] + case["spare"], case["n"], case["k"]
    first = torch.zeros(rows, n if case["op"] == "product" else k, dtype=f64, device="cuda")
    dw = None if case["op"] == "product" else torch.empty(case["experts"], n, k, dtype=f64, device="cuda")
    for e, (a, b) in enumerate(zip(s["bounds"], s["bounds"][1:])):
        w, x = s["w"][e].to(f64), s["x"][a:b].to(f64)
        if case["op"] == "product":
            first[a:b] = torch.mm(x, w.T)
        else:
            dy = s["dy"][a:b].to(f64)
            first[a:b] = torch.mm(dy, w)
            dw[e] = torch.mm(dy.T, x)
    return first if dw is None else [first, dw]


def _uniform16(count, tensor, step, seed):
    """The same random halves, with 32-bit multiplications done in 16-bit pieces."""
    mask = (1 << 32) - 1
    group = torch.arange((count + 7) // 8, dtype=torch.int64, device="cuda")

    def product(c, by):
        low, high = c * (by & 0xFFFF), c * (by >> 16)
        middle = (low >> 16) + high
        return middle >> 16, ((middle & 0xFFFF) << 16) | (low & 0xFFFF)

    c = [group, torch.full_like(group, tensor), torch.full_like(group, step & mask), torch.full_like(group, step >> 32 & mask)]
    for r in range(10):
        h0, l0 = product(c[0], 0xD2511F53)
        h1, l1 = product(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ ((seed + 0x9E3779B9 * r) & mask), l1, h0 ^ c[3] ^ (((seed >> 32) + 0xBB67AE85 * r) & mask), l0]
    out = torch.empty(group.numel(), 8, dtype=torch.int64, device="cuda")
    for j in range(8):
        out[:, j] = c[j // 2] >> (16 * (j % 2)) & 0xFFFF
    return out.view(-1)[:count]


def _adamw_exact(case, s):
    f64 = torch.float64
    out = {name: t.to(f64) for name, t in _adamw_outputs(s).items()}
    beta1, beta2, t = HYPER["beta1"], HYPER["beta2"], s["step"]

    def at(name, view):
        """The place in an output of a tensor's view into the arena."""
        start = view.storage_offset()
        return out[name][start:start + view.numel()]

    for number, (param, grad, state, master) in enumerate(s["tensors"]):
        g, count = grad.to(f64), grad.numel()
        old = (param if master is None else master).to(f64)
        if len(state) == 4:
            spread = [sc.to(f64).unsqueeze(1).expand(-1, BLOCK).reshape(-1)[:count] for sc in state[2:]]
            m0, v0 = state[0].to(f64) * spread[0], (state[1].to(f64) * spread[1]) ** 2
        else:
            m0, v0 = state[0].to(f64), state[1].to(f64)
        m1, v1 = torch.lerp(g, m0, beta1), torch.lerp(g ** 2, v0, beta2)
        update = (m1 / (1 - beta1 ** t)) / ((v1 / (1 - beta2 ** t)).sqrt() + HYPER["eps"])
        new = old - HYPER["rate"] * (HYPER["decay"] * old + update)
        at("param", param).copy_(new)
        if master is not None:
            at("master", master).copy_(new)
        if len(state) == 2:
            at("m", state[0]).copy_(m1)
            at("v", state[1]).copy_(v1)
            continue
        chance = _uniform16(count, number, t, s["seed"]).to(f64) / 65536
        for value, name, codes, scale in ((m1, "m8", state[0], state[2]), (v1.sqrt(), "r8", state[1], state[3])):
            size = value.abs()
            padded = torch.zeros(scale.numel() * BLOCK, dtype=f64, device="cuda")
            padded[:count] = size
            most = padded.view(-1, BLOCK).max(1).values
            power = torch.floor(torch.log2(most.clamp(min=2.0 ** -95))) - 7
            units = size / torch.exp2(power).unsqueeze(1).expand(-1, BLOCK).reshape(-1)[:count]
            step = torch.exp2(torch.floor(torch.log2(units.clamp(min=2.0 ** -6))) - 3)
            rounded = torch.floor(units / step + chance) * step
            if name == "r8":
                rounded = torch.where(size > 0, rounded.clamp(min=2.0 ** -9), rounded)
            at(name, codes).copy_(torch.sign(value) * rounded)
    # A scale is a choice and not a number that is computed: a block's largest value is a sum of a few bits each and lies on the
    # border between two scales, to the last bit, more often than chance would have it.
    out["m8_scale"] = out["r8_scale"] = None
    return out


# ------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    w = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "adamw":
        grad, total = 4 if case["grad"] == "fp32" else 2, 0
        for shape in _shapes(case):
            size = math.prod(shape)
            states = 4 * (1 + 4 / BLOCK) if case["bits"] == 8 and size >= SMALL else 16
            total += size * (grad + states + (8 + w if case["master"] else 2 * w))
        return {"bytes": int(total), "flops": 0}
    m, experts = case["m"], case["experts"]
    if case["op"] == "route":
        return {"bytes": m * experts * w + m * case["top"] * 24 + 8 * (experts + 1), "flops": 0}
    if case["op"] == "route_backward":
        return {"bytes": 2 * m * experts * w + 8 * m * case["top"], "flops": 0}
    n, k, bounds = case["n"], case["k"], _bounds(case, 1)
    used = sum(b > a for a, b in zip(bounds, bounds[1:]))
    if case["op"] == "product":
        return {"bytes": w * (m * k + used * n * k + m * n), "flops": 2 * m * n * k}
    return {"bytes": w * (2 * m * k + m * n + used * n * k + experts * n * k), "flops": 4 * m * n * k}
