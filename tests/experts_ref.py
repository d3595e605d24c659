"""The router and the experts' products written from their formulas in 64 bits (include/zvc_experts.h), and how far a result in
32-bit sums may lie from them.  Shares no code with the GPU path."""
import math

import torch

from tests.ffn_ref import F64, SUM, rounded

# relative: exp in 32 bits, which with an argument of down to -100 loses 100 x 2^-24 where it is the short one, sums of 64 terms in a lane and of 16 lanes, a division
EXP = 2.0 ** -16
LEAST = 2.0 ** -120           # what is smaller may be 0


def starts(offsets, m):
    """Where each expert's rows begin and the end of the last, with what the header says of offsets that are out of order."""
    out, most = [], 0
    for v in offsets:
        most = max(most, min(max(int(v), 0), m))
        out.append(most)
    return out


def choose(logits, top):
    """Lists of each token's experts, by falling logit and rising number; -1 where none is left."""
    out = []
    for row in logits.double().tolist():
        live = [e for e, v in enumerate(row) if not math.isnan(v) and v != -math.inf]
        live.sort(key=lambda e: (-row[e], e))
        out.append((live + [-1] * top)[:top])
    return out


def softmax(row, over):
    """exp(row) over its sum over `over`, as a dict."""
    if not over:
        return {}
    most = max(row[e] for e in over)
    terms = {e: math.exp(row[e] - most) for e in over}
    total = math.fsum(terms.values())
    return {e: t / total for e, t in terms.items()}


def route(logits, top, normalize):
    """chosen, weights, offsets, order, place as lists."""
    chosen, rows = choose(logits, top), logits.double().tolist()
    experts = logits.shape[1]
    weights = []
    for picked, row in zip(chosen, rows):
        live = [e for e, v in enumerate(row) if not math.isnan(v) and v != -math.inf]
        w = softmax(row, [e for e in picked if e >= 0] if normalize else live)
        weights.append([w.get(e, 0.0) for e in picked])
    entries = [[] for _ in range(experts)]
    for i, e in enumerate(e for picked in chosen for e in picked):
        if e >= 0:
            entries[e].append(i)
    offsets = [0]
    for e in entries:
        offsets.append(offsets[-1] + len(e))
    order = [i for e in entries for i in e]
    place = [-1] * (len(chosen) * top)
    for row, i in enumerate(order):
        place[i] = row
    order += [-1] * (len(place) - len(order))
    return chosen, weights, offsets, order, place


def route_backward(dweights, logits, chosen, normalize):
    """(value, bound) of the logits' gradient."""
    out = torch.zeros(logits.shape, dtype=F64)
    bound = torch.zeros(logits.shape, dtype=F64)
    for t, (row, picked, dw) in enumerate(zip(logits.double().tolist(), chosen, dweights.double().tolist())):
        live = [e for e, v in enumerate(row) if not math.isnan(v) and v != -math.inf]
        slots = [(e, d) for e, d in zip(picked, dw) if 0 <= e < len(row)]
        if normalize:
            most = max((row[e] for e, _ in slots if e in live), default=0.0)
            terms = [(e, d, math.exp(row[e] - most) if e in live else 0.0) for e, d in slots]
            total = math.fsum(v for _, _, v in terms) or 1.0
            mean = math.fsum(v / total * d for _, d, v in terms)
            size = math.fsum(v / total * abs(d) for _, d, v in terms)
            for e, d, v in terms:
                out[t, e] += v / total * (d - mean)
                bound[t, e] += v / total * (abs(d) + size) * 2 * EXP
        else:
            p = softmax(row, live)
            mean = math.fsum(p.get(e, 0.0) * d for e, d in slots)
            size = math.fsum(p.get(e, 0.0) * abs(d) for e, d in slots)
            for e in live:
                out[t, e] = -p[e] * mean
                bound[t, e] = p[e] * size * 2 * EXP
            for e, d in slots:
                if e in p:
                    out[t, e] += p[e] * d
                    bound[t, e] += p[e] * abs(d) * 2 * EXP
    return out, bound + rounded(out.abs() + bound, logits.dtype) + LEAST


def product(x, w, offsets, before):
    """(value, bound) of y, with `before` where there is no row."""
    y, bound = before.to(F64).clone(), torch.zeros(before.shape, dtype=F64, device=before.device)
    at = starts(offsets, x.shape[0])
    for e in range(w.shape[0]):
        rows = slice(at[e], at[e + 1])
        a, b = x[rows].to(F64), w[e].to(F64)
        y[rows] = a @ b.t()
        sums = x.shape[1] * SUM * (a.abs() @ b.abs().t())
        bound[rows] = sums + rounded(y[rows].abs() + sums, x.dtype)
    return y, bound


def gradients(dy, x, w, offsets, before):
    """[(value, bound)] of dx, with `before` where there is no row, and of dw."""
    dx, dx_bound = before.to(F64).clone(), torch.zeros(before.shape, dtype=F64, device=before.device)
    dw, dw_bound = (torch.zeros(w.shape, dtype=F64, device=w.device) for _ in range(2))
    at = starts(offsets, x.shape[0])
    for e in range(w.shape[0]):
        rows = slice(at[e], at[e + 1])
        g, a, b = dy[rows].to(F64), x[rows].to(F64), w[e].to(F64)
        dx[rows], dw[e] = g @ b, g.t() @ a
        sums = w.shape[1] * SUM * (g.abs() @ b.abs())
        dx_bound[rows] = sums + rounded(dx[rows].abs() + sums, x.dtype)
        sums = g.shape[0] * SUM * (g.abs().t() @ a.abs())
        dw_bound[e] = sums + rounded(dw[e].abs() + sums, x.dtype)
    return [(dx, dx_bound), (dw, dw_bound)]
