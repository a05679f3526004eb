"""The client's norms, gated activation and sampling from their definitions, in 64
bits on the CPU."""
from __future__ import annotations

import math
from fractions import Fraction

import torch

from tests import attention_ref as ref

ROUND = ref.ROUND


def norm(v, weight, bias, kind, eps):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    v = v / (v.square().mean(-1, keepdim=True) + eps).sqrt()
    if weight is not None:
        v = v * weight.double()
    return v if bias is None else v + bias.double()


def block(x, residual, before, after, gate, scale):
    """(before(h), h) of doubles; before, after: (weight, bias, kind, eps) or None."""
    h = torch.zeros_like(residual if residual is not None else x) if residual is None else residual
    if x is not None:
        t = norm(x, *after) if after is not None else x
        if gate is not None:
            t = t * gate.double()
        h = h + scale * t
    return (norm(h, *before) if before is not None else h), h


def activation(g, act):
    if act == "silu":
        return g / (1 + torch.exp(-g))
    if act == "gelu":
        return g * 0.5 * torch.special.erfc(-g / math.sqrt(2))
    if act == "gelu_tanh":
        # (1 + tanh y) / 2 = 1 / (1 + exp(-2 y)): 1 + tanh y itself is all rounding where y is far below zero
        return g / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g**3)))
    return torch.where(g > 0, g, torch.where(g.isnan(), g, 0.0))


def token(x, u, t, k, p, least):
    """(token, its probability among the kept ones) of a row of doubles."""
    n = len(x)
    x = [-math.inf if math.isnan(v) else v for v in x.tolist()]
    top = max(x)
    if top == -math.inf:
        return -1, 0.0
    if not t > 0:
        return x.index(top), 1.0
    order = sorted(range(n), key=lambda i: (-x[i], i))

    def w(i):
        if x[i] == top:
            return 1.0
        return 0.0 if x[i] == -math.inf or top == math.inf else math.exp((x[i] - top) / t)

    if 0 < k < n:
        order = order[:k]
    if p < 1:
        # (the product is not rounded: 0.9 in 64 bits is above 0.9, so 72 of 80 alike are less than 0.9 of them)
        need, sum_, kept = Fraction(p) * Fraction(math.fsum(w(i) for i in order)), 0.0, 0
        for i in order:
            if kept and sum_ >= need:
                break
            sum_ += w(i)
            kept += 1
        order = order[:kept]
    kept = sorted(i for i in order if w(i) > 0 and not w(i) < min(least, 1.0))
    total, sum_ = math.fsum(w(i) for i in kept), 0.0
    u = min(max(0.0 if math.isnan(u) else u, 0.0), 1 - 2.0**-24)
    for i in kept:
        sum_ += w(i)
        if sum_ > u * total:
            break
    return i, w(i) / total
