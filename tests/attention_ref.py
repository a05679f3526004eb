"""The client's attention operators from their definitions, in 64 bits on the
CPU: what the GPU tests compare with, and the error bounds that follow from the
kernels' types."""
from __future__ import annotations

import math

import torch

P = 2**31 - 1
# unit roundoff of one rounding to the type: 2^-(bits of the significand)
ROUND = {torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11, torch.float32: 2.0**-24}


def lift(x: torch.Tensor, scale: float = 1.0, p: int = P) -> torch.Tensor:
    """Values of floats, or of field elements as centred residues times scale."""
    if x.dtype != torch.int32:
        return x.double()
    x = x.long()
    return torch.where(x > p // 2, x - p, x).double() * scale


def embed(x: torch.Tensor, p: int = P) -> torch.Tensor:
    """Integers as field elements (int32)."""
    return torch.where(x < 0, x + p, x).to(torch.int32)


def frequencies(rot, base=10000.0, scaling=None, factor=1.0, original_len=0.0, slow=1.0, fast=32.0):
    if scaling == "base":
        base = base * factor ** (rot / (rot - 2))
    f = [base ** (-2 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "parts":
        keep = [min(1.0, max(0.0, (original_len * x / (2 * math.pi) - slow) / (fast - slow))) for x in f]
        f = [x / factor * (1 - k) + x * k for x, k in zip(f, keep)]
    return torch.tensor(f, dtype=torch.float64), 0.1 * math.log(factor) + 1 if scaling == "parts" else 1.0


def rotate(x, rows, layout):
    """x: T x H x D (64 bits); rows: T x rot of the table."""
    rot = rows.shape[1]
    c, s = rows[:, None, :rot // 2].double(), rows[:, None, rot // 2:].double()
    y = x.clone()
    i = torch.arange(rot // 2)
    a, b = (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def entries(pool, table_row, n):
    """kv_heads x n x dim of one sequence."""
    page = pool.shape[2]
    j = torch.arange(n)
    return pool[table_row.long()[j // page], :, j % page].transpose(0, 1).double()


class Attention:
    """o (T x heads x dim), lse, w, and the bounds of their errors."""

    def __init__(self, q, K, V, table, lens, q_start, scale=None, w_in=None, out_dtype=None):
        T, H, D = q.shape
        hk, page = K.shape[1], K.shape[2]
        grp = H // hk
        scale = D**-0.5 if scale is None else scale
        S, cap = table.shape[0], table.shape[1] * page
        self.o = torch.zeros((T, H, D), dtype=torch.float64)
        self.o_err = torch.zeros_like(self.o)
        self.lse = torch.full((T, H), -math.inf, dtype=torch.float64)
        self.lse_err = torch.zeros_like(self.lse)
        self.w = torch.zeros((S, hk, cap), dtype=torch.float64)
        self.w_err = torch.zeros_like(self.w)
        self.covered = torch.zeros(T, dtype=torch.bool)
        u, uo = ROUND[q.dtype], ROUND[out_dtype or q.dtype]
        tiny = 2.0**-25 if q.dtype == torch.float16 else 0.0  # spacing of the smallest half-precision weights
        for s in range(S):
            n, a, b = int(lens[s]), int(q_start[s]), int(q_start[s + 1])
            c = b - a
            self.covered[a:b] = True
            k, v = entries(K, table[s], n), entries(V, table[s], n)
            if w_in is not None:
                self.w[s, :, :max(0, n - c)] = w_in[s, :, :max(0, n - c)].double()
            for i in range(c):
                see = n - c + i + 1
                if see <= 0:
                    continue
                qi = q[a + i].double().view(hk, grp, D)
                kk, vv = k[:, :see], v[:, :see]
                x = qi @ kk.transpose(1, 2) * scale
                # each product is exact in 32 bits, sums of D of them are not
                dx = (D + 8) * 2.0**-24 * (qi.abs() @ kk.abs().transpose(1, 2) * abs(scale)).nan_to_num(0, 0, 0).amax()
                p = torch.softmax(x, -1)
                self.o[a + i] = (p @ vv).reshape(H, D)
                av = vv.abs().nan_to_num(0, 0, 0)
                self.o_err[a + i] = ((2 * u + 4 * dx + 2.0**-18) * (p @ av) + see * tiny * av.amax()
                                     ).reshape(H, D) + uo * self.o[a + i].abs()
                self.lse[a + i] = torch.logsumexp(x, -1).reshape(H)
                self.lse_err[a + i] = 2 * dx + 2.0**-20 * (1 + self.lse[a + i].abs().nan_to_num(0, 0, 0))
                self.w[s, :, :see] += p.sum(1)
                # (and what is below the smallest normal number of 32 bits may be lost)
                self.w_err[s, :, :see] += (4 * dx + 2.0**-18) * p.sum(1) + grp * 2.0**-126
            self.w_err[s] += 2.0**-22 * self.w[s].abs()


def evict(w, n, budget, recent, sinks):
    """Kept indices of one row of n weights (a list of floats), from the definition."""
    if n <= budget:
        return list(range(n))
    fixed = set(range(sinks)) | set(range(n - recent, n))
    others = [i for i in range(n) if i not in fixed]
    others.sort(key=lambda i: (1, 0.0, i) if math.isnan(w[i]) else (0, -w[i], i))
    return sorted(fixed | set(others[:budget - len(fixed)]))


def lay_out(lens, page, seed, spare=1):
    """A table of pages scattered over a pool, and the pool's page count."""
    g = torch.Generator().manual_seed(seed)
    used = [max(1, -(-n // page)) for n in lens]
    order = torch.randperm(sum(used) + spare, generator=g).tolist()
    table = torch.full((len(lens), max(used)), -7, dtype=torch.int32)  # beyond the used pages: nothing valid
    at = 0
    for s, u in enumerate(used):
        table[s, :u] = torch.tensor(order[at:at + u], dtype=torch.int32)
        at += u
    return table, sum(used) + spare


def starts(new):
    return torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32)
