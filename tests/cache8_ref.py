"""A cache held in 8 bits from its definition, in 64 bits on the CPU: a row's
exponent, the nearest codes by search of all codes, and what they stand for."""
from __future__ import annotations

import torch

E4M3, I8 = torch.float8_e4m3fn, torch.int8
LARGEST = {E4M3: 448.0, I8: 127.0}
LEAST, MOST, NAN = -96, 119, -128


def codes_of(dtype):
    """(values, their codes as bytes) in ascending order, finite ones, one zero."""
    if dtype == I8:
        v = torch.arange(-127, 128)
        return v.double(), v.to(torch.int8)
    bits = torch.arange(256).to(torch.uint8)
    v = bits.view(E4M3).double()
    order = [i for i in v.argsort().tolist() if bool(v[i].isfinite()) and int(bits[i]) != 0x80]
    return v[order], bits[order].view(torch.int8)


def hold(x, dtype):
    """Rows (the last axis) of x as (codes as int8 bytes, exponents).  Zeros of either sign
    have the code of +0 here: compare with same_codes."""
    x = x.double()
    finite = x.isfinite()
    top = torch.where(finite, x.abs(), 0.0).amax(-1)
    e = torch.full(top.shape, LEAST)
    for k in range(LEAST + 1, MOST + 1):
        e = torch.where(top > LARGEST[dtype] * 2.0 ** (k - 1), k, e)
    powers = torch.tensor([2.0**k for k in range(LEAST, MOST + 1)], dtype=torch.float64)
    y = torch.where(finite, x, 0.0) / powers[e - LEAST][..., None]
    values, codes = codes_of(dtype)
    hi = torch.searchsorted(values, y.contiguous()).clamp(1, len(values) - 1)
    down, up = y - values[hi - 1], values[hi] - y
    zero = int((values == 0).nonzero())
    even = (hi - 1 - zero) % 2 == 0  # the last bit of the lower one's code is clear
    at = torch.where((down < up) | ((down == up) & even), hi - 1, hi)
    got = codes[at]
    if dtype == E4M3:
        return torch.where(finite, got, 0x7F), e.to(torch.int8)
    whole = finite.all(-1)
    return torch.where(whole[..., None], got, 0), torch.where(whole, e, NAN).to(torch.int8)


def worth(codes, e, dtype):
    """What codes (int8 bytes) with exponents stand for, in 64 bits."""
    powers = torch.tensor([2.0**k for k in range(-128, 128)], dtype=torch.float64)
    two = torch.where(e == NAN, torch.nan, powers[e.long() + 128])
    return codes.view(dtype).double() * two[..., None]


def same_codes(got, want, dtype):
    """Equal bytes, but for the sign of zero (and of a not-a-number)."""
    if dtype == I8:
        return torch.equal(got, want)
    a, b = got.view(torch.uint8).int(), want.view(torch.uint8).int()
    least = torch.where((a & 0x7F == 0) | (a & 0x7F == 0x7F), a & 0x7F, a)
    other = torch.where((b & 0x7F == 0) | (b & 0x7F == 0x7F), b & 0x7F, b)
    return torch.equal(least, other)
