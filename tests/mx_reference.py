"""The 8-bit entries of a paged pool from their definition, in 64 bits: what the tests of the paged calls over such
pools compare with.  It shares nothing with the kernels: codes are found among all that there are."""
from __future__ import annotations

import torch

MOST = {"e4m3": 448.0, "int8": 127.0}
RANGE = {("e4m3", "f16"): (-15, 7), ("e4m3", "bf16"): (-117, 7), ("int8", "f16"): (-24, 9), ("int8", "bf16"): (-117, 119)}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
# every magnitude that an e4m3 code has, in order: subnormals of 2^-9, then eight a power of two; the last pattern is NaN
E4M3 = [m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1]


def exponents(y, code, dtype):
    """The power of two of each 32 values: the least with which the largest code reaches the largest magnitude."""
    lo, hi = RANGE[code, dtype]
    part, power = torch.frexp(y.abs().amax(-1).double() / MOST[code])
    e = torch.where(part > 0.5, power, power - 1).clamp(lo, hi)
    return torch.where(part == 0, lo, e)


def nearest(z, code):
    """The nearest code's value, ties to the even one; what is past the largest becomes it."""
    z = z.double().clamp(-MOST[code], MOST[code])
    if code == "int8":
        return torch.round(z)
    grid = torch.tensor(E4M3, dtype=torch.float64, device=z.device)
    a = z.abs()
    i = (torch.searchsorted(grid, a, right=True) - 1).clamp(0, len(E4M3) - 2)
    below, above = a - grid[i], grid[i + 1] - a
    i = torch.where((above < below) | ((above == below) & (i % 2 == 1)), i + 1, i)
    return torch.copysign(grid[i], z)


def spacing(z, code):
    """The distance of the codes around a value."""
    if code == "int8":
        return torch.ones_like(z)
    return torch.exp2(torch.floor(torch.log2(z.abs().clamp(2.0 ** -6, 448.0))) - 3)


def encode(y, code, dtype):
    """(codes as values, scale bytes) of finite values [..., d]."""
    blocks = y.double().unflatten(-1, (-1, 32))
    e = exponents(blocks, code, dtype)
    return nearest(blocks * torch.exp2(-e.double())[..., None], code).flatten(-2), (e + 127).to(torch.uint8)


def decode(codes, scales):
    """The values of codes (a tensor of their type, or of their values) and scale bytes, in 64 bits."""
    power = torch.exp2(scales.view(torch.uint8).double() - 127)
    return (codes.double().unflatten(-1, (-1, 32)) * power[..., None]).flatten(-2)
