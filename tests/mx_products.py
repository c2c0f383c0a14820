"""Products of microscaled operands whose float32 sums are exact, so that an output is right to the bit or wrong.

A value is a multiple of half its scale, a product of a quarter of both; where the magnitudes of all products of an output
add up to less than 2^24 of the smallest such unit, every partial sum is a float32, in any order."""
import numpy as np
import torch

import mx_reference as R


def operand(rng, rows, d, binades):
    """A random matrix in the 4-bit form with scales of 2^-binades to 2^binades: all codes; a zero row and a zero block
    among them, pad bytes that must not matter."""
    codes = rng.integers(0, 16, (rows, d))
    b = rng.integers(127 - binades, 128 + binades, (rows, d // 32))
    if rows > 3:
        codes[1] = 0
        codes[2, :32] = 8
    q, s = R.pack(codes, b)
    s[:, d // 32:] = 255
    return torch.from_numpy(q), torch.from_numpy(s)


def binades(d):
    """What keeps d products' magnitudes within 2^24 units: their mean is about 9 times the scales', a unit 4^-(1 + binades)."""
    return 2 if d <= 4096 else 1 if d <= 16384 else 0


def values(q, s, device):
    """(values float64, the smallest half of a scale)"""
    codes, b = R.unpack(q.cpu().numpy(), s.cpu().numpy())
    return torch.from_numpy(R.values(codes, b)).to(device), 0.5 * 2.0 ** (float(b.min()) - 127)


def expected(xq, xs, wq, ws, device="cpu"):
    """x W^T in float64, having asserted that float32 holds every partial sum."""
    (x, ux), (w, uw) = values(xq, xs, device), values(wq, ws, device)
    assert float((x.abs() @ w.abs().T).max()) < 2.0 ** 24 * ux * uw, "the sums are not exact: other operands"
    return x @ w.T


def check(y, want):
    """y is the exact product, rounded once where it has 16 bits."""
    want = want.to(y.device).float().to(y.dtype)
    assert torch.equal(y, want), f"{int((y != want).sum())} of {y.numel()} outputs differ"
