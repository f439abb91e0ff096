"""Caches held in 4 or 8 bits and rotary positions from their definitions, in float64 on the CPU. Test infrastructure only."""
import math

import numpy as np

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])  # by code
E4M3 = np.array([m / 8 * 2.0**-6 if e == 0 else (1 + m / 8) * 2.0**(e - 7) for e in range(16) for m in range(8)])[:127]  # 127: NaN
LARGEST = {4: 1.75 * 2**2, 8: 1.75 * 2**8}  # no value of a block lies above this times its scale


def grid(bits):
    return E2M1 if bits == 4 else E4M3


def quantise(x, bits):
    """x [..., d] -> codes [..., d] (one an element, sign and magnitude), scale bytes [..., d / 32]."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    whole = np.isfinite(blocks).all(-1)
    top = np.abs(np.where(whole[..., None], blocks, 0)).max(-1)
    e = np.full(top.shape, 16)
    some = top[top > LARGEST[bits] * 2.0**(16 - 127)]
    lo, hi = (int(np.floor(np.log2(x / LARGEST[bits]))) + 127 for x in (some.min(), some.max())) if some.size else (0, 0)
    for b in range(max(17, lo), min(254, hi + 2) + 1):  # the smallest power of two that is large enough
        e = np.where(top > LARGEST[bits] * 2.0**(e - 127), b, e)
    y = np.where(whole[..., None], blocks / 2.0**(e[..., None] - 127), 0.0)
    g, a = grid(bits), np.abs(y)
    hi = np.clip(np.searchsorted(g, a), 0, len(g) - 1)  # the first element not below
    lo = np.maximum(hi - 1, 0)
    below, above = a - g[lo], g[hi] - a
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    code = np.where(a >= g[-1], len(g) - 1, code)
    code = code + (np.signbit(y) & whole[..., None]) * (8 if bits == 4 else 128)
    return code.reshape(x.shape).astype(np.uint8), np.where(whole, e, 255).astype(np.uint8)


def packed(codes, bits):
    """Codes as they lie in memory."""
    return codes if bits == 8 else codes[..., 0::2] | codes[..., 1::2] << 4


def values(codes, scales, bits):
    """What codes (one an element) and scales stand for."""
    g, sign = grid(bits), 8 if bits == 4 else 128
    x = g[np.minimum(codes & (sign - 1), len(g) - 1)] * np.where(codes & sign, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0**(scales.astype(np.float64) - 127))
    return x * np.repeat(s, 32, -1)


def rotate(x, positions, inv_freq, axis, neighbours, inverse=False):
    """x [B,N,H,d], positions [axes,B,N] -> the rotated x, angles as exact products in the precision of Python's integers and fractions."""
    from fractions import Fraction
    B, N, H, d = x.shape
    n = len(inv_freq)
    pi = Fraction(31415926535897932384626433832795028841971693993751058209749445923, 10**64)
    c, s = np.empty((B, N, n)), np.empty((B, N, n))
    for b in range(B):
        for i in range(N):
            for p in range(n):
                a = int(positions[axis[p]][b][i]) * Fraction(float(inv_freq[p]))
                a -= 2 * pi * round(a / (2 * pi))
                c[b, i, p], s[b, i, p] = math.cos(a), math.sin(a)
    if inverse:
        s = -s
    first = np.arange(n) * (2 if neighbours else 1)
    second = first + (1 if neighbours else n)
    y = np.array(x, np.float64)
    x1, x2 = x[..., first], x[..., second]
    y[..., first] = x1 * c[:, :, None] - x2 * s[:, :, None]
    y[..., second] = x1 * s[:, :, None] + x2 * c[:, :, None]
    return y
