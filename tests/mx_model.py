"""Microscaled matrices in NumPy, exactly: what the device operators are compared
with."""

from __future__ import annotations

import numpy as np

BLOCK = 32
FP4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
# E4M3: 2^-9 times the mantissa below the first exponent, then 2^(e - 7) (1 + m / 8); code 127 is NaN.
FP8 = np.array([m * 2.0 ** -9 if e == 0 else 2.0 ** (e - 7) * (1 + m / 8) for e in range(16) for m in range(8)][:127])


def grid(bits):
    return FP4 if bits == 4 else FP8


def stride(cols):
    return -(-cols // 512) * 16


def scale_bytes(v, bits):
    """Scale byte of every block of v [R, C] (float64): the smallest from 0 on whose
    power of two brings the largest magnitude to the type's largest value."""
    blocks = np.abs(v.reshape(v.shape[0], -1, BLOCK))
    out = np.full(blocks.shape[:2], 255, dtype=np.uint8)
    finite = np.isfinite(blocks).all(-1)
    top = np.where(finite, blocks.max(-1, where=np.isfinite(blocks), initial=0.0), 0.0)
    fraction, e = np.frexp(top / grid(bits)[-1])  # quotient in [1/2, 1) 2^e; exact comparison below
    e = e + 127 - 2
    for _ in range(3):
        e = np.where(top > grid(bits)[-1] * np.ldexp(1.0, e - 127), e + 1, e)
    out[finite] = np.clip(np.where(top == 0, 0, e), 0, 254)[finite]
    return out


def round_to_grid(x, bits):
    """Codes of the nearest grid values, ties to the even code; |x| within the grid."""
    g = grid(bits)
    size = np.abs(x)
    above = np.clip(np.searchsorted(g, size, side="left"), 1, len(g) - 1)
    below = above - 1
    d = (size - g[below]) - (g[above] - size)  # exact for fp32 inputs over powers of two
    code = np.where(d < 0, below, np.where(d > 0, above, np.where(below % 2 == 0, below, above)))
    code = np.where(size == g[above], above, code)
    return (code | (np.signbit(x).astype(int) << (3 if bits == 4 else 7))).astype(np.uint8)


def quantize(v, bits):
    """Codes (one byte each, FP4 unpacked) [R, C] and scale bytes [R, C / 32]."""
    s = scale_bytes(v, bits)
    wide = np.repeat(s, BLOCK, axis=1)
    x = np.where(wide == 255, 0.0, np.ldexp(np.where(np.isfinite(v), v, 0.0), 127 - wide.astype(int)))
    return round_to_grid(x, bits), s


def pack(codes):
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def unpack(packed):
    return np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[0], -1)


def values(codes, scales, bits):
    """float64 values of unpacked codes under scale bytes [R, C / 32]."""
    g = np.append(grid(bits), np.nan) if bits == 8 else grid(bits)
    sign = codes >> (3 if bits == 4 else 7)
    v = g[codes & (7 if bits == 4 else 127)] * np.where(sign == 1, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))
    return v * np.repeat(s, BLOCK, axis=1)


def half_step(x, bits):
    """Half of the grid's step at |x| (the larger one at a border), as a rounding may be off."""
    size = np.minimum(np.abs(x), grid(bits)[-1])
    least = 0 if bits == 4 else -6  # exponent of the first normal value
    _, e = np.frexp(size)
    return np.ldexp(1.0, np.maximum(e - 1, least) - (1 if bits == 4 else 3)) / 2


def check_rounded(codes, scales, v, bits, rel):
    """codes [R, C] and scales [R, C / 32] are v rounded, v known to a relative `rel`:
    the scale fits a largest magnitude within `rel` of the exact one, and an element is at
    most half a step plus that away."""
    top = np.abs(v.reshape(v.shape[0], -1, BLOCK)).max(-1)
    x = np.ldexp(1.0, scales.astype(int) - 127)
    most = grid(bits)[-1]
    assert np.all(top * (1 - rel) <= most * x)
    assert np.all((most * x / 2 < top * (1 + rel)) | (scales == 0))
    exact = v / np.repeat(x, BLOCK, axis=1)
    got = values(codes, np.full_like(scales, 127), bits)
    off = np.abs(got - exact) - half_step(np.maximum(np.abs(got), np.abs(exact)), bits) - rel * np.abs(exact)
    assert np.all(off <= 0), (float(off.max()), np.unravel_index(off.argmax(), off.shape))
