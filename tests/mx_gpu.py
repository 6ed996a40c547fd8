"""Microscaled matrices between the device and NumPy, for the GPU tests."""

from __future__ import annotations

import numpy as np
import torch

import mx_model as mm


def to_device(codes, scales, bits, padding=0xFF):
    """A device matrix of unpacked codes [R, C] and scale bytes [R, C / 32]; the padding
    of the scales holds NaN scales."""
    rows, cols = codes.shape
    c = torch.from_numpy(np.ascontiguousarray(mm.pack(codes) if bits == 4 else codes)).cuda()
    s = np.full((rows, mm.stride(cols)), padding, dtype=np.uint8)
    s[:, :cols // 32] = scales
    return (c if bits == 4 else c.view(torch.float8_e4m3fn)), torch.from_numpy(s).cuda().view(torch.float8_e8m0fnu)


def room(rows, cols, bits):
    """A device matrix whose bytes are all 0xA5."""
    c = torch.full((rows, cols // 2 if bits == 4 else cols), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((rows, mm.stride(cols)), 0xA5, dtype=torch.uint8, device="cuda")
    return (c if bits == 4 else c.view(torch.float8_e4m3fn)), s.view(torch.float8_e8m0fnu)


def to_host(codes, scales, bits):
    """Unpacked codes, scale bytes and the padding behind them."""
    c = codes.view(torch.uint8).cpu().numpy()
    s = scales.view(torch.uint8).cpu().numpy()
    c = mm.unpack(c) if bits == 4 else c
    return c, s[:, :c.shape[1] // 32], s[:, c.shape[1] // 32:]


def random_matrix(rng, rows, cols, bits, low=117, high=137):
    """Unpacked codes without NaN and scale bytes in [low, high]."""
    codes = rng.integers(0, 16 if bits == 4 else 256, (rows, cols)).astype(np.uint8)
    if bits == 8:
        codes[(codes & 127) == 127] = 0
    return codes, rng.integers(low, high + 1, (rows, cols // 32)).astype(np.uint8)
