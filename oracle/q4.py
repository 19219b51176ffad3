"""4-bit cache rows (oracle; test infrastructure only).

A block of 32 values with largest magnitude a is scaled by 2^e, e the smallest integer in
[-127, 125] with a <= 7 * 2^e; every value becomes the nearest of +-{0, .5, 1, 1.5, 2, 3, 4, 6}
to x / 2^e, ties to the even index, above 6 to 6.  A block with an infinity or a NaN is NaN.
"""
from __future__ import annotations

import numpy as np

from .attention import bf16_bits_to_f64

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def encode(bits):
    """bf16 bits [..., d] -> (codes uint8 [..., d], scale bytes uint8 [..., d / 32])."""
    bits = np.asarray(bits, np.uint16)
    flat = bits.reshape(-1, BLOCK)
    codes, scales = np.zeros(flat.shape, np.uint8), np.zeros(len(flat), np.uint8)
    limits = np.ldexp(7.0, np.arange(-127, 125))       # past the last one e is 125
    for i in range(0, len(flat), 1 << 15):
        x = bf16_bits_to_f64(flat[i:i + (1 << 15)])
        good = np.all(np.isfinite(x), axis=1)
        x = np.where(good[:, None], x, 0.0)
        top = np.abs(x).max(1)
        e = np.searchsorted(limits, top, side="left") - 127   # the first limit not below the magnitude
        u = np.minimum(np.abs(x) / np.ldexp(1.0, e)[:, None], 6.0)
        below = np.searchsorted(GRID, u, side="right") - 1
        above = np.minimum(below + 1, 7)
        to_below, to_above = u - GRID[below], GRID[above] - u
        index = np.where((to_above < to_below) | ((to_above == to_below) & (below % 2 == 1)), above, below)
        codes[i:i + (1 << 15)] = np.where(good[:, None], index + 8 * np.signbit(x), 0)
        scales[i:i + (1 << 15)] = np.where(good, e + 127, 255)
    return codes.reshape(bits.shape), scales.reshape(bits.shape[:-1] + (-1,))


def decode(codes, scales):
    """The values (float64) of unpacked codes [..., d] under scale bytes [..., d / 32]."""
    codes = np.asarray(codes)
    value = np.where(codes < 8, 1.0, -1.0) * GRID[codes % 8]
    scale = np.where(np.asarray(scales) == 255, np.nan, np.ldexp(1.0, np.asarray(scales, np.int64) - 127))
    return (value.reshape(scale.shape + (BLOCK,)) * scale[..., None]).reshape(codes.shape)


def rounded(bits):
    """The values that 4-bit rows made of bf16 bits stand for."""
    return decode(*encode(bits))


def pack(codes):
    """Codes [..., d] -> bytes [..., d / 2], the even element in the low half."""
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).astype(np.uint8)


def unpack(packed):
    out = np.empty(packed.shape[:-1] + (2 * packed.shape[-1],), np.uint8)
    out[..., 0::2] = packed & 15
    out[..., 1::2] = packed >> 4
    return out
