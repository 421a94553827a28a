"""Microscaled matrices in plain NumPy, 64 bits: the block format of the OCP
Microscaling Formats specification 1.0 with 4-bit (E2M1) and 8-bit (E4M3) codes.
Values of a format are listed and searched, not computed bit by bit, so that
nothing is shared with the library's arithmetic."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32
LOWEST = -117          # exponent of the smallest scale
NAN_SCALE = 255


def format_values(bits: int) -> np.ndarray:
    """The value of every code of a format (NaN where a code is none)."""
    if bits == 4:
        half = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    else:
        half = [m / 8 * 2.0 ** -6 for m in range(8)]
        half += [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)]
        half[-1] = math.nan
    return np.array(half + [-v for v in half])


def quantize(A: np.ndarray, bits: int):
    """(codes one a byte, rows x whole blocks; scale bytes, rows x blocks) of a matrix."""
    A = np.asarray(A, dtype=np.float64)
    rows, cols = A.shape
    blocks = -(-cols // BLOCK)
    wide = np.zeros((rows, blocks * BLOCK))
    wide[:, :cols] = A
    table = format_values(bits)
    size = table[:len(table) // 2]
    size = size[np.isfinite(size)]
    emax = 2 if bits == 4 else 8
    codes = np.zeros(wide.shape, dtype=np.uint8)
    scales = np.zeros((rows, blocks), dtype=np.uint8)
    for t in range(rows):
        for b in range(blocks):
            v = wide[t, b * BLOCK:(b + 1) * BLOCK]
            if not np.all(np.isfinite(v)):
                scales[t, b] = NAN_SCALE
                continue
            m = float(np.max(np.abs(v)))
            e = LOWEST if m == 0 else max(math.frexp(m)[1] - 1 - emax, LOWEST)
            scales[t, b] = e + 127
            a = np.abs(v) / 2.0 ** e
            hi = np.minimum(np.searchsorted(size, a), len(size) - 1)
            lo = np.maximum(hi - 1, 0)
            up, down = size[hi] - a, a - size[lo]
            near = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
            codes[t, b * BLOCK:(b + 1) * BLOCK] = near + np.where(np.signbit(v), len(table) // 2, 0)
    return codes, scales


def pack(codes: np.ndarray, scales: np.ndarray, bits: int):
    """Code rows and scale rows as the library lays them out (smallest pitches)."""
    if bits == 4:
        codes = codes[:, 0::2] | (codes[:, 1::2] << 4)
    wide = np.zeros((scales.shape[0], -(-scales.shape[1] // 4) * 4), dtype=np.uint8)
    wide[:, :scales.shape[1]] = scales
    return np.ascontiguousarray(codes), wide


def unpack(codes: np.ndarray, cols: int, bits: int) -> np.ndarray:
    """Codes one a byte, rows x whole blocks, of the library's code rows."""
    n = -(-cols // BLOCK) * BLOCK
    if bits == 8:
        return codes[:, :n]
    both = np.empty((codes.shape[0], codes.shape[1] * 2), dtype=np.uint8)
    both[:, 0::2] = codes & 15
    both[:, 1::2] = codes >> 4
    return both[:, :n]


def values(codes: np.ndarray, scales: np.ndarray, cols: int, bits: int) -> np.ndarray:
    """The matrix (fp64) that codes (one a byte) and scale bytes stand for."""
    v = format_values(bits)[codes]
    s = np.where(scales == NAN_SCALE, math.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v * np.repeat(s, BLOCK, axis=1)[:, :v.shape[1]])[:, :cols]
