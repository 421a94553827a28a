"""Matrices in 8 bits with an fp32 scale for each block of 128 columns, dropout and embeddings in plain NumPy,
64 bits.  Codes are searched in the list of E4M3's values, random words are Python integers: nothing is shared
with the library's arithmetic."""
from __future__ import annotations

import math

import numpy as np

from oracle.mx import format_values

BLOCK = 128


def quantize(A: np.ndarray, block_rows: int):
    """(codes, rows x whole blocks; scales fp32, blocks x groups of rows) of a matrix."""
    A = np.asarray(A, dtype=np.float64)
    rows, cols = A.shape
    blocks, groups = -(-cols // BLOCK), -(-rows // block_rows)
    wide = np.zeros((rows, blocks * BLOCK))
    wide[:, :cols] = A
    size = format_values(8)[:127]
    codes = np.zeros(wide.shape, dtype=np.uint8)
    scales = np.zeros((blocks, groups), dtype=np.float32)
    for b in range(blocks):
        for g in range(groups):
            at = np.s_[g * block_rows:(g + 1) * block_rows, b * BLOCK:(b + 1) * BLOCK]
            v = wide[at]
            if not np.all(np.isfinite(v)):
                scales[b, g] = math.nan
                continue
            m = max(float(np.max(np.abs(v))), 2.0 ** -100)
            scales[b, g] = np.float32(m / 448.0)
            u = float(np.float32(448.0 / m))
            a = (np.abs(v) * u).astype(np.float32).astype(np.float64)
            hi = np.minimum(np.searchsorted(size, a), len(size) - 1)
            lo = np.maximum(hi - 1, 0)
            up, down = size[hi] - a, a - size[lo]
            near = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
            codes[at] = near + np.where(np.signbit(v), 128, 0)
    return codes, scales


def values(codes: np.ndarray, scales: np.ndarray, cols: int, block_rows: int) -> np.ndarray:
    """The matrix (fp64) that codes and scales stand for."""
    v = format_values(8)[codes]
    i = np.arange(codes.shape[0]) // block_rows
    k = np.arange(codes.shape[1]) // BLOCK
    return (v * scales.astype(np.float64)[k[None, :], i[:, None]])[:, :cols]


_MASK = (1 << 64) - 1


def word(seed: int, number: int) -> int:
    """Output `number` of the SplitMix64 generator seeded with `seed`."""
    z = (seed + (number + 1) * 0x9E3779B97F4A7C15) & _MASK
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & _MASK
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & _MASK
    return z ^ (z >> 31)


def kept(q: int, r: int, p: float, seed: int, draw: int, first_row: int) -> np.ndarray:
    """Which elements of rows first_row .. first_row + q - 1 dropout keeps."""
    key = word(seed, 10 << 56 | draw)
    least = round(p * 2 ** 32)
    out = np.zeros((q, r), dtype=bool)
    for t in range(q):
        for c in range(0, r, 2):
            w = word(key, (first_row + t) * ((r + 1) // 2) + c // 2)
            out[t, c] = (w & 0xFFFFFFFF) >= least
            if c + 1 < r:
                out[t, c + 1] = (w >> 32) >= least
    return out


def embed(E: np.ndarray, tok: np.ndarray, scale: float, skip: int) -> np.ndarray:
    out = np.full((len(tok), E.shape[1]), math.nan)
    for i, t in enumerate(tok):
        if 0 <= t < len(E):
            out[i] = 0.0 if t == skip else scale * E[t]
    return out


def embed_grad(G: np.ndarray, tok: np.ndarray, vocab: int, skip: int):
    """(sums, sums of magnitudes, number of terms) for every row of the table."""
    total, size, count = np.zeros((vocab, G.shape[1])), np.zeros((vocab, G.shape[1])), np.zeros(vocab, dtype=np.int64)
    for i, t in enumerate(tok):
        if t != skip and 0 <= t < vocab:
            total[t] += G[i]
            size[t] += np.abs(G[i])
            count[t] += 1
    return total, size, count
