"""Microscaled 4-bit floating point from its definition, in 64 bits (test infrastructure only).

E2M1 values 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign bit; block scales E8M0 (MXFP4, 32 columns) or E4M3 (NVFP4, 16 columns).
"""

from __future__ import annotations

import numpy as np

BLOCK = {0: 32, 1: 16}
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def _e4m3(byte: int) -> float:
    e, m = byte >> 3 & 15, byte & 7
    return m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)


E4M3 = np.array([_e4m3(b) for b in range(127)])                 # 0 .. 448, ascending


def scale_values(scales: np.ndarray, fmt: int) -> np.ndarray:
    if fmt == 0:
        return np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return np.where(scales == 127, np.nan, np.append(E4M3, np.nan)[np.minimum(scales, 127)])


def values(codes: np.ndarray, scales: np.ndarray, fmt: int) -> np.ndarray:
    rows, half = codes.shape
    c = np.empty((rows, 2 * half))
    for i, nib in enumerate((codes & 15, codes >> 4)):
        c[:, i::2] = np.where(nib & 8, -1.0, 1.0) * E2M1[nib & 7]
    return c * np.repeat(scale_values(scales, fmt), BLOCK[fmt], axis=1)


def _nearest(v: np.ndarray, grid: np.ndarray) -> np.ndarray:
    """Index of the nearest grid value (v >= 0 in 64 bits, few enough bits that differences are exact); ties to the even index."""
    hi = np.minimum(np.searchsorted(grid, v), len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    dl, dh = np.abs(v - grid[lo]), np.abs(grid[hi] - v)
    return np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)


def quantize(y: np.ndarray, fmt: int):
    """y float32 [rows, K] -> codes, scales.  What the definition rounds to fp32 (amax / 6) is rounded here too."""
    rows, K = y.shape
    B = BLOCK[fmt]
    b = y.astype(np.float32).reshape(rows, K // B, B)
    bad = ~np.isfinite(b).all(axis=2)
    b = np.where(bad[..., None], np.float32(0), b)
    top = np.abs(b).max(axis=2)
    if fmt == 0:
        e = np.frexp(top.astype(np.float64))[1] - 1                    # floor(log2 top)
        byte = np.where(top == 0, 0, np.maximum(e - 2 + 127, 0))
    else:
        byte = _nearest(np.minimum((top / np.float32(6)).astype(np.float64), 448.0), E4M3)
    s = scale_values(byte, fmt)[..., None]
    # |y| against code * scale, both exact in 64 bits: the nearest multiple is the code of the exact quotient
    m = np.abs(b.astype(np.float64))
    lo = np.zeros(b.shape, dtype=np.int64)
    for i in range(1, 8):
        mid = (E2M1[i - 1] + E2M1[i]) / 2 * s
        lo += ((m > mid) | ((m == mid) & (i % 2 == 0))) & (s > 0)
    code = (lo | (np.signbit(b) << 3)).astype(np.uint8).reshape(rows, K)
    code[np.repeat(bad, B, axis=1)] = 0
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8), np.where(bad, 255 if fmt == 0 else 127, byte).astype(np.uint8)


def matmul(xc, xs, wc, ws, fmt: int, alpha: float = 1.0) -> np.ndarray:
    return alpha * (values(xc, xs, fmt) @ values(wc, ws, fmt).T)


def magnitude(xc, xs, wc, ws, fmt: int, alpha: float = 1.0) -> np.ndarray:
    """|X| |W|^T: what the roundings of a sum are measured against."""
    return abs(alpha) * (np.abs(values(xc, xs, fmt)) @ np.abs(values(wc, ws, fmt)).T)
