"""Rotary positions, a paged cache and attention from their definitions, in 64 bits (test infrastructure only)."""

from __future__ import annotations

import numpy as np

from . import mx4

KV_16, KV_E4M3, KV_NVFP4 = range(3)


def frequencies(rot: int, theta: float, scaling: int = 0, factor: float = 1.0, low: float = 1.0, high: float = 4.0, original: float = 8192.0) -> np.ndarray:
    f = theta ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    if scaling == 1:
        return f / factor
    if scaling == 2:
        out = []
        for x in f:
            turns = original * x / (2 * np.pi)
            s = (turns - low) / (high - low)
            out.append(x if turns >= high else x / factor if turns <= low else x * (s + (1 - s) / factor))
        return np.array(out)
    return f


def angles(n_pos: int, f: np.ndarray, magnitude: float = 1.0) -> np.ndarray:
    """Table [n_pos, rot]: cosines, then sines."""
    a = np.arange(n_pos, dtype=np.float64)[:, None] * f
    return np.concatenate([np.cos(a), np.sin(a)], axis=1) * magnitude


def rotate(x: np.ndarray, table: np.ndarray, positions: np.ndarray, interleaved: bool) -> np.ndarray:
    """x [tokens, heads, D] (fp32) with table fp32 [n_pos, rot]: every product and sum rounded to fp32."""
    x = x.astype(np.float32).copy()
    rot = table.shape[1]
    h = rot // 2
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        c, s = (table[positions, k].astype(np.float32)[:, None] for k in (i, h + i))
        x1, x2 = x[:, :, a].copy(), x[:, :, b].copy()
        x[:, :, a] = x1 * c - x2 * s
        x[:, :, b] = x2 * c + x1 * s
    return x


def _e4m3_nearest(v: np.ndarray) -> np.ndarray:
    """fp32 -> E4M3 bytes, ties to even, 448 at most, NaN 127."""
    m = np.minimum(np.abs(v.astype(np.float64)), 448.0)
    nan = np.isnan(v)
    byte = mx4._nearest(np.where(nan, 0.0, m).ravel(), mx4.E4M3).reshape(v.shape)
    return np.where(nan, 127, byte | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def _e4m3_values(b: np.ndarray) -> np.ndarray:
    v = np.append(mx4.E4M3, np.nan)[b & 127]
    return np.where(b & 128, -v, v)


def stored(y: np.ndarray, fmt: int, factor: np.ndarray | None):
    """fp32 [tokens, heads, D] -> (bytes, scales or None) of a quantised cache."""
    y = y.astype(np.float32)
    if factor is not None:
        with np.errstate(all="ignore"):
            y = y * (np.float32(1) / factor.astype(np.float32))[:, None]
    if fmt == KV_E4M3:
        return _e4m3_nearest(y), None
    t, h, d = y.shape
    codes, scales = mx4.quantize(y.reshape(t * h, d), 1)
    return codes.reshape(t, h, d // 2), scales.reshape(t, h, d // 16)


def held(codes: np.ndarray, scales, fmt: int, factor: np.ndarray | None) -> np.ndarray:
    """What stored() stands for, in 64 bits."""
    if fmt == KV_E4M3:
        v = _e4m3_values(codes)
    else:
        t, h, d = codes.shape
        v = mx4.values(codes.reshape(t * h, d), scales.reshape(t * h, -1), 1).reshape(t, h, 2 * d)
    return v if factor is None else v * factor.astype(np.float64)[:, None]


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float, sees: np.ndarray):
    """One sequence: q [n, Hq, D], k and v [m, H, D], row i sees the first sees[i] keys.  (result, weighted magnitudes sum w |v|, largest score magnitude sum |q| |k|
    scale per row and head, largest |v| seen): what roundings are measured against."""
    n, Hq, D = q.shape
    g = Hq // k.shape[1]
    out, mag, span, big = (np.zeros((n, Hq, D)), np.zeros((n, Hq, D)), np.zeros((n, Hq)), np.zeros((n, Hq)))
    for i in range(n):
        m = int(min(max(sees[i], 0), len(k)))
        if m == 0:
            continue
        for h in range(Hq):
            kk, vv = k[:m, h // g].astype(np.float64), v[:m, h // g].astype(np.float64)
            s = kk @ q[i, h].astype(np.float64) * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h], mag[i, h] = w @ vv, w @ np.abs(vv)
            span[i, h] = (np.abs(kk) @ np.abs(q[i, h].astype(np.float64))).max() * scale
            big[i, h] = np.abs(vv).max()
    return out, mag, span, big


def tolerance(out, mag, span, big, D: int, keys: int, half_step_p: float, half_step: float, base: float = 2.0 ** -4):
    """Bound on an output's error.  Scores: fp32 sums of D exact products, each addition off by 2^-23 of the sum of magnitudes at most, a few more roundings of
    the score itself: delta = (D + 8) 2^-23 span.  A weight is then off by a factor exp(delta), in
    the sum and in the numerator, and by 2^-21 in the exponential; numerators are rounded to 16 bits (half_step_p relative, or 2^-25 where fp16 runs out of exponents,
    against a sum of `1 / base` at least); the sums over keys are fp32; the result is rounded once more (half_step, or the subnormal 2^-25)."""
    delta = (D + 8) * 2.0 ** -23 * span
    rel = 2 * (np.expm1(delta) + 2.0 ** -21) + half_step_p + (keys + 64) * 2.0 ** -23
    return mag * rel[..., None] + (keys * 2.0 ** -25 * base * big)[..., None] + half_step * np.abs(out) * 1.01 + 2.0 ** -25
