"""Rotary positions from the definition, in float64 (test infrastructure only).

Frequencies and angles are taken in numpy's long double, so that the angle of a position of
2^31 is exact far below float32's step; turned values come out in float64.
"""
from __future__ import annotations

import numpy as np

TWO_PI = np.longdouble("6.283185307179586476925286766559005768")


def frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "plain",
                factor: float = 1.0, original_length: int = 0, fast: float = 0.0,
                slow: float = 0.0, given=None) -> np.ndarray:
    """theta_j of each pair (long double)."""
    j = np.arange(rotary_dim // 2, dtype=np.longdouble)
    b = np.longdouble(base)
    if scaling == "base":
        b = b * np.longdouble(factor) ** (np.longdouble(rotary_dim) / (rotary_dim - 2))
    th = b ** (-2 * j / rotary_dim) if given is None else np.asarray(given, np.longdouble)
    if scaling == "linear":
        th = th / np.longdouble(factor)
    if scaling == "bands":
        n = original_length * np.abs(th) / TWO_PI
        w = np.clip((n - slow) / (np.longdouble(fast) - slow), 0, 1)
        th = th * w + th * (1 - w) / np.longdouble(factor)
    return th


def turn(x, positions, theta, interleaved: bool = False, amplitude: float = 1.0,
         backward: bool = False) -> np.ndarray:
    """x [rows, heads, D] turned by its rows' positions, float64."""
    x = np.asarray(x, np.float64)
    R = 2 * len(theta)
    angle = np.asarray(positions, np.longdouble)[:, None] * theta
    angle = (angle - TWO_PI * np.floor(angle / TWO_PI)).astype(np.float64)[:, None, :]
    a = float(np.float32(amplitude))
    c, s = a * np.cos(angle), a * np.sin(angle)
    if backward:
        s = -s
    first = np.arange(0, R, 2) if interleaved else np.arange(R // 2)
    second = first + 1 if interleaved else first + R // 2
    out = x.copy()
    with np.errstate(invalid="ignore"):
        out[..., first] = x[..., first] * c - x[..., second] * s
        out[..., second] = x[..., second] * c + x[..., first] * s
    return out


def partner_size(x, theta, interleaved: bool = False) -> np.ndarray:
    """|x1| + |x2| of each channel's pair (0 where nothing turns): what an absolute error of
    the cosine and sine is multiplied by."""
    x = np.abs(np.asarray(x, np.float64))
    R = 2 * len(theta)
    first = np.arange(0, R, 2) if interleaved else np.arange(R // 2)
    second = first + 1 if interleaved else first + R // 2
    out = np.zeros_like(x)
    out[..., first] = out[..., second] = x[..., first] + x[..., second]
    return out
