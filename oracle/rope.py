"""Norm and rotation of head rows in fp64 (oracle side, test infrastructure).

The paper leaves the inside of a decode module's forward pass open (F_theta); the readings taken are the usual ones: every head
row x[d] of q and k is x * rsqrt(mean x^2 + eps) * weight, and the first 2 n elements turn pair by pair, pair i by the angle
position * radians[i], (a, b) -> (a cos - b sin, a sin + b cos), with the pairs (i, i + n) ("halves") or (2 i, 2 i + 1)
("neighbours").  Angles are taken modulo a turn in exact rational arithmetic on the float64 rates, so that a far position
costs nothing.
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

# 2 pi to 60 digits
_TWO_PI = Fraction(628318530717958647692528676655900576839433879875021164194989, 10 ** 59)


def angles(positions, radians) -> np.ndarray:
    """[T, pairs] angles in [0, 2 pi), float64, from exact products."""
    rates = [Fraction(float(r)) / _TWO_PI for r in radians]
    out = np.zeros((len(positions), len(rates)))
    for t, p in enumerate(positions):
        for i, r in enumerate(rates):
            turns = int(p) * r
            out[t, i] = float((turns - (turns.numerator // turns.denominator)) * _TWO_PI)
    return out


def norm_rotate(x: np.ndarray, positions, radians, pairing: str, weight=None, eps: float = 0.0) -> np.ndarray:
    """x [T, heads, d] float64 -> the same, normed (with a weight) and rotated."""
    y = np.array(x, np.float64)
    if weight is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    n = len(radians)
    if n == 0 or len(y) == 0:
        return y
    phi = angles(positions, radians)[:, None, :]
    a, b = (slice(0, n), slice(n, 2 * n)) if pairing == "halves" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    first, second = y[..., a].copy(), y[..., b].copy()
    y[..., a] = first * np.cos(phi) - second * np.sin(phi)
    y[..., b] = first * np.sin(phi) + second * np.cos(phi)
    return y
