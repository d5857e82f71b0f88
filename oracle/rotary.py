"""Rotary positions in plain numpy: the rotation of rows and the families of frequencies, from the definitions in
include/kvevict.h, in float64.

TEST INFRASTRUCTURE ONLY (see the package docstring).
"""
from __future__ import annotations

import math

import numpy as np


def rotate(x: np.ndarray, pos: np.ndarray, freq: np.ndarray, layout: str, factor: float = 1.0, inverse: bool = False):
    """x [T, heads, d] at positions pos [T] -> rotated rows, and the sums |a c| + |b s| of their elements (the scale of
    rounding errors; the element itself where it is not rotated)."""
    x = np.asarray(x, dtype=np.float64)
    half = len(freq)
    angle = np.asarray(pos, dtype=np.float64)[:, None] * np.asarray(freq, dtype=np.float64)
    c, s = factor * np.cos(angle)[:, None], factor * np.sin(angle)[:, None] * (-1 if inverse else 1)
    i = np.arange(half)
    ia, ib = (i, i + half) if layout == "half" else (2 * i, 2 * i + 1)
    a, b = x[..., ia], x[..., ib]
    out, mag = x.copy(), np.abs(x)
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    mag[..., ia], mag[..., ib] = np.abs(a * c) + np.abs(b * s), np.abs(b * c) + np.abs(a * s)
    return out, mag


def frequencies(family: str, rot_dim: int, base: float, params=()):
    """-> (radians a position [rot_dim / 2], factor)."""
    f = np.array([base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)])
    if family == "plain":
        return f, 1.0
    F = params[0]
    if family == "linear":
        return f / F, 1.0
    if family == "ntk":
        wider = base * F ** (rot_dim / (rot_dim - 2.0))
        return np.array([wider ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)]), 1.0
    out = []
    if family == "yarn":
        _, old, fast, slow = params
        pair_of = lambda turns: rot_dim * math.log(old / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(pair_of(fast)), 0), min(math.ceil(pair_of(slow)), rot_dim - 1)
        for i, x in enumerate(f):
            ramp = min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0)
            out.append(x / F * ramp + x * (1 - ramp))
        return np.array(out), 0.1 * math.log(F) + 1
    _, old, low, high = params
    for x in f:
        wave = 2 * math.pi / x
        if wave < old / high:
            out.append(x)
        elif wave > old / low:
            out.append(x / F)
        else:
            t = (old / wave - low) / (high - low)
            out.append((1 - t) * x / F + t * x)
    return np.array(out), 1.0
