"""fp64 NumPy oracle of the norms with rotation and of the cache of pages in 8 bits.

Written from the definitions; nothing here is shared with the library.
"""
from __future__ import annotations

import math

import numpy as np


def rates(pairs, theta=10000.0, shared=True, factor=1.0, trained=4096.0, slow=1.0, fast=32.0, axes=()):
    """Radians per position step of every pair: those of the given axes are slowed by up to `factor`."""
    P, out = sum(pairs), []
    for a, count in enumerate(pairs):
        for i in range(count):
            rate = theta ** (-(len(out) / P) if shared else -(i / count))
            if a in axes:
                keep = min(1.0, max(0.0, (trained * rate / (2 * math.pi) - slow) / (fast - slow)))
                rate *= keep + (1.0 - keep) / factor
            out.append((a, rate))
    return out


def turn(x, positions, pairs, halves=True, inverse=False, amplitude=1.0, **spectrum):
    """x [..., n, d], positions [axes, n] -> the turned copy."""
    x = np.asarray(x, dtype=np.float64)
    y, P = x.copy(), sum(pairs)
    for p, (a, rate) in enumerate(rates(pairs, **spectrum)):
        angle = np.asarray(positions[a], dtype=np.float64) * rate * (-1.0 if inverse else 1.0)
        u, v = (p, p + P) if halves else (2 * p, 2 * p + 1)
        y[..., u] = amplitude * (x[..., u] * np.cos(angle) - x[..., v] * np.sin(angle))
        y[..., v] = amplitude * (x[..., u] * np.sin(angle) + x[..., v] * np.cos(angle))
    return y


def norm(x, eps):
    """Rows at unit mean square, and the factors that brought them there."""
    x = np.asarray(x, dtype=np.float64)
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return x * r, r


def norm_turn(x, weight=None, eps=None, positions=None, pairs=None, **how):
    """[..., heads, n, d] -> normalised (eps given), weighted ([d] or [heads, d]) and turned (pairs given)."""
    y = norm(x, eps)[0] if eps is not None else np.asarray(x, dtype=np.float64)
    if weight is not None:
        y = y * (weight[:, None] if weight.ndim == 2 else weight)
    return turn(y, positions, pairs, **how) if pairs else y


def norm_turn_gradient(x, dy, weight=None, eps=None, positions=None, pairs=None, **how):
    """dX, and the gradient of every row's weights before it is summed, [..., heads, n, d]."""
    g = turn(dy, positions, pairs, inverse=True, **how) if pairs else np.asarray(dy, dtype=np.float64)
    if eps is None:
        return g, None
    u, r = norm(x, eps)
    h = g if weight is None else g * (weight[:, None] if weight.ndim == 2 else weight)
    return r * (h - u * (h * u).mean(-1, keepdims=True)), g * u


def e4m3_values():
    """What the codes 0 .. 255 stand for: sign, 4 bits of exponent (bias 7), 3 of mantissa; 127 and 255 are NaN."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = (math.nan if c & 127 == 127 else v) * (-1.0 if c & 128 else 1.0)
    return out


def quantise(y):
    """Rows y -> codes' values and scales, in 64 bits from the fp32 definition of the scale."""
    y = np.asarray(y, dtype=np.float64)
    bad = ~np.isfinite(y).all(-1)
    y = np.where(bad[..., None], 0.0, y)
    scale = np.maximum(np.abs(y).max(-1) * float(np.float32(1.0) / np.float32(448.0)), 2.0 ** -126)
    grid = np.sort(e4m3_values()[:127])
    x = np.abs(y) / scale[..., None]
    above = np.clip(np.searchsorted(grid, x), 1, 126)
    low, high = grid[above - 1], grid[above]
    nearer = np.where(x - low < high - x, low, high)
    even = np.where((above - 1) % 2 == 0, low, high)
    value = np.where(x - low == high - x, even, nearer)
    value[bad], scale[bad] = 0.0, np.nan
    return np.copysign(value, y), scale
