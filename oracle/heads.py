"""TEST INFRASTRUCTURE ONLY -- norms and rotations of heads by definition, in 64 bits with numpy.

Every function also returns `mag`, for each element the magnitude that an error of the arithmetic is relative to: the length of the
element's pair after the norm, times the factor.
"""

from __future__ import annotations

import math

import numpy as np


def frequencies(rot, base=10000.0, scaling="none", scale=1.0, original=0.0, low=None, high=None):
    """(radians a position of every pair, factor)."""
    if scaling == "base":
        base = base * scale ** (rot / (rot - 2))
    f = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return np.array(f) / scale, 1.0
    if scaling not in ("dimension", "wavelength"):
        return np.array(f), 1.0
    low = low or 1.0
    high = high or (32.0 if scaling == "dimension" else 4.0)
    out = []
    for i, x in enumerate(f):
        if scaling == "wavelength":
            turns = original * x / (2 * math.pi)
            keep = 1.0 if turns >= high else 0.0 if turns <= low else (turns - low) / (high - low)
        else:
            where = [rot / 2 * math.log(original / (2 * math.pi * t)) / math.log(base) for t in (high, low)]
            a, b = max(math.floor(where[0]), 0), min(math.ceil(where[1]), rot - 1)
            keep = 1.0 if i <= a else 0.0 if i >= max(b, a + 0.001) else 1.0 - (i - a) / (b - a)
        out.append(keep * x + (1.0 - keep) * x / scale)
    return np.array(out), (0.1 * math.log(scale) + 1.0 if scaling == "dimension" and scale > 1 else 1.0)


def norm(x, weight, eps, offset):
    """x [n, H, d]; weight [d] or [H, d]"""
    mean = np.zeros(x.shape[:-1])
    for c in range(x.shape[-1]):
        mean = mean + x[..., c] * x[..., c] / x.shape[-1]
    return x / np.sqrt(mean + eps)[..., None] * (weight + offset)


def rotate(x, positions, f, factor, interleaved):
    """(rotated, mag) of x [n, H, d]"""
    x = np.asarray(x, dtype=np.float64)
    y, mag, half = x.copy(), np.abs(x), len(f)
    for i, w in enumerate(f):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        # the angle modulo a turn, in extended precision: far positions lose nothing that matters
        angle = np.asarray(positions, dtype=np.longdouble) * np.longdouble(w)
        c, s = (factor * t(angle).astype(np.float64)[:, None] for t in (np.cos, np.sin))
        a, b = x[..., p], x[..., q]
        y[..., p], y[..., q] = a * c - b * s, a * s + b * c
        mag[..., p] = mag[..., q] = np.hypot(a, b) * abs(factor)
    return y, mag


def heads(x, positions=None, f=None, factor=1.0, interleaved=False, weight=None, eps=1e-6, offset=0.0):
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.asarray(x, dtype=np.float64)
        if weight is not None:
            x = norm(x, np.asarray(weight, dtype=np.float64), eps, offset)
        return rotate(x, positions, f, factor, interleaved) if f is not None else (x, np.abs(x))
