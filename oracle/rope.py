"""Plain form of rotary positions, in float64: pairs of dims as complex numbers."""

from __future__ import annotations

import math

import numpy as np


def frequencies(rotary_dim, base=10000.0, scaling="none", factor=1.0, low=1.0, high=32.0, original_len=0):
    """Radians per position of every pair, one after another."""
    out = []
    pair_at = lambda turns: rotary_dim * math.log(original_len / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
    for i in range(rotary_dim // 2):
        w = base ** (-2.0 * i / rotary_dim)
        if scaling == "linear":
            w /= factor
        elif scaling == "bands":
            turns = original_len * w / (2 * math.pi)
            if turns <= low:
                w /= factor
            elif turns < high:
                m = (turns - low) / (high - low)
                w = m * w + (1 - m) * w / factor
        elif scaling == "ramp":
            start = max(math.floor(pair_at(high)), 0)
            end = min(math.ceil(pair_at(low)), rotary_dim - 1)
            m = min(max((i - start) / max(end - start, 0.001), 0.0), 1.0)
            w = m * w / factor + (1 - m) * w
        out.append(w)
    return np.array(out)


def rotate(x, positions, w, interleaved=False, magnitude=1.0):
    """x [rows, heads, dim] (float64), rotated by positions * w."""
    half = len(w)
    z = magnitude * np.exp(1j * np.asarray(positions, np.float64)[:, None] * w)[:, None, :]
    y = np.array(x, np.float64)
    first, second = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    turned = (y[..., first] + 1j * y[..., second]) * z
    y[..., first], y[..., second] = turned.real, turned.imag
    return y
