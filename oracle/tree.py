"""Plain form of the attention of drafted tokens, in float64."""

from __future__ import annotations

import numpy as np


def sees(masks, base, rows):
    """Which keys each row of a request sees: all `base` before its rows, and row j if bit j of its mask is set."""
    out = np.zeros((rows, base + rows), bool)
    out[:, :base] = True
    for i in range(rows):
        for j in range(rows):
            out[i, base + j] = (masks[i] >> j) & 1
    return out


def weights(q, k, seen, scale):
    """softmax of scale * q k^T over the keys that are seen; a row that sees none has no weights."""
    s = np.where(seen, (q @ np.where(seen.any(0)[:, None], k, 0.0).T) * scale, -np.inf)
    top = s.max(1, keepdims=True, initial=-np.inf)
    p = np.where(seen, np.exp(s - np.where(np.isfinite(top), top, 0.0)), 0.0)
    total = p.sum(1, keepdims=True)
    return p / np.where(total > 0, total, 1.0)
