"""Plain form of sampling, one row at a time, in float64 with sums in extended precision.

``draw`` returns (token, its share of what is kept, margin): the margin is how far,
relative to the sum concerned, the numbers stay from the borders that decide the token:
the uniform number from the ends of its token's interval, the weight that top-p asks
for from the sums before and after its cut, and a weight from min-p's floor."""

from __future__ import annotations

import numpy as np

LD = np.longdouble


def draw(x, uniform, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    x = np.asarray(x, np.float64)
    x = np.where(np.isnan(x), -np.inf, x) + 0.0
    order = np.argsort(-x, kind="stable")
    top = x[order[0]]
    if top == -np.inf:
        return -1, 0.0, np.inf
    if not temperature > 0:
        return int(order[0]), 1.0, np.inf
    w = np.where(x == top, 1.0, 0.0) if np.isinf(top) else np.exp((x - top) / np.float64(temperature))
    margin = np.inf
    if 0 < top_k < len(x):
        order = order[:top_k]
    if top_p <= 0:
        order = order[:1]
    elif top_p < 1:
        upto = np.cumsum(w[order].astype(LD))
        want = LD(np.float64(top_p)) * upto[-1]
        n = int(np.argmax(upto >= want))
        near = [upto[n] - want] + ([want - upto[n - 1]] if n else [])
        margin = min(margin, float(min(near) / upto[-1]))
        order = order[:n + 1]
    if min_p > 0:
        floor = min(float(np.float64(min_p)), 1.0)
        margin = min([margin] + [abs(float(v - floor)) for v in w[order] if v != 1.0 or floor != 1.0])
        order = order[w[order] >= floor]
    kept = np.sort(order)
    upto = np.cumsum(w[kept].astype(LD))
    at = LD(np.float64(uniform)) * upto[-1]
    i = int(np.argmax(upto > at))
    margin = min(margin, float((upto[i] - at) / upto[-1]))
    if at > 0:            # nothing is below 0, which is 0 of any sum
        margin = min(margin, float((at - (upto[i] - LD(w[kept[i]]))) / upto[-1]))
    return int(kept[i]), float(w[kept[i]] / upto[-1]), margin
