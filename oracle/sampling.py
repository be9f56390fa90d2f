"""A token out of a row of logits (test infrastructure; plain numpy, fp64).

The definition of include/apar.h written out: the row sorted (value descending, index ascending), the three cuts as prefixes, the first kept
token whose cumulated mass exceeds u times the kept mass.  `margin` tells how far the draw was from falling on another token, as a share of
the kept mass: a comparison of tokens means something only where that is more than the roundings of the sums.
"""
from __future__ import annotations

import numpy as np

NONE = -2 ** 31


def draw(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """-> (token, log-probability, margin)"""
    x = np.asarray(x, dtype=np.float64)
    real = np.flatnonzero(x > -np.inf)  # (drops NaN too)
    if real.size == 0:
        return NONE, -np.inf, 1.0
    order = real[np.argsort(-x[real], kind="stable")]
    if not temperature > 0:
        return int(order[0]), 0.0, 1.0
    top = x[order[0]]
    with np.errstate(invalid="ignore"):
        w = np.where(x[order] == top, 1.0, np.exp((x[order] - top) / np.float64(temperature)))
    keep = len(w) if top_k <= 0 else min(int(top_k), len(w))
    margin = 1.0
    if top_p < 1:
        c = np.cumsum(w[:keep])
        goal = max(np.float64(top_p), 0.0) * c[-1]
        keep_p = int(np.searchsorted(c, goal, side="left")) + 1
        keep_p = max(1, min(keep_p, keep))
        margin = min(margin, float(np.abs(c - goal).min() / c[-1]))
        keep = keep_p
    if min_p > 0:
        keep = max(int((w[:keep] == 1.0).sum()), int((w[:keep] >= min(min_p, 1.0)).sum()))
    c = np.cumsum(w[:keep])
    goal = np.float64(u) * c[-1]
    at = min(int(np.searchsorted(c, goal, side="right")), keep - 1)
    margin = min(margin, float(np.abs(c - goal).min() / c[-1]))
    return int(order[at]), float(np.log(w[at] / c[-1])), margin
