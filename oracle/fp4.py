"""What a pool that keeps rows in 4 bits holds (test infrastructure; plain numpy).

The definition is the library header's: the values of a row of a kv head, K and V each, in groups of 32 consecutive ones.  A group's
scale is s = 2^e with the smallest e for which max|x| / s <= 6, no less than -120 and no more than 125 (e = 0 for a group of
zeros); a value is held as the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 times s, of two equally near ones the one whose place in
that list is even, with its sign.  Infinities, and whatever is beyond 6 * 2^125, count as 6 * 2^125, NaN as 0.
Attention over such a pool is dense.attend over these values.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
MOST = 6.0 * 2.0 ** 125


def group_exponent(top: float) -> int:
    if not top > 0.0:
        return 0
    e = -120
    while e < 125 and top > 6.0 * 2.0 ** e:
        e += 1
    return e


def nearest(y: np.ndarray) -> np.ndarray:
    """|y| <= 6 -> the nearest magnitude of the grid, by comparing with all eight."""
    d = np.abs(np.abs(y)[..., None] - GRID)
    # two equally near ones are neighbours: the even place wins
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    return GRID[order[np.argmin(d[..., order], axis=-1)]] * np.where(np.signbit(y), -1.0, 1.0)


def held(x: np.ndarray) -> np.ndarray:
    """[..., multiple of 32] -> the values the pool keeps, fp64."""
    x = np.array(x, dtype=np.float64)
    x[np.isnan(x)] = 0.0
    x = np.clip(x, -MOST, MOST)
    g = x.reshape(-1, 32)
    top = np.abs(g).max(axis=1)
    e = np.arange(-120, 126)[np.searchsorted(6.0 * 2.0 ** np.arange(-120.0, 126.0), top, side="left")]
    e = np.where(top > 0.0, e, 0).astype(np.float64)[:, None]
    return (nearest(g / 2.0 ** e) * 2.0 ** e).reshape(x.shape)
