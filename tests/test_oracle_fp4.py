"""The 4-bit values of oracle.fp4 against the format's definition, and what the GPU tests take from it (CPU)."""
import numpy as np
import pytest

from oracle import fp4


def test_every_value_rounds_to_the_nearest_and_ties_to_the_even_code():
    y = np.arange(0, 6.0 + 1e-9, 1.0 / 64)
    got = fp4.nearest(y)
    for a, g in zip(y, got):
        away = np.abs(fp4.GRID - a)
        best = [i for i in range(8) if away[i] == away.min()]
        assert g == fp4.GRID[best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1]]
    assert np.array_equal(fp4.nearest(-y), -got)
    for tie, want in ((0.25, 0.0), (0.75, 1.0), (1.25, 1.0), (1.75, 2.0), (2.5, 2.0), (3.5, 4.0), (5.0, 4.0)):
        assert fp4.nearest(np.array([tie]))[0] == want


@pytest.mark.parametrize("top,e", [(6.0, 0), (6.0001, 1), (3.0, -1), (3.01, 0), (0.0, 0), (1e-38, -120), (np.inf, 125), (3.3e38, 125)])
def test_scale_is_the_smallest_that_covers_the_group(top, e):
    assert fp4.group_exponent(min(top, fp4.MOST)) == e


def test_groups_are_independent_and_special_values_have_a_place():
    x = np.zeros((2, 128))
    x[0, :32], x[0, 32:64], x[1, 0], x[1, 1] = 5.0, 100.0, np.inf, np.nan
    x[1, 2], x[1, 40], x[1, 41] = -np.inf, -1.0, 0.3
    h = fp4.held(x)
    assert (h[0, :32] == 4.0).all() and (h[0, 32:64] == 96.0).all() and (h[0, 64:] == 0).all()
    assert h[1, 0] == fp4.MOST and h[1, 2] == -fp4.MOST and h[1, 1] == 0 and h[1, 40] == -1.0 and h[1, 41] == 0.25
    assert np.isfinite(h).all()


def test_held_values_are_held_again_as_they_are():
    """Rounding a second time changes nothing: the largest code of a group is above 3 of its scale, or, where it was rounded down to 3, the
    next smaller scale holds twice every code up to 3."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((400, 32)) * 10.0 ** rng.uniform(-30, 30, (400, 1))
    once = fp4.held(x)
    assert np.array_equal(fp4.held(once), once)
    assert np.abs(once - x).max(axis=1).max() > 0
    # off by at most half a step: 1/4 below 2, 1/2 below 4, 1 below 6, of the group's scale
    s = 2.0 ** np.array([fp4.group_exponent(t) for t in np.abs(x).max(axis=1)])[:, None]
    a = np.abs(x) / s
    assert (np.abs(once - x) / s <= np.where(a < 2, 0.25, np.where(a < 4, 0.5, 1.0))).all()
