"""Rotary positions without a GPU: frequencies against the header's formulas, refusals, and the checks of listed threads (dry-run pool)."""
import math

import pytest

import paper_2401_06761_amd as ap


@pytest.mark.parametrize("r", [2, 6, 64, 96, 128, 256])
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "ramp"])
def test_frequencies(r, scaling):
    base, f, L, lo, hi = 10000.0, 8.0, 4096.0, 1.0, 32.0
    if scaling == "base" and r == 2:
        with pytest.raises(ap.AparError):
            ap.Rotary(256, r, base=base, scaling=scaling, factor=f)
        return
    with ap.Rotary(256, r, base=base, scaling=scaling, factor=f, original_len=L, low_turns=lo, high_turns=hi) as rot:
        got = ap.apar_rotary_frequencies(rot.handle)
    assert len(got) == r // 2
    for i, g in enumerate(got):
        b = base * f ** (r / (r - 2)) if scaling == "base" else base
        want = b ** (-2 * i / r)
        if scaling == "linear":
            want /= f
        if scaling == "ramp":
            n = L * want / (2 * math.pi)
            k = min(max((n - lo) / (hi - lo), 0), 1)
            want = k * want + (1 - k) * want / f
        assert abs(g - want) <= 1e-14 * want


@pytest.mark.parametrize("change,status", [
    ({"head_dim": 0}, -1), ({"head_dim": 127}, -1), ({"rotary_dim": 3}, -1), ({"rotary_dim": 0}, -1), ({"rotary_dim": 130}, -1),
    ({"head_dim": 258, "rotary_dim": 258}, -6), ({"layout": 2}, -1), ({"scaling": 4}, -1), ({"base": 0.0}, -1), ({"base": math.inf}, -1),
    ({"base": math.nan}, -1), ({"scaling": 1, "factor": 0.0}, -1), ({"magnitude": 0.0}, -1), ({"magnitude": math.nan}, -1),
    ({"scaling": 3, "original_len": 0.0}, -1), ({"scaling": 3, "low_turns": 32.0, "high_turns": 32.0}, -1), ({"base": 1e-300}, 0)])
def test_configurations_that_are_refused(change, status):
    cfg = ap.AparRotaryConfig(128, 128, 0, 0, 10000.0, 1.0, 4096.0, 1.0, 32.0, 1.0)
    for k, v in change.items():
        setattr(cfg, k, v)
    if status == 0:
        ap.apar_rotary_destroy(ap.apar_rotary_create(cfg))
        return
    with pytest.raises(ap.AparError) as e:
        ap.apar_rotary_create(cfg)
    assert e.value.status == status


def test_null_handles():
    ap.apar_rotary_destroy(None)
    with ap.Pool(4, 2, 128, "bf16", 8, dry_run=True) as pool:
        with pytest.raises(ap.AparError):
            ap.apar_rotate_threads(pool.handle, None, [], None)


def test_listed_threads_are_checked():
    with ap.Pool(4, 2, 128, "bf16", 64, dry_run=True) as pool, ap.Rotary(128) as rot, ap.Rotary(64) as narrow:
        h = pool.handle
        a = ap.apar_thread_create(h)
        b = ap.apar_thread_create(h)
        ap.apar_append_kv(h, a, None, None, 5)

        def status(threads, rotary=rot, **kw):
            try:
                ap.apar_rotate_threads(h, rotary.handle, threads, None, **kw)
                return 0
            except ap.AparError as e:
                return e.status

        assert status([]) == status([a, b, a]) == status([a], m=[5], where=ap.APAR_ROWS_LAST) == status([a, b], m=[0, 7]) == 0
        assert status([a], rotary=narrow) == -1
        assert status([7]) == -2 and status([-1]) == -2
        assert status([a], m=[6], where=ap.APAR_ROWS_LAST) == status([b], where=ap.APAR_ROWS_LAST) == -1
        assert status([a], m=[0], where=ap.APAR_ROWS_LAST) == status([a], m=[-1]) == status([a], where=2) == -1
        assert status([a], n_cand=9) == status([a], n_cand=-1) == status([a], n_cand=2, m=[2]) == -1
        assert status([a], n_cand=2, where=ap.APAR_ROWS_LAST) == -1
        assert status([a, a], m=[2 ** 31 - 6, 1]) == 0 and status([a, b, a], m=[2 ** 30, 1, 2 ** 30]) == -6 and status([a], m=[2 ** 31 - 4]) == -6  # (the last position is 2^31 - 1)
        assert ap.apar_thread_len(h, a) == 5  # (nothing changes)
        with pytest.raises(ValueError):
            ap.apar_rotate_threads(h, rot.handle, [a], None, m=[1, 2])
