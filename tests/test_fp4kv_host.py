"""4-bit pools without a GPU: sizes, books, plans and refusals (dry-run pools)."""
import numpy as np
import pytest

import paper_2401_06761_amd as ap
from apar_workloads import HeadConfig, manual_tree
from oracle import BlockLedger

from harness import blocks_upper_bound, books_equal, check_plan_covers_tables, check_prefill_plan, pool_for, random_forest, replay_trace

F4 = "bf16_fp4kv"


def test_block_takes_2176_bytes_per_head():
    with ap.Pool(32, 8, 128, F4, 10, dry_run=True) as pool:
        assert ap.apar_pool_stats(pool.handle).block_bytes == 8 * ap.APAR_FP4_TILE_BYTES == pool.block_bytes == 8 * 16 * 136


@pytest.mark.parametrize("d,hq,hkv,status", [(64, 8, 2, -6), (256, 8, 2, -6), (128, 34, 2, -6), (128, 7, 2, -1)])
def test_shapes_that_are_refused(d, hq, hkv, status):
    with pytest.raises(ap.AparError) as e:
        ap.Pool(hq, hkv, d, F4, 10, dry_run=True)
    assert e.value.status == status


def test_buffers_that_are_too_small_are_refused():
    cfg = ap.AparPoolConfig(8, 2, 128, 16, ap.APAR_BF16_FP4KV, 10, 4, 0.0)
    for at, n in ((4096, 4 * 2 * 2176 - 1), (4096 + 64, 4 * 2 * 2176)):  # (the address is not looked at before the checks)
        with pytest.raises(ap.AparError) as e:
            ap.apar_pool_create(cfg, at, n)
        assert e.value.status == -1


@pytest.mark.parametrize("seed", range(8))
def test_books_and_plans(seed):
    rng = np.random.default_rng(seed)
    n_kv, group = int(rng.choice([1, 2, 8])), int(rng.choice([1, 2, 4, 8, 16]))
    parents, segs = random_forest(rng, int(rng.integers(1, 4)), int(rng.integers(8, 160)))
    w = manual_tree(parents, segs, HeadConfig(n_kv * group, n_kv, 128, F4), seed=seed)
    n = blocks_upper_bound(w)
    with pool_for(w, n, dry_run=True) as pool:
        led = BlockLedger(n)
        live, _ = replay_trace(w, pool, led, dry_run=True)
        books_equal(pool.handle, led)
        if seed % 2:
            ap.apar_set_chunk_blocks(pool.handle, int(rng.integers(1, 9)))
            ap.apar_set_matrix_units(pool.handle, 1, 1)  # (ignored: no matrix units)
        ap.apar_decode_attention(pool.handle, None, live, None)
        check_plan_covers_tables(pool.handle, live, n_kv, group)
        info = ap.apar_last_plan_info(pool.handle)
        assert info.algorithmic_bytes == info.unique_tokens * n_kv * 136 + 2 * len(live) * n_kv * group * 128 * 2
        if seed % 2:
            wgs = np.array(ap.apar_last_plan_export(pool.handle, ap.APAR_PLAN_WORKGROUPS)).reshape(-1, 32)
            assert all(x & 255 in (1, 2) for x in wgs[:, 3])
        m = [int(rng.integers(1, led.len[t] + 1)) for t in live]
        ap.apar_prefill_attention(pool.handle, None, live, m, None)
        check_prefill_plan(pool.handle, live, m, group)
