"""4-bit pools without a GPU: sizes, books, plans and refusals (dry-run pools)."""
import numpy as np
import pytest

import paper_2401_06761_amd as ap
from apar_workloads import HeadConfig, manual_tree
from oracle import BlockLedger

from harness import blocks_upper_bound, books_equal, check_plan_covers_tables, check_prefill_plan, pool_for, random_forest, replay_trace
from test_few_units import every_row_group_once

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


@pytest.mark.parametrize("group,C", [(16, 5), (16, 8), (13, 5), (11, 7), (9, 8)])
def test_plans_of_threads_with_more_than_64_rows(group, C):
    """Candidate calls of 65 to 128 query rows a thread: plans over random forests and knobs, and along a few steps; other pools refuse them."""
    rng = np.random.default_rng(group * C)
    for seed in range(12):
        parents, segs = random_forest(rng, int(rng.integers(1, 5)), int(rng.integers(3, 80)))
        w = manual_tree(parents, segs, HeadConfig(2 * group, 2, 128, F4), seed=seed)
        with ap.Pool(2 * group, 2, 128, F4, blocks_upper_bound(w) + 400, dry_run=True) as pool:
            if seed % 3:
                ap.apar_set_chunk_blocks(pool.handle, int(rng.choice([1, 2, 5, 64])))
            if seed % 4 == 1:
                ap.apar_set_inline_shared(pool.handle, False)
            live, _ = replay_trace(w, pool, None, dry_run=True)
            for step in range(4):
                ap.apar_decode_attention_spec(pool.handle, None, None, None, None, C, live, None)
                if ap.apar_last_plan_info(pool.handle).n_units // 2 == len(live) * -(-C * group // 16):  # (a unit per slice: a call of few units)
                    every_row_group_once(pool.handle, live, -(-C * group // 16))
                else:
                    check_plan_covers_tables(pool.handle, live, 2, C * group)
                ap.apar_append_kv_batch(pool.handle, live, None, None)
    for dtype in ("bf16", "bf16_fp8kv", "f32"):
        with ap.Pool(16, 1, 128, dtype, 8, dry_run=True) as pool:
            th = ap.apar_thread_create(pool.handle)
            ap.apar_append_kv(pool.handle, th, None, None, 3)
            ap.apar_decode_attention_spec(pool.handle, None, None, None, None, 4, [th], None)
            with pytest.raises(ap.AparError) as e:
                ap.apar_decode_attention_spec(pool.handle, None, None, None, None, 5, [th], None)
            assert e.value.status == -6
