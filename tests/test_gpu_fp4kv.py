"""Pools that keep rows in 4 bits (APAR_BF16_FP4KV) against the oracle, through the C ABI (GPU only).

The quantiser: rows of arbitrary bf16 values go in, are read back, and must equal oracle.fp4 bit for bit.  The attention path: rows that the
rounding leaves alone (its own values, tests/test_oracle_fp4.py) go to the library and to the dense oracle alike, and outputs are
held to the bounds of the bf16 pools: an output is rounded once, 2^-9 of it at most half a step of 2^-8, and the probabilities
once; the products of queries and keys are kept to 2^-20 of the largest, which is nothing beside that."""
import numpy as np
import pytest

import paper_2401_06761_amd as ap
from apar_workloads import (HeadConfig, draw_candidate_tree, make_config, manual_tree, mask_rows_from_parents, node_kv, quantise, step_q)
from oracle import BlockLedger, DenseThreads, attend, attend_spec, fp4

from harness import (assert_close, blocks_upper_bound, books_equal, check_plan_covers_tables, nested_wide_tree, pool_for, random_forest,
                     replay_trace, to_dev, to_host)

pytestmark = pytest.mark.gpu
F4 = "bf16_fp4kv"


def torch():
    import torch as t

    return t


def held_rows(w, node):
    k, v = node_kv(w, node)
    return fp4.held(k).astype(np.float32), fp4.held(v).astype(np.float32)


def bf16(rng, shape, scale=1.0):
    return quantise((scale * rng.standard_normal(shape)).astype(np.float32), "bf16")


def built(w, pool, led=None):
    hd = w.heads
    dense = DenseThreads(hd.n_q_heads, hd.n_kv_heads, hd.head_dim)
    live, _ = replay_trace(w, pool, led, dense, kv_of=held_rows)
    return dense, live


def assert_within(got, want, top_v, what):
    """Bounds from the roundings alone: an output is rounded to bf16 once, at most 2^-8 of it; the probabilities p are rounded to
    bf16 before they meet V, at most 2^-8 of each, which moves sum p v by at most 2^-8 sum p |v| <= 2^-8 max|V|.  1 % more for the second
    order and for the logits (2^-20)."""
    assert np.isfinite(got).all(), what
    off = np.abs(got - want) - 1.01 * 2.0 ** -8 * (np.abs(want) + top_v)
    assert off.max() <= 0, f"{what}: {off.max()} beyond the bound, outputs up to {np.abs(want).max()}"


def decode_and_compare(w, pool, dense, live, step=0, call=None):
    q = step_q(w, step, len(live))
    qd = to_dev(q, F4)
    out = torch().full_like(qd, 9.0)
    (call or ap.apar_decode_attention)(pool.handle, qd, live, out)
    torch().cuda.synchronize()
    return assert_close(to_host(out), dense.decode(q, live), F4, w.name)


def run(w, chunk=None, inline=True):
    n, hd = blocks_upper_bound(w), w.heads
    with pool_for(w, n) as pool:
        pool.kv.fill_(0xFF)
        if chunk:
            ap.apar_set_chunk_blocks(pool.handle, chunk)
        if not inline:
            ap.apar_set_inline_shared(pool.handle, False)
        led = BlockLedger(n)
        dense, live = built(w, pool, led)
        books_equal(pool.handle, led)
        decode_and_compare(w, pool, dense, live)
        check_plan_covers_tables(pool.handle, live, hd.n_kv_heads, hd.n_q_heads // hd.n_kv_heads)
        return ap.apar_last_plan_info(pool.handle)


def read_back(pool, thread, n, n_kv):
    ko = torch().empty((n, n_kv, 128), dtype=torch().bfloat16, device="cuda:0")
    vo = torch().empty_like(ko)
    ap.apar_read_kv_rows(pool.handle, thread, 0, n, ko, vo)
    torch().cuda.synchronize()
    return to_host(ko), to_host(vo)


def test_quantiser_matches_the_definition_bit_for_bit():
    """Arbitrary bf16 rows (many magnitudes, groups of zeros, outliers, every bf16 magnitude of a binade), appended in pieces that end
    inside blocks, at block ends and across them; forks that copy a filling block."""
    rng = np.random.default_rng(5)
    L = 16 * 6 + 11
    with ap.Pool(4, 2, 128, F4, 32) as pool:
        ap.apar_set_write_checks(pool.handle, True)
        pool.kv.fill_(0xFF)
        th = ap.apar_thread_create(pool.handle)
        scale = 10.0 ** rng.uniform(-37, 37, (L, 2, 4, 1))
        scale[rng.random(scale.shape) < 0.1] = 0.0
        K = bf16(rng, (L, 2, 4, 32))
        K = quantise((K * scale).astype(np.float32), "bf16").reshape(L, 2, 128)
        V = bf16(rng, (L, 2, 128))
        V[:, :, :64] = (1.0 + np.arange(64) / 128.0) * 2.0 ** rng.integers(-3, 4, (L, 2, 1))  # ties among them
        K[37, 1, 5] = 6.0e4
        pos = 0
        for n in (5, 11, 1, 15, 16, 33, L - 81):
            ap.apar_append_kv(pool.handle, th, to_dev(K[pos:pos + n], F4), to_dev(V[pos:pos + n], F4))
            pos += n
        ko, vo = read_back(pool, th, L, 2)
        assert np.array_equal(ko, fp4.held(K)) and np.array_equal(vo, fp4.held(V))
        kids = ap.apar_fork(pool.handle, th, 2)
        extra = bf16(rng, (7, 2, 128))
        for kid in kids:
            ap.apar_append_kv(pool.handle, kid, to_dev(extra, F4), to_dev(extra, F4))
        for kid in kids:
            k2, v2 = read_back(pool, kid, L + 7, 2)
            assert np.array_equal(k2, fp4.held(np.concatenate([K, extra]))) and np.array_equal(v2, fp4.held(np.concatenate([V, extra])))
        k3, v3 = read_back(pool, th, L, 2)
        assert np.array_equal(k3, ko) and np.array_equal(v3, vo)


def test_special_values_are_held_as_documented():
    rng = np.random.default_rng(6)
    K = bf16(rng, (21, 1, 128))
    K[0, 0, 3], K[1, 0, 40], K[17, 0, 100], K[20, 0, 0] = np.inf, -np.inf, np.nan, 3.38e38
    K[2, 0, :32] = np.nan
    K[3, 0, 32:64] = 1e-39
    K = quantise(np.where(np.isfinite(K), K, 0), "bf16") + np.where(np.isfinite(K), 0, K)
    with ap.Pool(2, 1, 128, F4, 4) as pool:
        th = ap.apar_thread_create(pool.handle)
        ap.apar_append_kv(pool.handle, th, to_dev(K, F4), to_dev(K, F4))
        ko, vo = read_back(pool, th, 21, 1)
        assert np.array_equal(ko, fp4.held(K)) and np.array_equal(vo, fp4.held(K))


def test_every_bf16_value_alone_in_its_group():
    """All finite bf16 values of either sign, each the largest of a group beside values at its ties."""
    bits = np.arange(0, 0x7F80, 7, dtype=np.uint32)
    top = (bits << 16).view(np.float32)
    n = len(top)
    rows = np.zeros((-(-n // 4), 4, 32), dtype=np.float32)
    flat = rows.reshape(-1, 32)
    flat[:n, 0] = top * np.where(np.arange(n) % 2, -1, 1)
    flat[:n, 1:9] = quantise((top[:, None].astype(np.float64) * np.array([0.5, 0.25, 0.75, 0.125, 1 / 3, 5 / 6, 5 / 12, 0.0625])).astype(np.float32), "bf16")
    rows = rows.reshape(-1, 1, 128)
    with ap.Pool(1, 1, 128, F4, len(rows) // 16 + 1) as pool:
        th = ap.apar_thread_create(pool.handle)
        ap.apar_append_kv(pool.handle, th, to_dev(rows, F4), to_dev(-rows, F4))
        ko, vo = read_back(pool, th, len(rows), 1)
    want = fp4.held(rows)
    assert np.array_equal(ko, want) and np.array_equal(vo, -want)


def test_batches_gathers_and_the_last_holder_that_fills_a_shared_block():
    t = torch()
    rng = np.random.default_rng(7)
    with ap.Pool(2, 2, 128, F4, 64) as pool:
        ap.apar_set_write_checks(pool.handle, True)
        pool.kv.fill_(0xFF)
        root = ap.apar_thread_create(pool.handle)
        base = bf16(rng, (13, 2, 128))
        ap.apar_append_kv(pool.handle, root, to_dev(base, F4), to_dev(-base, F4))
        kids = ap.apar_fork(pool.handle, root, 3)
        rows = bf16(rng, (11, 2, 128))
        listed = [kids[0], kids[1], kids[0], root, kids[0], kids[2], root, root, root, kids[1], kids[0]]
        ap.apar_append_kv_batch(pool.handle, listed, to_dev(rows, F4), to_dev(2 * rows, F4))
        src = [10, 3, 3, 0]
        ap.apar_append_kv_gather(pool.handle, [kids[2], root, kids[2], kids[1]], src, to_dev(rows, F4), to_dev(2 * rows, F4))
        own = {th: [rows[i] for i, x in enumerate(listed) if x == th] for th in [root] + kids}
        for th, i in zip([kids[2], root, kids[2], kids[1]], src):
            own[th].append(rows[i])
        for th, extra in own.items():
            k = np.concatenate([base, np.array(extra)])
            v = np.concatenate([-base, 2 * np.array(extra)])
            ko, vo = read_back(pool, th, len(k), 2)
            assert np.array_equal(ko, fp4.held(k)) and np.array_equal(vo, fp4.held(v))


def test_attention_over_rows_off_the_grid():
    rng = np.random.default_rng(8)
    L = 16 * 9 + 6
    with ap.Pool(8, 2, 128, F4, 64) as pool:
        pool.kv.fill_(0xFF)
        th = ap.apar_thread_create(pool.handle)
        K, V = bf16(rng, (L, 2, 128)), bf16(rng, (L, 2, 128))
        ap.apar_append_kv(pool.handle, th, to_dev(K, F4), to_dev(V, F4))
        q = bf16(rng, (1, 8, 128))
        qd = to_dev(q, F4)
        out = torch().empty_like(qd)
        ap.apar_decode_attention(pool.handle, qd, [th], out)
        want = attend(q[0], fp4.held(K), fp4.held(V), 1.0 / np.sqrt(128.0))
        assert_close(to_host(out)[0], want, F4, "rounded rows")
        plain = attend(q[0], K, V, 1.0 / np.sqrt(128.0))
        assert np.abs(plain - want).max() > 4 * np.abs(to_host(out)[0] - want).max()


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 47, 64, 500, 4097])
@pytest.mark.parametrize("n_q,n_kv", [(1, 1), (8, 1), (16, 1), (20, 4)])
def test_one_thread_of_any_length(length, n_q, n_kv):
    w = manual_tree([-1], [length], HeadConfig(n_q, n_kv, 128, F4), seed=length)
    run(w)


@pytest.mark.parametrize("chunk", [1, 2, 8, None])
def test_ragged_trees_every_block_boundary(chunk):
    parents = [-1, 0, 0, 0, 1, 1, 3, 3, 3, -1, -1, 10, 10]
    segs = [1, 15, 16, 17, 1, 33, 16, 15, 2, 1, 47, 1, 130]
    assert run(manual_tree(parents, segs, HeadConfig(4, 4, 128, F4), seed=11), chunk=chunk).n_threads == 9


@pytest.mark.parametrize("name,n_req,scale", [("mha64", 4, 1.0), ("ht256", 6, 1.0), ("gqa1024", 2, 1.0)])
def test_config_shaped_subsets(name, n_req, scale):
    w = make_config(name, n_requests=n_req, data_scale=scale)
    w = type(w)(**{**w.__dict__, "heads": HeadConfig(w.heads.n_q_heads, w.heads.n_kv_heads, 128, F4)})
    run(w)


@pytest.mark.parametrize("inline", [True, False])
@pytest.mark.parametrize("n_q,n_kv", [(2, 2), (8, 2)])
def test_wide_sharing_groups_cut_by_rank_or_standing_alone(n_q, n_kv, inline):
    info = run(nested_wide_tree(HeadConfig(n_q, n_kv, 128, F4), seed=6), inline=inline)
    assert inline or info.n_partial_rows > 0


@pytest.mark.parametrize("n_req,segs,heads", [(1, 9000, (8, 2)), (3, 2500, (32, 8)), (40, 300, (8, 8))])
def test_units_cut_into_slices(n_req, segs, heads):
    parents, lens = [], []
    for r in range(n_req):
        parents += [-1] + [len(parents)] * 3
        lens += [segs + 13 * r, 40, 1, 77]
    run(manual_tree(parents, lens, HeadConfig(*heads, 128, F4), seed=3))


@pytest.mark.parametrize("C,chunk", [(5, None), (3, 2), (8, None), (1, None)])
def test_multi_candidate_step_and_commit(C, chunk):
    t = torch()
    w = manual_tree([-1, 0, 0, 2, 2, -1], [30, 16, 9, 1, 25, 3], HeadConfig(4, 2, 128, F4), seed=9, data_scale=0.7)
    n_blocks = blocks_upper_bound(w) + 8
    with pool_for(w, n_blocks) as pool:
        pool.kv.fill_(0xFF)
        if chunk:
            ap.apar_set_chunk_blocks(pool.handle, chunk)
        led = BlockLedger(n_blocks)
        dense, live = built(w, pool, led)
        n = len(live)
        rng = np.random.default_rng(1)
        for step in range(3):
            q = bf16(rng, (n, C, 4, 128), 0.7)
            ck, cv = (fp4.held(bf16(rng, (n, C, 2, 128), 0.7)).astype(np.float32) for _ in range(2))
            masks = np.stack([mask_rows_from_parents(draw_candidate_tree(rng, C)) for _ in range(n)])
            qd, ckd, cvd = to_dev(q, F4), to_dev(ck, F4), to_dev(cv, F4)
            out = t.empty_like(qd)
            ap.apar_decode_attention_spec(pool.handle, qd, ckd, cvd, t.from_numpy(masks).cuda(), C, live, out)
            assert_close(to_host(out), dense.decode_spec(q, ck, cv, masks, live), F4, f"step {step}")
            accept = np.array([masks[i, int(rng.integers(0, C))] for i in range(n)], dtype=np.uint8)
            ap.apar_commit_candidates(pool.handle, live, ckd, cvd, C, accept)
            led.commit_candidates(live, accept)
            dense.commit_candidates(live, ck, cv, accept)
            books_equal(pool.handle, led)
        decode_and_compare(w, pool, dense, live, step=7)


def test_candidates_that_are_not_finite_stay_with_the_rows_that_see_them():
    """A candidate with infinities or NaN in V (or K) belongs to the rows whose mask names it, whatever shares the wavefront."""
    t = torch()
    rng = np.random.default_rng(12)
    w = manual_tree([-1, 0, 0, 0], [40, 3, 20, 9], HeadConfig(4, 2, 128, F4), seed=2)
    with pool_for(w, blocks_upper_bound(w)) as pool:
        dense, live = built(w, pool)
        n, C = len(live), 4
        q, ck, cv = bf16(rng, (n, C, 4, 128)), bf16(rng, (n, C, 2, 128)), bf16(rng, (n, C, 2, 128))
        masks = np.tile(np.array([1, 3, 5, 9], dtype=np.uint8), (n, 1))  # 1, 2, 3 hang on 0
        cv[0, 1, 0, 7], cv[1, 2, 1, 50], ck[2, 3, 0, 9] = np.inf, np.nan, np.nan
        out = t.empty((n, C, 4, 128), dtype=t.bfloat16, device="cuda:0")
        ap.apar_decode_attention_spec(pool.handle, to_dev(q, F4), to_dev(ck, F4), to_dev(cv, F4), t.from_numpy(masks).cuda(), C, live, out)
        got = to_host(out)
        spoilt = {(0, 1, 0), (1, 2, 1), (2, 3, 0)}  # (thread, candidate, kv head)
        want = dense.decode_spec(q, np.nan_to_num(ck, posinf=0), np.nan_to_num(cv, posinf=0), masks, live)
        for i in range(n):
            for c in range(C):
                for h in range(4):
                    if (i, c, h // 2) not in spoilt:
                        assert_close(got[i, c, h], want[i, c, h], F4, f"{i} {c} {h}")
        assert np.isposinf(got[0, 1, :2, 7]).all() and np.isnan(got[1, 2, 2:, 50]).all() and np.isnan(got[2, 3, :2]).all()


def test_rows_of_others_cannot_spoil_a_row():
    """Queries and cached rows with infinities in one thread, another one on the same prefix: the other's outputs are the oracle's."""
    t = torch()
    rng = np.random.default_rng(13)
    with ap.Pool(4, 1, 128, F4, 32) as pool:
        pool.kv.fill_(0xFF)
        root = ap.apar_thread_create(pool.handle)
        base = fp4.held(bf16(rng, (37, 1, 128))).astype(np.float32)
        ap.apar_append_kv(pool.handle, root, to_dev(base, F4), to_dev(base, F4))
        a, b = ap.apar_fork(pool.handle, root, 2)
        bad = np.full((9, 1, 128), np.inf, dtype=np.float32)
        bad[3], bad[5, 0, ::2] = np.nan, -np.inf
        ap.apar_append_kv(pool.handle, a, to_dev(bad, F4), to_dev(bad, F4))
        more = fp4.held(bf16(rng, (4, 1, 128))).astype(np.float32)
        ap.apar_append_kv(pool.handle, b, to_dev(more, F4), to_dev(more, F4))
        q = bf16(rng, (3, 4, 128))
        q[0, 1, 5], q[0, 2, 6] = np.inf, np.nan
        out = t.empty((3, 4, 128), dtype=t.bfloat16, device="cuda:0")
        ap.apar_decode_attention(pool.handle, to_dev(q, F4), [a, b, root], out)
        got = to_host(out)
        k = np.concatenate([base, more])
        assert_close(got[1], attend(q[1], k, k, 128 ** -0.5), F4, "the thread beside it")
        assert_close(got[2], attend(q[2], base, base, 128 ** -0.5), F4, "the root")


def test_a_query_of_many_magnitudes_keeps_its_small_parts():
    """Queries go into the products as two e4m3 terms per 32 dims: values down to 2^-10 of the group's largest are exact.  One loud dim per
    group that meets zeros in K, the others decide."""
    t = torch()
    rng = np.random.default_rng(14)
    K = fp4.held(bf16(rng, (300, 1, 128)))
    K[:, :, ::32] = 0.0
    K = fp4.held(K).astype(np.float32)
    V = fp4.held(bf16(rng, (300, 1, 128))).astype(np.float32)
    q = bf16(rng, (1, 16, 128), 3.0)
    q[:, :, ::32] = 500.0
    q = quantise(q, "bf16")
    with ap.Pool(16, 1, 128, F4, 32) as pool:
        th = ap.apar_thread_create(pool.handle)
        ap.apar_append_kv(pool.handle, th, to_dev(K, F4), to_dev(V, F4))
        out = t.empty((1, 16, 128), dtype=t.bfloat16, device="cuda:0")
        ap.apar_decode_attention(pool.handle, to_dev(q, F4), [th], out)
        assert_close(to_host(out)[0], attend(q[0], K, V, 128 ** -0.5), F4)


@pytest.mark.parametrize("seed", range(6))
def test_random_forests_decode_spec_prefill_and_fixed(seed):
    t = torch()
    rng = np.random.default_rng(4000 + seed)
    n_kv = int(rng.choice([1, 2, 3]))
    group = int(rng.choice([1, 2, 4, 8, 16]))
    n_q = n_kv * group
    parents, segs = random_forest(rng, int(rng.integers(1, 4)), int(rng.integers(8, 100)))
    w = manual_tree(parents, segs, HeadConfig(n_q, n_kv, 128, F4), seed=seed, data_scale=0.5 if seed % 2 else 1.5)
    n_blocks = blocks_upper_bound(w)
    with pool_for(w, n_blocks) as pool:
        pool.kv.fill_(0xFF)
        chunk = int(rng.choice([0, 0, 1, 3, 7]))
        if chunk:
            ap.apar_set_chunk_blocks(pool.handle, chunk)
        if seed % 3 == 0:
            ap.apar_set_inline_shared(pool.handle, False)
        led = BlockLedger(n_blocks)
        dense, live = built(w, pool, led)
        books_equal(pool.handle, led)
        listed = [live[i] for i in rng.permutation(len(live))]
        listed += listed[:2]  # (duplicates)
        # (assert_close's absolute bound, 2e-2, is for outputs up to about 2.5: one of 5, as values of N(0, 1.5^2) give where a row sees one
        # token, is rounded by up to 2^-6 = 1.6e-2 by itself, and its V with probabilities off by 2^-8 is as far off again)
        top_v = max(np.abs(dense.rows(th)[1]).max() for th in live)
        for call in (ap.apar_decode_attention, ap.apar_decode_attention_fixed):
            q = step_q(w, seed, len(listed))
            out = t.full((len(listed), n_q, 128), 9.0, dtype=t.bfloat16, device="cuda:0")
            call(pool.handle, to_dev(q, F4), listed, out)
            assert_within(to_host(out), dense.decode(q, listed), top_v, "decode")
        n, C = len(listed), int(rng.integers(1, min(8, 64 // group) + 1))
        q = bf16(rng, (n, C, n_q, 128), 0.5)
        ck, cv = bf16(rng, (n, C, n_kv, 128), 0.5), bf16(rng, (n, C, n_kv, 128), 0.5)
        masks = np.stack([mask_rows_from_parents(draw_candidate_tree(rng, C)) for _ in range(n)])
        out = t.empty((n, C, n_q, 128), dtype=t.bfloat16, device="cuda:0")
        ap.apar_decode_attention_spec(pool.handle, to_dev(q, F4), to_dev(ck, F4), to_dev(cv, F4), t.from_numpy(masks).cuda(), C, listed, out)
        assert_within(to_host(out), dense.decode_spec(q, ck, cv, masks, listed), max(top_v, np.abs(cv).max()), "candidates")
        for kernel in (ap.APAR_PREFILL_ROW_TILES, ap.APAR_PREFILL_AUTO):
            m = [int(rng.integers(1, dense.length(th) + 1)) for th in listed]
            qp = bf16(rng, (sum(m), n_q, 128))
            outp = t.empty((sum(m), n_q, 128), dtype=t.bfloat16, device="cuda:0")
            ap.apar_set_prefill_kernel(pool.handle, kernel)
            ap.apar_prefill_attention(pool.handle, to_dev(qp, F4), listed, m, outp)
            assert_within(to_host(outp), dense.prefill(qp, listed, m), top_v, "prefill")


def test_a_loop_of_steps_carries_its_plan():
    """Forks, appends, frees and attention step by step; every step against the oracle."""
    t = torch()
    rng = np.random.default_rng(21)
    n_q, n_kv = 8, 2
    with ap.Pool(n_q, n_kv, 128, F4, 400) as pool:
        ap.apar_set_write_checks(pool.handle, True)
        pool.kv.fill_(0xFF)
        dense = DenseThreads(n_q, n_kv, 128)
        live = []
        for n in (33, 100, 7):
            th = ap.apar_thread_create(pool.handle)
            assert dense.create() == th
            k, v = fp4.held(bf16(rng, (n, n_kv, 128))), fp4.held(bf16(rng, (n, n_kv, 128)))
            ap.apar_append_kv(pool.handle, th, to_dev(k, F4), to_dev(v, F4))
            dense.append(th, k, v)
            live += [th]
        for step in range(24):
            if step % 6 == 2:
                kids = ap.apar_fork(pool.handle, live[step % len(live)], 2)
                assert dense.fork(live[step % len(live)], 2) == kids
                live += kids
            if step % 9 == 8:
                gone = live.pop(1)
                ap.apar_free_thread(pool.handle, gone)
                dense.free(gone)
            k, v = (fp4.held(bf16(rng, (len(live), n_kv, 128))) for _ in range(2))
            ap.apar_append_kv_batch(pool.handle, live, to_dev(k, F4), to_dev(v, F4))
            for i, th in enumerate(live):
                dense.append(th, k[i], v[i])
            q = bf16(rng, (len(live), n_q, 128))
            out = t.empty((len(live), n_q, 128), dtype=t.bfloat16, device="cuda:0")
            ap.apar_decode_attention(pool.handle, to_dev(q, F4), live, out)
            assert_close(to_host(out), dense.decode(q, live), F4, f"step {step}")
        assert ap.apar_plan_counts(pool.handle)[1] > 10


@pytest.mark.parametrize("group", [1, 2, 4, 8, 16])
def test_prompts_and_segments_on_the_matrix_kernel(group):
    """Whole prompts around block, super-block and workgroup borders, and last segments, forced onto the 32x32 kernel."""
    t = torch()
    rng = np.random.default_rng(40 + group)
    n_kv = 2
    lens = [1, 5, 16, 31, 32, 33, 64, 65, 127, 128, 129, 300]
    w = manual_tree([-1] * len(lens) + [len(lens) - 1] * 2, lens + [40, 7], HeadConfig(n_kv * group, n_kv, 128, F4), seed=group)
    with pool_for(w, blocks_upper_bound(w)) as pool:
        pool.kv.fill_(0xFF)
        dense, live = built(w, pool)
        ap.apar_set_prefill_kernel(pool.handle, ap.APAR_PREFILL_MATRIX)
        for m in ([dense.length(th) for th in live], [max(1, dense.length(th) // 3) for th in live], [1] * len(live)):
            q = bf16(rng, (sum(m), n_kv * group, 128))
            out = t.full((sum(m), n_kv * group, 128), 9.0, dtype=t.bfloat16, device="cuda:0")
            ap.apar_prefill_attention(pool.handle, to_dev(q, F4), live, m, out)
            assert ap.apar_last_prefill_kernel(pool.handle) == ap.APAR_PREFILL_MATRIX
            top_v = max(np.abs(dense.rows(th)[1]).max() for th in live)
            assert_within(to_host(out), dense.prefill(q, live, m), top_v, f"group {group}")


@pytest.mark.parametrize("group", [3, 5, 6, 7, 8, 11, 12, 13, 15, 16])
def test_any_group_with_the_most_candidates(group):
    """Groups that divide no tile, and up to eight candidates a thread, 128 query rows.  Refused as on all pools: prefills with groups that do not
    divide a row tile."""
    t = torch()
    rng = np.random.default_rng(5000 + group)
    n_kv = 2
    n_q = n_kv * group
    w = manual_tree([-1, 0, 0, 2, 2, -1, -1, 6], [30, 16, 9, 1, 25, 3, 200, 33], HeadConfig(n_q, n_kv, 128, F4), seed=group, data_scale=0.7)
    with pool_for(w, blocks_upper_bound(w)) as pool:
        pool.kv.fill_(0xFF)
        dense, live = built(w, pool)
        top_v = max(np.abs(dense.rows(th)[1]).max() for th in live)
        n = len(live)
        q = bf16(rng, (n, n_q, 128))
        out = t.full((n, n_q, 128), 9.0, dtype=t.bfloat16, device="cuda:0")
        ap.apar_decode_attention(pool.handle, to_dev(q, F4), live, out)
        assert_within(to_host(out), dense.decode(q, live), top_v, "decode")
        for C in (8, 7, 3, 1):
            q = bf16(rng, (n, C, n_q, 128), 0.7)
            ck, cv = bf16(rng, (n, C, n_kv, 128), 0.7), bf16(rng, (n, C, n_kv, 128), 0.7)
            masks = np.stack([mask_rows_from_parents(draw_candidate_tree(rng, C)) for _ in range(n)])
            out = t.full((n, C, n_q, 128), 9.0, dtype=t.bfloat16, device="cuda:0")
            call = (pool.handle, to_dev(q, F4), to_dev(ck, F4), to_dev(cv, F4), t.from_numpy(masks).cuda(), C, live, out)
            ap.apar_decode_attention_spec(*call)
            assert_within(to_host(out), dense.decode_spec(q, ck, cv, masks, live), max(top_v, np.abs(cv).max()), f"{C} candidates")
        for kernel in (ap.APAR_PREFILL_ROW_TILES, ap.APAR_PREFILL_MATRIX, ap.APAR_PREFILL_AUTO):
            m = [int(rng.integers(1, dense.length(th) + 1)) for th in live]
            q = bf16(rng, (sum(m), n_q, 128))
            out = t.full((sum(m), n_q, 128), 9.0, dtype=t.bfloat16, device="cuda:0")
            ap.apar_set_prefill_kernel(pool.handle, kernel)
            if 16 % group:
                with pytest.raises(ap.AparError) as e:
                    ap.apar_prefill_attention(pool.handle, to_dev(q, F4), live, m, out)
                assert e.value.status == -6
                continue
            ap.apar_prefill_attention(pool.handle, to_dev(q, F4), live, m, out)
            assert_within(to_host(out), dense.prefill(q, live, m), top_v, "prefill")


@pytest.mark.parametrize("group,C,chunk,inline", [(16, 8, None, True), (16, 5, 2, True), (16, 7, 3, False), (11, 8, 1, False), (13, 6, None, False)])
def test_threads_of_more_rows_than_a_wavefront_holds(group, C, chunk, inline):
    """65 to 128 query rows of a thread, in five to eight slices, in units of their own, cut lists and partial results."""
    t = torch()
    rng = np.random.default_rng(group * C)
    parents, segs = random_forest(rng, 2, 40)
    w = manual_tree(parents, segs, HeadConfig(group, 1, 128, F4), seed=C, data_scale=0.7)
    with pool_for(w, blocks_upper_bound(w) + 200) as pool:
        pool.kv.fill_(0xFF)
        if chunk:
            ap.apar_set_chunk_blocks(pool.handle, chunk)
        if not inline:
            ap.apar_set_inline_shared(pool.handle, False)
        dense, live = built(w, pool)
        for step in range(3):  # (the second call carries the first one's plan)
            n = len(live)
            q, ck, cv = bf16(rng, (n, C, group, 128), 0.7), fp4.held(bf16(rng, (n, C, 1, 128), 0.7)), fp4.held(bf16(rng, (n, C, 1, 128), 0.7))
            masks = np.stack([mask_rows_from_parents(draw_candidate_tree(rng, C)) for _ in range(n)])
            out = t.full((n, C, group, 128), 9.0, dtype=t.bfloat16, device="cuda:0")
            ckd, cvd = to_dev(ck, F4), to_dev(cv, F4)
            ap.apar_decode_attention_spec(pool.handle, to_dev(q, F4), ckd, cvd, t.from_numpy(masks).cuda(), C, live, out)
            if chunk:
                check_plan_covers_tables(pool.handle, live, 1, C * group)
            top_v = max(max(np.abs(dense.rows(th)[1]).max() for th in live), np.abs(cv).max())
            assert_within(to_host(out), dense.decode_spec(q, ck, cv, masks, live), top_v, f"step {step}")
            accept = np.array([masks[i, int(rng.integers(0, C))] for i in range(n)], dtype=np.uint8)
            ap.apar_commit_candidates(pool.handle, live, ckd, cvd, C, accept)
            dense.commit_candidates(live, ck, cv, accept)


def test_reads_of_few_and_many_rows():
    """Tables that travel with the arguments and such that do not; first rows inside a block; the smallest reads."""
    t = torch()
    rng = np.random.default_rng(6000)
    n = 16000
    with ap.Pool(1, 1, 128, F4, n // 16 + 8) as pool:
        th = ap.apar_thread_create(pool.handle)
        k, v = bf16(rng, (n, 1, 128)), bf16(rng, (n, 1, 128))
        ap.apar_append_kv(pool.handle, th, to_dev(k, F4), to_dev(v, F4))
        ku, vu = fp4.held(k), fp4.held(v)
        for first, m in ((0, 1), (15, 1), (15, 2), (n - 1, 1), (7, 14368), (15, 14368), (16, 14368), (7, 14369), (3, n - 3), (0, n)):
            ko = t.full((m + 1, 1, 128), 7.0, dtype=t.bfloat16, device="cuda:0")
            vo = ko.clone()
            ap.apar_read_kv_rows(pool.handle, th, first, m, ko[:m], vo[:m])
            assert np.array_equal(to_host(ko[:m]), ku[first:first + m]) and np.array_equal(to_host(vo[:m]), vu[first:first + m]), (first, m)
            assert (ko[m:] == 7.0).all() and (vo[m:] == 7.0).all()
