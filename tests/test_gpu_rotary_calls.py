"""Calls of the rotary operators that a user may make with tensors of other shapes and strides (GPU only)."""
import numpy as np
import pytest

import paper_2401_06761_amd as ap

from test_gpu_rotary import check, draw, torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 256])
def test_heads_that_are_not_the_rotarys_are_refused(d):
    t = torch()
    rng = np.random.default_rng(d)
    with ap.Rotary(128) as rot, ap.Pool(8, 8, 128, "bf16", 4) as pool:
        th = [ap.apar_thread_create(pool.handle) for _ in range(3)]
        p = t.arange(3, dtype=t.int32, device="cuda")
        qk = draw(rng, (3, 16, d), "bf16")
        was = qk.clone()
        for q, k in ((qk[:, :8], qk[:, 8:]), (qk[:, :8].contiguous(), qk[:, 8:].contiguous())):
            for call in (lambda: ap.apar_rotate_rows(rot.handle, p, q, k), lambda: ap.apar_rotate_rows(rot.handle, p, None, k),
                         lambda: ap.apar_rotate_threads(pool.handle, rot.handle, th, q, k)):
                with pytest.raises(ap.AparError) as e:
                    call()
                assert e.value.status == -1
        assert t.equal(qk, was)


@pytest.mark.parametrize("n_cand,of", [(1, 4), (1, 1), (4, 4)])
def test_candidates_out_of_a_wider_projection(n_cand, of):
    """[threads, n_cand, heads, 128] slices of [threads, `of` tokens, q, k and v heads, 128]; rows are evenly spaced where all tokens or one are taken."""
    t = torch()
    rng = np.random.default_rng(n_cand + of)
    with ap.Pool(4, 2, 128, "bf16_fp4kv", 64) as pool, ap.Rotary(128) as rot:
        threads, lens = [], [3, 20, 1]
        for n in lens:
            threads.append(ap.apar_thread_create(pool.handle))
            z = draw(rng, (n, 2, 128), "bf16")
            ap.apar_append_kv(pool.handle, threads[-1], z, z)
        qkv = draw(rng, (3, of, 8, 128), "bf16")
        was, q, k = qkv.clone(), qkv[:, :n_cand, :4], qkv[:, :n_cand, 4:6]
        chain = t.tensor([(2 << c) - 1 for c in range(n_cand)], dtype=t.uint8, device="cuda").expand(3, n_cand).contiguous()
        ap.apar_rotate_threads(pool.handle, rot.handle, threads, q, k, mask=chain, n_cand=n_cand)
        at = [n + c for n in lens for c in range(n_cand)]
        check(q.reshape(-1, 4, 128), was[:, :n_cand, :4].reshape(-1, 4, 128), at, rot)
        check(k.reshape(-1, 2, 128), was[:, :n_cand, 4:6].reshape(-1, 2, 128), at, rot)
        assert t.equal(qkv[:, n_cand:], was[:, n_cand:]) and t.equal(qkv[:, :, 6:], was[:, :, 6:])
