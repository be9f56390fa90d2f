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
