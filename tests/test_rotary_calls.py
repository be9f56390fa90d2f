"""What the rotary calls make of tensors, without a GPU: tensors of the host that say they are on one.  Calls here are refused before
anything is launched."""
import pytest
import torch

import paper_2401_06761_amd as ap


class OnGpu:
    """A host tensor with a GPU's name on it."""

    is_cuda = True

    def __init__(self, t, device="cuda:0"):
        self.t, self.device = t, torch.device(device)
        self.shape, self.dtype = t.shape, t.dtype

    def get_device(self):
        return self.device.index

    def __getattr__(self, name):
        return getattr(self.t, name)


def status(call):
    with pytest.raises(ap.AparError) as e:
        call()
    return e.value.status


def positions(n):
    return OnGpu(torch.zeros(n, dtype=torch.int32))


@pytest.mark.parametrize("d", [64, 126, 256])
def test_heads_that_are_not_the_rotarys_are_refused(d):
    """(A slice of a projection with smaller heads has rows as far apart as the library would have them: 512 elements of the last row's
    would lie behind the tensor's end.)"""
    p = positions(3)
    with ap.Rotary(128) as rot:
        qk = torch.zeros(3, 16, d)
        for q, k in ((qk[:, :8], qk[:, 8:]), (qk[:, :8].contiguous(), None), (None, qk[:, 8:].contiguous())):
            q, k = (x if x is None else OnGpu(x) for x in (q, k))
            out = OnGpu(torch.zeros(3, 8, d))
            assert status(lambda: ap.apar_rotate_rows(rot.handle, p, q, k, stream=0)) == -1
            assert status(lambda: ap.apar_rotate_rows(rot.handle, p, q, k, None if q is None else out, None if k is None else out, stream=0)) == -1


def test_rows_carry_their_heads():
    rows = ap.binding._rotary_rows(OnGpu(torch.zeros(5, 6, 32)[:, 2:5]), None, 5)
    assert (rows.n_heads, rows.head_dim, rows.in_stride, rows.out_stride) == (3, 32, 192, 192)
    assert ap.AparRotaryRows(1, 1, 2, 2, 3).head_dim == 0


def test_rows_behind_dims_of_size_one():
    """One candidate a thread out of a wider projection, and other leading dims that say nothing."""
    step = ap.binding._row_step
    x = torch.zeros(7, 5, 6, 32)
    assert step(OnGpu(x[:, :1, :2])) == (7, 5 * 6 * 32)
    assert step(OnGpu(x[:, 2, 1:4][:, None])) == (7, 5 * 6 * 32)
    assert step(OnGpu(x[:, None])) == (35, 6 * 32) and step(OnGpu(x[None, :, :, None, :3])) == (35, 6 * 32)
    assert step(OnGpu(x[:1, :, :3])) == (5, 6 * 32) and step(OnGpu(x[:1, :1])) == (1, 6 * 32)
    assert step(OnGpu(x[:, 2, :3][None].transpose(0, 1))) == (7, 5 * 6 * 32)
    for empty in (x[:0], x[:, :0], x[:0, :, None]):
        assert step(OnGpu(empty))[0] == 0
    # a dim of size one says nothing of the ones around it
    flat = torch.zeros(4096)
    for bad in (flat.as_strided((2, 1, 3, 2, 32), (1000, 1000, 64, 32, 1)), flat.as_strided((2, 1, 3, 2, 32), (192, 192, 100, 32, 1)), x[:, :3],
                x[:, :3, None], flat.as_strided((3, 1, 2, 32), (60, 60, 32, 1))):
        with pytest.raises(ValueError):
            step(OnGpu(bad))


def test_tensors_of_several_devices_are_refused():
    x, y = torch.zeros(3, 4, 128), torch.zeros(3, 2, 128)
    masks = torch.ones(3, 1, dtype=torch.uint8)
    with ap.Pool(4, 2, 128, "f32", 8, dry_run=True) as pool, ap.Rotary(128) as rot:
        th = [ap.apar_thread_create(pool.handle) for _ in range(3)]
        for bad in (lambda: ap.apar_rotate_threads(pool.handle, rot.handle, th, OnGpu(x), OnGpu(y, "cuda:1"), stream=0),
                    lambda: ap.apar_rotate_threads(pool.handle, rot.handle, th, OnGpu(x), OnGpu(y), mask=OnGpu(masks, "cuda:1"), n_cand=1, stream=0),
                    lambda: ap.apar_rotate_threads(pool.handle, rot.handle, th, None, OnGpu(y), mask=OnGpu(masks, "cuda:1"), n_cand=1, stream=0),
                    lambda: ap.apar_rotate_threads(pool.handle, rot.handle, th, OnGpu(x), OnGpu(y), OnGpu(x, "cuda:1"), stream=0),
                    lambda: ap.apar_rotate_rows(rot.handle, positions(3), OnGpu(x), OnGpu(y, "cuda:1"), stream=0)):
            with pytest.raises(ValueError):
                bad()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "bf16_fp8kv", "bf16_fp4kv"])
def test_bookkeeping_pools_of_every_type_check_listed_threads(dtype):
    """(There are no rows, and so no type of rows to compare with the pool's.)"""
    with ap.Pool(4, 2, 128, dtype, 8, dry_run=True) as pool, ap.Rotary(128) as rot:
        th = ap.apar_thread_create(pool.handle)
        ap.apar_append_kv(pool.handle, th, None, None, 5)
        ap.apar_rotate_threads(pool.handle, rot.handle, [th, th], None)
        ap.apar_rotate_threads(pool.handle, rot.handle, [th], None, m=[5], where=ap.APAR_ROWS_LAST)
        assert status(lambda: ap.apar_rotate_threads(pool.handle, rot.handle, [th], None, m=[6], where=ap.APAR_ROWS_LAST)) == -1
        assert status(lambda: ap.apar_rotate_threads(pool.handle, rot.handle, [9], None)) == -2
