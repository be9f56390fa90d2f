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
