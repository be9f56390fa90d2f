"""oracle.sampling on rows whose draws can be told by hand (CPU), and the library's refusals that need no GPU."""
import numpy as np
import pytest

import paper_2401_06761_amd as ap
from oracle import sampling

LN = np.log


def test_shares_are_drawn_in_order_of_value():
    x = LN([0.1, 0.4, 0.2, 0.3])
    got = [sampling.draw(x, u=u)[0] for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91, 0.99)]
    assert got == [1, 1, 3, 3, 2, 2, 0, 0]
    assert abs(sampling.draw(x, u=0.95)[1] - LN(0.1)) < 1e-12


def test_cuts():
    x = LN([0.1, 0.4, 0.2, 0.3])
    assert {sampling.draw(x, top_k=2, u=u)[0] for u in np.linspace(0, 0.999, 50)} == {1, 3}
    assert {sampling.draw(x, top_p=0.75, u=u)[0] for u in np.linspace(0, 0.999, 50)} == {1, 3, 2}
    assert {sampling.draw(x, top_p=0.0, u=u)[0] for u in np.linspace(0, 0.999, 50)} == {1}
    assert {sampling.draw(x, min_p=0.6, u=u)[0] for u in np.linspace(0, 0.999, 50)} == {1, 3}
    # top_p counts the mass that top_k keeps: 0.4 / 0.7 is more than half
    assert {sampling.draw(x, top_k=2, top_p=0.5, u=u)[0] for u in np.linspace(0, 0.999, 50)} == {1}


def test_ties_empty_rows_and_greedy():
    assert [sampling.draw([2.0, 2.0, 2.0, 1.0], top_k=2, u=u)[0] for u in (0.0, 0.49, 0.51, 0.99)] == [0, 0, 1, 1]
    assert sampling.draw([np.nan, -np.inf])[0] == sampling.NONE
    assert sampling.draw([1.0, np.nan, 5.0, 5.0], temperature=0.0)[0] == 2
    assert [sampling.draw([np.inf, 3.0, np.inf], u=u)[0] for u in (0.0, 0.6)] == [0, 2]


@pytest.mark.parametrize("args,status", [((4, 0), -1), ((-1, 10), -1), ((4, (1 << 20) + 1), -6)])
def test_workspace_refusals(args, status):
    with pytest.raises(ap.AparError) as e:
        ap.apar_sample_workspace_bytes(*args)
    assert e.value.status == status


def test_call_refusals():
    import ctypes as C

    L = ap.binding._L()
    ok = dict(logits=4096, dtype=ap.APAR_BF16, n=2, vocab=10, stride=10, rows=None, u=4096, ids=None, tokens=4096, logp=None, ws=None, bytes=1 << 30)

    def status(**kw):
        a = {**ok, **kw}
        return L.apar_sample_tokens(a["logits"], a["dtype"], a["n"], a["vocab"], a["stride"], a["rows"], a["u"], a["ids"], a["tokens"], a["logp"],
                                    a["ws"], a["bytes"], None)

    assert status(n=0) == 0
    for kw in ({"logits": None}, {"u": None}, {"tokens": None}, {"n": -1}, {"vocab": 0}, {"dtype": 2}, {"stride": 9}, {"logits": 4097},
               {"dtype": ap.APAR_F32, "logits": 4098}, {"u": 4098}, {"tokens": 4098}, {"rows": 4098}, {"logp": 4098}):
        assert status(**kw) == -1, kw
    assert status(vocab=(1 << 20) + 1, stride=1 << 21) == -6
    with pytest.raises(ValueError):
        import torch

        ap.apar_sample_tokens(torch.zeros(2, 3), torch.zeros(2), torch.zeros(2, dtype=torch.int32))  # not on a GPU
