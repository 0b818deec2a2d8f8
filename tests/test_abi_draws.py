"""Truncated draws: refusals on the host (no GPU is needed), and the oracle against hand-worked rows."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

from oracle import draws


@pytest.fixture(scope="module")
def amd():
    import paper_2408_11850_amd as amd
    if not os.path.exists(amd.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    amd.load_library()
    return amd


P, Q = 4096, 8192         # aligned addresses that are never read
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("change", [
    dict(logits=None), dict(s=None), dict(work=None), dict(q=None, masked=None, tok=None), dict(n=0), dict(n=65536), dict(v=0),
    dict(v=(1 << 20) + 1, ld=1 << 21), dict(ld=99), dict(ld=0), dict(t=-1.0), dict(t=NAN), dict(t=INF), dict(scale=0.0), dict(scale=-1.0),
    dict(scale=NAN), dict(scale=INF), dict(k=-1), dict(p=-0.1), dict(p=1.5), dict(p=NAN), dict(m=-0.1), dict(m=1.01), dict(m=NAN),
    dict(u=None), dict(masked=Q), dict(q=P, ld=128), dict(masked=P, ld=101), dict(logits=P + 2), dict(u=P + 1), dict(work=P + 8),
    dict(tok=P + 2)], ids=str)
def test_refuses(amd, change):
    a = dict(logits=P, ld=100, n=2, v=100, t=1.0, scale=1.0, k=0, p=1.0, m=0.0, u=P, q=Q, masked=None, tok=P, work=P, s=1)
    a.update(change)
    s = amd.Sampling(a["t"], a["scale"], a["k"], a["p"], a["m"])
    rc = amd.load_library().spec_sample_rows(a["logits"], a["ld"], a["n"], a["v"], C.byref(s) if a["s"] else None, a["u"], a["q"],
                                             a["masked"], a["tok"], a["work"], None)
    assert rc == amd.SPEC_E_INVAL


def test_workspace_and_python_refusals(amd):
    size = amd.load_library().spec_sample_rows_workspace_bytes
    assert size(0, 100) == 0 and size(1, 0) == 0 and size(1, (1 << 20) + 1) == 0
    assert 0 < size(1, 100) < size(1, 128256) < size(8, 128256) < 8 << 20
    with pytest.raises(ValueError):
        amd.sample_rows(torch.zeros(2, 8), torch.zeros(2))
    with pytest.raises(ValueError):
        amd.filter_rows(torch.zeros(2, 8))
    for k in (-1, 1 << 31, (1 << 32) + 5):
        with pytest.raises(ValueError):
            amd.sample_rows(torch.zeros(2, 8), torch.zeros(2), top_k=k)


def test_the_oracle_on_hand_worked_rows():
    x = np.log(np.array([1, 8, 2, 8, 4, 1], dtype=np.float64)).astype(np.float32)      # weights 1/8 1 1/4 1 1/2 1/8
    kept = lambda **how: np.flatnonzero(draws.weights(x, **how)).tolist()
    assert kept(top_k=1) == [1] and kept(top_k=2) == [1, 3] and kept(top_k=5) == [0, 1, 2, 3, 4]
    assert kept(top_p=0.0) == [1] and kept(top_p=0.3) == [1] and kept(top_p=0.5) == [1, 3] and kept(top_p=0.8) == [1, 3, 4]
    assert kept(top_k=3, top_p=0.7) == [1, 3]              # 2 of 2.5; of all 3 it would be 0.667
    assert kept(min_p=0.3) == [1, 3, 4] and kept(min_p=1.0) == [1, 3] and kept(temperature=0.0) == [1]
    assert kept(temperature=0.5, min_p=0.3) == [1, 3]
    tok, q = draws.row(x, 0.55, top_k=3)
    assert tok == 3 and np.allclose(q, [0, 0.4, 0, 0.4, 0.2, 0])
    assert draws.row(x, 0.35, top_k=3)[0] == 1 and draws.row(x, 1.0, top_k=3)[0] == 4
    assert draws.row(np.full(4, -np.inf), 0.5)[0] == -1
