"""Three limits at once, the k-th id not found by groups: every order in which the borders of top-k, top-p and min-p can stand,
against the oracle in 64 bits (run with -m gpu)."""
import numpy as np
import pytest
import torch

import synth
from oracle import draws
from tests.test_gpu_draws import _check, _logits, _u
from tests.util import gpu_available

TOP_P, MIN_P = (0.25, 0.5, 0.9), (1 / 128, 0.02, 0.1)
GRID = [(5000, 1025), (32000, 1025), (32000, 2000), (32000, 5000), (128256, 1500), (128256, 40000)]


def _rows(V, coarse):
    return _logits(2, V, 141, coarse)


def _two_levels():
    """1000 ids near 0 and 19000 near -3; 40 ids down to -1.2 before 4960 at -6."""
    a = torch.full((1, 20000), -3.0)
    a[0, ::20] = 0.05 * synth.normal_tensor((1000,), 1.0, 142, 1, torch.float32)
    b = torch.full((1, 20000), -6.0)
    b[0, 7:7 + 40 * 100:100] = torch.linspace(0, -1.2, 40)
    b[0, 5000:] = -float("inf")
    return torch.cat([a, b])


# logits, settings: the k-th id inside the lower level, min-p between the two
LEVELS = [dict(top_k=k, top_p=p, min_p=m) for k, p, m in ((5000, 0.5, 0.1), (1100, 0.5, 0.25), (1100, 0.7, 0.25), (3000, 0.9, 0.06),
                                                          (1100, 0.95, 0.001), (19000, 0.25, 0.1))]
# so steep that the k-th id lies more than 32 below the largest
STEEP = [dict(top_k=k, top_p=p, min_p=m, temperature=0.125) for k in (1500, 20000) for p in (0.5, 0.9) for m in (0.02, 0.1)]


def _order(row, top_k, top_p, min_p, temperature=1.0):
    """The borders by how many ids lie before each, each on its own (top-p's among the first k)."""
    count = lambda **how: int((draws.weights(row, temperature=temperature, **how) > 0).sum())
    at = {"p": count(top_k=top_k, top_p=top_p), "k": top_k, "m": count(min_p=min_p)}
    return "".join(sorted(at, key=at.get))


def test_every_order_occurs():
    """Host logic, no GPU needed: top-p's border never lies behind the k-th id."""
    seen = {_order(row, k, p, m) for V, k in GRID[:4] for row in _rows(V, False).numpy() for p in TOP_P for m in MIN_P}
    assert seen == {"mpk", "pmk", "pkm"}
    levels = [_order(row, **how) for row in _two_levels().numpy() for how in LEVELS]
    assert levels.count("pmk") >= 4 and "pkm" in levels
    row = _rows(32000, False).numpy()[0]
    assert all(_order(row, **how) in ("pmk", "mpk") for how in STEEP)
    assert (np.sort(row)[::-1][1500] - row.max()) / 0.125 < -32


def _all_results(x, how, u):
    import paper_2408_11850_amd as amd
    xd = x.cuda()
    tokens, q = amd.sample_rows(xd, u.cuda(), **how)
    masked = amd.filter_rows(xd, **how)
    _check(x, u, tokens, q, masked, **how)
    assert torch.equal(masked > -float("inf"), q > 0)


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs a GPU")
@pytest.mark.parametrize("V,top_k", GRID)
@pytest.mark.parametrize("coarse", [False, True])
def test_three_limits(V, top_k, coarse):
    x, u = _rows(V, coarse), _u(2, V + top_k)
    for top_p in TOP_P:
        for min_p in MIN_P:
            how = dict(top_k=top_k, top_p=top_p, min_p=min_p)
            print(f"borders V={V} {how} coarse={coarse}", flush=True)
            _all_results(x, how, u)


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs a GPU")
@pytest.mark.parametrize("how", LEVELS, ids=str)
def test_two_levels(how):
    print(f"levels {how}", flush=True)
    _all_results(_two_levels(), how, torch.tensor([0.3, 0.99]))


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs a GPU")
@pytest.mark.parametrize("how", STEEP, ids=str)
def test_a_kth_id_far_below(how):
    print(f"steep {how}", flush=True)
    _all_results(_rows(32000, False), how, torch.tensor([0.3, 0.99]))
