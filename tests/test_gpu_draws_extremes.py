"""Truncated draws at the ends of what temperatures, scales and logits can be, against the oracle (run with -m gpu)."""
import pytest
import torch

import synth
from tests.test_gpu_draws import _check, _u
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]
INF, LOWEST = float("inf"), torch.finfo(torch.float32).min


def _all_results(x, u, how):
    import paper_2408_11850_amd as amd
    print(f"extremes {tuple(x.shape)} {how}", flush=True)
    tokens, q = amd.sample_rows(x.cuda(), u.cuda(), **how)
    _check(x, u, tokens, q, amd.filter_rows(x.cuda(), **how), **how)


@pytest.mark.parametrize("temperature", [1e37, 3e38])
@pytest.mark.parametrize("masked", [-INF, LOWEST])
@pytest.mark.parametrize("base", [-1e30, 0.0, 5.0, 1e30])
def test_more_ids_asked_for_than_there_are(temperature, masked, base):
    """Where a class of z is wider than fp32, its edge has no fp32 value."""
    V = 28640
    x = torch.full((3, V), base)
    x[0, ::2] = masked
    x[1, 100:] = masked
    x[2, :-1] = masked
    for how in (dict(top_k=16645), dict(top_k=16645, top_p=0.0), dict(top_k=16645, top_p=0.5), dict(top_k=16645, top_p=0.9, min_p=0.5),
                dict(top_k=20000, min_p=0.9), dict(top_k=900, top_p=0.5)):
        _all_results(x, torch.tensor([0.3, 0.5, 0.99]), dict(how, temperature=temperature))


@pytest.mark.parametrize("temperature,scale", [(1e-44, 1.0), (1e-30, 1e30), (3e38, 1e-30), (1.0, 3e38), (3e38, 3e38)])
@pytest.mark.parametrize("how", [dict(), dict(top_k=50), dict(top_k=5000), dict(top_p=0.5), dict(top_k=3000, top_p=0.9, min_p=0.01)], ids=str)
def test_steep_and_flat(temperature, scale, how):
    V = 20000
    x = synth.normal_tensor((4, V), 2.5, 171, V, torch.float32)
    x[1] = (x[1] * 4).round() / 4
    x[2, ::3] = -INF
    x[3] *= 1e37
    _all_results(x, 0.02 + 0.96 * _u(4, 172), dict(how, temperature=temperature, logit_scale=scale))
