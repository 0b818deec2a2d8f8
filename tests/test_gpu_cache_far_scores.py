"""Attention at references far from 0, with scores that fp32 holds exactly, so that every weight is known (run with -m gpu)."""
import numpy as np
import pytest
import torch

from oracle import cache8
from tests.cache8 import EPS, make, starts_of, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]
SCALE = float(np.float32(np.log(2.0)))           # times log2(e), in fp32, exactly 1: scores to the base 2 are those of q and k


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _batch(rng, lengths, rows, heads, kv, d, width=None):
    """Scores a * 2^21 - gap: a in {-1, 0, 1} by the row and head, gap 0, 1 or 30 by the entry.  Keys (64, gap, 0, ...) under page scales 2^-2 .. 2^2."""
    assert np.float32(SCALE) * np.float32(1.4426950408889634) == 1
    c = make(rng, lengths, kv, d, width=width)
    e = rng.integers(-2, 3, c.scale.shape[:2])
    gap = rng.choice([0.0, 1.0, 1.0, 30.0], c.k.shape[:3])
    k = np.zeros(c.k.shape)
    k[..., 0], k[..., 1] = 64 * 2.0 ** -e[..., None], gap * 2.0 ** -e[..., None]
    c.k, c.scale[:, :, 0] = cache8.encode(k), 2.0 ** e
    assert np.array_equal(cache8.DECODE[c.k], k)
    q = np.zeros((sum(rows), heads, d), np.float32)
    q[..., 0], q[..., 1] = rng.integers(-1, 2, q.shape[:2]) * 2.0 ** 15, -1
    return c, q


@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 3)])
@pytest.mark.parametrize("lengths,rows,heads,kv,d,width", [
    ([300], [5], 4, 2, 128, None), ([200, 90], [1, 1], 2, 2, 64, None), ([2000], [2], 8, 1, 128, None),        # one tile of 16 rows, alone and in parts
    ([400, 300], [40, 7], 8, 1, 64, None), ([300], [150], 4, 2, 64, None),
    ([900], [300], 8, 1, 64, 15), ([900], [300], 8, 1, 128, 15), ([1000], [300], 8, 1, 128, None),             # through LDS, alone and in parts
    ([700, 900, 0, 77, 300], [600, 1, 0, 5, 40], 8, 2, 128, None)])                                            # two passes
def test_weights_are_powers_of_two(lengths, rows, heads, kv, d, width, window, sinks):
    """Weights 1, 1/2 and 2^-30 are exact in bf16; what is left are sums in fp32 (and ln 2's rounding: 2^-25 of a gap of 30), and the
    result's rounding.  The logarithm is as exact as fp32 at 2^21: a sum and two products rounded."""
    amd, rng = _amd(), np.random.default_rng(sum(lengths) + d)
    c, q = _batch(rng, lengths, rows, heads, kv, d, width)
    start = starts_of(rows)
    out, lse = amd.attend_fp8(to_gpu(amd, c), torch.from_numpy(q).cuda().to(torch.bfloat16), torch.from_numpy(start).cuda(), SCALE, window, sinks, want_lse=True)
    want, want_lse, mass, _ = cache8.attend(c, start, q, SCALE, window, sinks)
    got, lse, n = out.float().cpu().numpy(), lse.cpu().numpy(), max(lengths)
    assert np.isfinite(want).all() and np.abs(want_lse).max() > 2.0 ** 20
    bound = 2.0 ** -8 * np.abs(want) + ((2 * n + 32) * EPS + 2.0 ** -20) * mass
    assert (np.abs(got - want) <= bound * 1.01).all(), float((np.abs(got - want) / bound).max())
    assert (np.abs(lse - want_lse) <= 3.1 * EPS * np.abs(want_lse) + (n + 32) * EPS).all()
