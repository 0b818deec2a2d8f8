"""Attention and weights where a page's scale times the softmax's is beyond fp32 (run with -m gpu)."""
import numpy as np
import pytest
import torch

from oracle import cache8
from tests.cache8 import EPS, bf16, check_attention, make, normal, starts_of, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _zero_keys(c, rng):
    c.k = np.where(rng.random(c.k.shape) < 0.5, 0, 0x80).astype(np.uint8)


def _pages_of_zeros(c, rng):
    _zero_keys(c, rng)
    c.scale[:, :, 0] = 2.0 ** -100


def _small_keys(c, rng):
    c.scale[:, :, 0] = 2.0 ** -100


def _some(c, rng):
    """Zeros at the least scale in every other page."""
    c.k[::2] = 0
    c.scale[::2, :, 0] = 2.0 ** -100


def _zeros_at_the_largest(c, rng):
    _zero_keys(c, rng)
    c.scale[:, :, 0] = 2.0 ** 112


KINDS = [(_pages_of_zeros, 2.0 ** -60), (_small_keys, 2.0 ** -60), (_some, 2.0 ** -60), (_some, 2.0 ** -126), (_some, 2.0 ** -149), (_zeros_at_the_largest, 2.0 ** 20)]
# lengths, rows, heads, kv, d: one token, tiles of 16 and 32 rows in registers, rows through LDS, two passes
SIZES = [([300, 65], [1, 1], 4, 2, 128), ([300], [5], 4, 2, 64), ([130, 500], [40, 3], 8, 1, 128), ([1500], [200], 16, 2, 128), ([1500], [200], 16, 2, 64),
         ([700, 900, 300], [600, 1, 5], 8, 2, 128)]


@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
@pytest.mark.parametrize("lengths,rows,heads,kv,d", SIZES)
@pytest.mark.parametrize("change,scale", KINDS)
def test_hidden_entries_stay_hidden(change, scale, lengths, rows, heads, kv, d, window, sinks):
    """Scores are 0, or next to it, and a hidden one is not 0 times an infinity."""
    amd, rng = _amd(), np.random.default_rng(2)
    c = make(rng, lengths, kv, d)
    change(c, rng)
    start = starts_of(rows)
    q = bf16(normal(rng, int(start[-1]), heads, d))
    g, qg, sg = to_gpu(amd, c), torch.from_numpy(q).cuda().to(torch.bfloat16), torch.from_numpy(start).cuda()
    out, lse = amd.attend_fp8(g, qg, sg, scale, window, sinks, want_lse=True)
    want, want_lse, mass, size = cache8.attend(c, start, q, scale, window, sinks)
    assert np.isfinite(want).all()
    check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), want, want_lse, mass, size, d, max(lengths))
    weight = np.zeros((len(lengths), kv, g.capacity), np.float32)
    got = amd.weigh_fp8(g, qg, lse, torch.from_numpy(weight).cuda(), sg, scale, window, sinks).cpu().numpy()
    want, slack = cache8.weigh(c, start, q, lse.cpu().numpy(), weight, scale, window, sinks)
    bound = slack * (d + 5) * EPS * 1.1 + want * (max(rows) * heads // kv + 48) * EPS
    assert np.isfinite(got).all() and (np.abs(got - want) <= bound + 1e-37).all()
