"""Rotation next to quarter turns, where a cosine is small and the angle's rounding would show in the codes (run with -m gpu)."""
import numpy as np
import pytest
import torch

from oracle import cache8
from tests.cache8 import codes, make, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("theta,far", [(10000.0, 0), (10000.0, 4000), (500000.0, 100000), (100.0, 700)])
def test_codes_next_to_a_border(theta, far, d):
    """Keys (0, .., x, .., 0) whose x * cos lies 9 to 11 * 2^-24 of itself beside the border of two codes.  cos is off by 4 * 2^-24 of itself
    at most (2 ulp), its correction's sum and the product by 2^-24 each; an angle rounded to fp32 would count 2^-26 of a turn,
    6 to 80 * 2^-24 of a cosine of 0.1 to 0.019."""
    import paper_2408_11850_amd as amd
    amd.load_library()
    rng, half = np.random.default_rng(far + d), d // 2
    rows = 64 * 8
    c = make(rng, [rows], 1, d)
    angle = (far + np.arange(rows))[:, None] * np.float64(theta) ** (-np.arange(half) / half)
    turn = angle / (2 * np.pi)
    turn -= np.rint(turn)
    at = (np.abs(turn) >= 0.2535) & (np.abs(turn) <= 0.266)
    cos = np.cos(angle)
    # a border between neighbouring codes for x between 1 and 1.7: the page's scale is 2^-8 where one of them is there
    level = 256 * np.abs(cos) * rng.uniform(1.02, 1.65, cos.shape)
    step = 2.0 ** (np.floor(np.log2(level)) - 3)
    border = (np.floor(level / step) + 0.5) * step
    beside = rng.choice([-1.0, 1.0], cos.shape) * 10 * 2.0 ** -24
    x = (border / 256 / np.abs(cos) * (1 + beside)).astype(np.float32)
    k = np.zeros((rows, 1, d), np.float32)
    k[:, 0, half:] = np.where(at, x, 0)
    k[::64, 0, 0] = 0
    away = x.astype(np.float64) * np.abs(cos) * 256 / border - 1
    assert at.sum() > 100 and (np.abs(away[at]) > 8.9 * 2.0 ** -24).all() and (np.sign(away[at]) == np.sign(beside[at])).all()
    g = to_gpu(amd, c)
    amd.append_fp8(g, torch.from_numpy(k).cuda(), torch.from_numpy(np.zeros_like(k)).cuda(), theta=theta,
                   position=torch.tensor([far], dtype=torch.int32, device="cuda"))
    c.append([0, rows], k, np.zeros_like(k), theta, [far])
    assert np.array_equal(g.scale.cpu().numpy(), c.scale)
    pages = c.table[0, :rows // 64]
    got = cache8.DECODE[codes(g.k)[pages, 0].reshape(rows, d)][:, half:]
    want = cache8.DECODE[c.k[pages, 0].reshape(rows, d)][:, half:]
    assert (got == want)[at].all(), f"{int((got != want)[at].sum())} of {int(at.sum())}"
