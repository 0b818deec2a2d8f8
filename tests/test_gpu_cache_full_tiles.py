"""A row's attention does not depend on whether other rows fill its tile of 16 (run with -m gpu)."""
import numpy as np
import pytest
import torch

from tests.cache8 import make, normal, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [30, 300, 3000])
@pytest.mark.parametrize("heads", [1, 5, 8])
def test_the_same_bits_in_full_tiles(heads, n, d):
    """The heads of one token, and the same heads several times over."""
    import paper_2408_11850_amd as amd
    amd.load_library()
    rng = np.random.default_rng(n + heads)
    g = to_gpu(amd, make(rng, [n, n - 7], 1, d, junk=True))
    q = torch.from_numpy(normal(rng, 2, heads, d)).cuda().to(torch.bfloat16)
    out, lse = amd.attend_fp8(g, q, want_lse=True)
    times = 16 // heads
    full, full_lse = amd.attend_fp8(g, q.repeat(1, times, 1), want_lse=True)
    assert torch.equal(full.view(2, times, heads, d), out[:, None].expand(2, times, heads, d))
    assert torch.equal(full_lse.view(2, times, heads), lse[:, None].expand(2, times, heads))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("level", [1.0, 50.0, 1e7])
@pytest.mark.parametrize("m,n,width", [(1, 300, None), (1, 3000, None), (300, 900, 15)])
def test_the_same_bits_beside_other_rows(m, n, width, level, d):
    """Eight heads alone, and beside eight whose scores rise further: references of a tile's rows are their own.  300 rows go through LDS."""
    import paper_2408_11850_amd as amd
    amd.load_library()
    rng = np.random.default_rng(n + d)
    g = to_gpu(amd, make(rng, [n], 1, d, width=width))
    q = torch.from_numpy(normal(rng, m, 16, d)).cuda()
    q[:, 8:] *= level
    q = q.to(torch.bfloat16)
    both, both_lse = amd.attend_fp8(g, q, want_lse=True)
    for half in (slice(0, 8), slice(8, 16)):
        out, lse = amd.attend_fp8(g, q[:, half].contiguous(), want_lse=True)
        assert torch.equal(both[:, half], out) and torch.equal(both_lse[:, half], lse)
