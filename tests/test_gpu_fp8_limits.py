"""8-bit operators where a neighbour's values or the largest sizes could do harm (run with -m gpu)."""
import pytest
import torch

import synth
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]
F8 = torch.float8_e4m3fn


def _rows(M, K, seed):
    import paper_2408_11850_amd as amd
    return amd.quant_fp8(synth.normal_tensor((M, K), 1.0, seed, K, torch.float32).cuda())


@pytest.mark.parametrize("K", [16, 128, 144, 272, 640, 1168, 2176, 4352])
@pytest.mark.parametrize("M", [1, 8, 9, 16, 17, 32, 33, 100])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_panel_is_not_reached_by_its_neighbours(M, K, bad):
    """Matrices of one panel each; those with scales that are no numbers leave the results of the others bit by bit."""
    import paper_2408_11850_amd as amd
    print(f"neighbours M={M} K={K} {bad}", flush=True)
    x, xs = _rows(M, K, 41)
    mats = [amd.quant_weight_fp8(synth.normal_tensor((16, K), 0.1, 42, n, torch.float32).bfloat16().cuda()) for n in range(6)]
    for dtype in (torch.float32, torch.bfloat16):
        want = amd.gemm_fp8(x, xs, amd.pack_weights_fp8(mats), dtype=dtype)
        spoilt = [(q, torch.full_like(s, bad) if n in (1, 4) else s) for n, (q, s) in enumerate(mats)]
        got = amd.gemm_fp8(x, xs, amd.pack_weights_fp8(spoilt), dtype=dtype)
        good = [c for n in (0, 2, 3, 5) for c in range(16 * n, 16 * n + 16)]
        assert torch.equal(got[:, good], want[:, good])
        assert not torch.isfinite(got[:, 16:32]).any() and not torch.isfinite(got[:, 64:80]).any()


@pytest.mark.parametrize("M", [1, 7, 8, 9, 16, 30, 33, 100])
def test_a_row_is_not_reached_by_its_neighbours(M):
    import paper_2408_11850_amd as amd
    K = 1168
    x, xs = _rows(M, K, 43)
    w = amd.pack_weights_fp8([amd.quant_weight_fp8(synth.normal_tensor((160, K), 0.1, 44, 1, torch.float32).bfloat16().cuda())])
    want = amd.gemm_fp8(x, xs, w, dtype=torch.float32)
    bad = xs.clone()
    bad[:, ::3] = float("nan")
    got = amd.gemm_fp8(x, bad, w, dtype=torch.float32)
    keep = [m for m in range(M) if m % 3]
    assert torch.equal(got[keep], want[keep]) and got[::3].isnan().all()
