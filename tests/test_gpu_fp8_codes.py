"""The codes and scales of rows and weights, bit by bit (run with -m gpu).

scale = largest magnitude / 448 and the code of v / scale, each quotient rounded once to fp32, are what IEEE division gives: nothing
is left to a tolerance.  A product with a rounded reciprocal instead is off in the scale of every third block or so."""
import pytest
import torch

import synth
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


def _codes(blocks):
    """[..., 128] fp32 -> codes and scales [..., 1]."""
    scale = blocks.abs().amax(dim=-1, keepdim=True).clamp_min(2.0 ** -100) / 448
    return (blocks / scale).to(torch.float8_e4m3fn).view(torch.uint8), scale


@pytest.mark.parametrize("M,K,std", [(513, 4096, 1.0), (33, 28672, 40.0), (1, 128, 2.0 ** -60), (7, 11008, 2.0 ** 90)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows(M, K, std, dtype):
    import paper_2408_11850_amd as amd
    print(f"codes M={M} K={K} std={std} {dtype}", flush=True)
    x = (synth.normal_tensor((M, K), 1.0, 31, K, torch.float32) * std).to(dtype)
    q, scale = amd.quant_fp8(x.cuda())
    want_q, want_s = _codes(x.float().view(M, K // 128, 128))
    assert torch.equal(scale.cpu(), want_s[..., 0].t())
    assert torch.equal(q.cpu().view(torch.uint8), want_q.reshape(M, K))


@pytest.mark.parametrize("N,K", [(256, 128), (2048, 5632)])
def test_weights(N, K):
    import paper_2408_11850_amd as amd
    w = synth.normal_tensor((N, K), 0.02, 32, N, torch.float32).bfloat16()
    q, scale = amd.quant_weight_fp8(w.cuda())
    blocks = w.float().view(N // 128, 128, K // 128, 128).transpose(1, 2).reshape(N // 128, K // 128, 128 * 128)
    want_q, want_s = _codes(blocks)
    assert torch.equal(scale.cpu(), want_s[..., 0])
    want_q = want_q.view(N // 128, K // 128, 128, 128).transpose(1, 2).reshape(N, K)
    assert torch.equal(q.cpu().view(torch.uint8), want_q)
