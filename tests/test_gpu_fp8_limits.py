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


def test_the_most_weight_rows():
    """2^20 of them: 65536 panels."""
    import paper_2408_11850_amd as amd
    N, K = 1 << 20, 16
    w = synth.normal_tensor((N, K), 0.1, 45, 1, torch.float32).bfloat16().cuda()
    q, s = amd.quant_weight_fp8(w)
    packed = amd.pack_weights_fp8([(q, s)])
    plain = (q.double() * s.double().repeat_interleave(128, 0)).contiguous()
    for M in (1, 20, 40):
        x, xs = _rows(M, K, 46)
        y = amd.gemm_fp8(x, xs, packed, dtype=torch.float32).double()
        xd = x.double() * xs.double().t()
        want, size = xd @ plain.t().contiguous(), xd.abs() @ plain.abs().t().contiguous()
        # 16 exact products: 15 additions, two scalings and the last multiply-add, 2^-24 of the sum of magnitudes each
        assert ((y - want).abs() <= 18 * 2.0 ** -24 * size).all()


def test_many_rows_of_few_columns():
    import paper_2408_11850_amd as amd
    M = (1 << 22) + 3
    x = torch.arange(M, dtype=torch.float32, device="cuda")[:, None] + torch.arange(16, dtype=torch.float32, device="cuda")
    q, s = amd.quant_fp8(x)
    xc, sc = x.cpu(), s[0].cpu()
    assert torch.equal(sc, xc[:, -1] / 448)
    assert torch.equal(q.cpu().view(torch.uint8), (xc / sc[:, None]).to(F8).view(torch.uint8))
    with pytest.raises(ValueError):
        amd.quant_fp8(x[:1].expand(2 ** 32 + 1, 16))
    with pytest.raises(RuntimeError):
        amd.quant_fp8(x[:1].expand(1 << 26, 16))


def test_delta_is_h_itself():
    import paper_2408_11850_amd as amd
    h = synth.normal_tensor((5, 1040), 1.0, 47, 1, torch.float32).cuda()
    gain = torch.ones(1040, dtype=torch.bfloat16, device="cuda")
    ref, twice = h.clone(), h.clone()
    want = amd.add_norm_fp8(ref, h, gain, 1e-5)
    got = amd.add_norm_fp8(twice, twice, gain, 1e-5)
    assert torch.equal(ref, twice) and torch.equal(want[1], got[1])
    assert torch.equal(want[0].view(torch.uint8), got[0].view(torch.uint8))


def test_weights_of_other_sizes_are_refused():
    import paper_2408_11850_amd as amd
    data = torch.zeros(2 * 2 * 2048, dtype=torch.uint8, device="cuda")
    scale = torch.ones((2, 2), device="cuda")
    amd.Fp8Weight(data, scale, 32, 144, False)
    for d, s, n, k in ((data[:-1], scale, 32, 144), (data, scale, 48, 144), (data, scale, 32, 272), (data, scale, 24, 144),
                       (data, scale.t()[:1], 32, 144), (data, scale.double(), 32, 144), (data.cpu(), scale.cpu(), 32, 144),
                       (data.view(torch.int8), scale, 32, 144), (data, scale, 0, 144)):
        with pytest.raises(ValueError):
            amd.Fp8Weight(d, s, n, k, False)
