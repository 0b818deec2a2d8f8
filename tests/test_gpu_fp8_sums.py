"""What the 8-bit matrix instructions leave out of a sum, seen where two blocks cancel (run with -m gpu).

The second block of 128 columns is the first one in another order, its weights negated: the exact result is 0, and what comes out is
the two blocks' own errors, far above the rounding of so small a number to bf16."""
import pytest
import torch

import synth
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]
N = 1024


def _normal(shape, seed):
    return synth.normal_tensor(shape, 1.0, seed, 181, torch.float32)


def _cancelling(M, outlier):
    """Operands, and of one block the sums and the sums of magnitudes in 64 bits."""
    import paper_2408_11850_amd as amd
    x = _normal((M, 128), 1)
    x[:, 5] *= outlier
    q, s = amd.quant_fp8(x.cuda())
    w, ws = amd.quant_weight_fp8(_normal((N, 128), 2).bfloat16().cuda())
    order = torch.randperm(128, generator=torch.Generator().manual_seed(3)).cuda()
    codes = lambda t: t.view(torch.uint8)
    x2 = torch.cat([codes(q), codes(q)[:, order]], 1).contiguous().view(torch.float8_e4m3fn)
    w2 = torch.cat([codes(w), codes(w)[:, order] ^ 128], 1).contiguous().view(torch.float8_e4m3fn)
    packed = amd.pack_weights_fp8([(w2, torch.cat([ws, ws], 1).contiguous())])
    xf, wf = q.double() * s.double().t(), (w.double() * ws.double().repeat_interleave(128, 0)).t().contiguous()
    return x2, torch.cat([s, s], 0).contiguous(), packed, xf @ wf, xf.abs() @ wf.abs()


@pytest.mark.parametrize("M", [33, 64, 1000])
@pytest.mark.parametrize("outlier", [1.0, 12.0])
def test_many_rows_to_bf16(M, outlier):
    """A term is off by less than 2^-13 of the largest of its group of 8, so a group by less than 2^-10 of its magnitudes, and both
    blocks together by twice that share of theirs.  For normal operands the share of the 2-norm is the one that include/spec.h
    states; it follows the largest products, so with a column that stands out there is no bound but that of the magnitudes."""
    import paper_2408_11850_amd as amd
    x, xs, w, y, mag = _cancelling(M, outlier)
    off = amd.gemm_fp8(x, xs, w).double()
    assert (off.abs() <= 2 * 2.0 ** -10 * mag).all()
    if outlier == 1.0:
        assert off.norm() <= 1.5e-5 * 2 ** 0.5 * y.norm()


@pytest.mark.parametrize("M,dtype", [(1, torch.bfloat16), (8, torch.bfloat16), (32, torch.bfloat16), (32, torch.float32),
                                     (33, torch.float32), (1000, torch.float32)])
def test_exact_products(M, dtype):
    """Up to 32 rows, and to fp32: 2 x 128 additions and two multiply-adds, each off by at most 2^-23 of the magnitudes."""
    import paper_2408_11850_amd as amd
    x, xs, w, y, mag = _cancelling(M, 12.0)
    off = amd.gemm_fp8(x, xs, w, 0, dtype).double()
    assert (off.abs() <= 2 * 130 * 2.0 ** -23 * mag).all()
    assert off.norm() <= 1e-6 * y.norm()


def test_rows_beyond_fp32_behind_a_norm():
    """As include/spec.h says: 0 where such a row is finite, NaN where it is not; the rows beside it as they were."""
    import paper_2408_11850_amd as amd
    h = _normal((5, 640), 4).cuda()
    gain = torch.ones(640, dtype=torch.bfloat16, device="cuda")
    want, want_s = amd.add_norm_fp8(h.clone(), None, gain, 1e-5)
    h[1, 7], h[2], h[3, 600] = float("inf"), h[2] * 1e20, float("nan")
    q, s = amd.add_norm_fp8(h, None, gain, 1e-5)
    v = q.float() * s.t().repeat_interleave(128, 1)
    assert v[1, 7].isnan() and (v[1].nan_to_num() == 0).all() and v[1].isnan().sum() == 1
    assert (v[2] == 0).all() and v[3].isnan().all()
    for m in (0, 4):
        assert torch.equal(q[m].view(torch.uint8), want[m].view(torch.uint8)) and torch.equal(s[:, m], want_s[:, m])
