"""Residual add + RMS norm to e4m3, and rows to e4m3, against the definition in 64 bits (run with -m gpu)."""
import pytest
import torch

import synth
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]
EPS = 1e-5
E4M3 = torch.float8_e4m3fn
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _normal(shape, std, seed, tensor_id):
    return synth.normal_tensor(shape, std, seed, tensor_id, torch.float32)


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _blocks(y):
    """Scales [blocks][M] in 64 bits."""
    return torch.stack([y[:, b:b + 128].abs().amax(dim=1).clamp_min(2.0 ** -100) / 448 for b in range(0, y.shape[1], 128)])


def _check_rows(q, scale, y, scale_rel):
    """q is a nearest e4m3 value of y / scale.  In fp32 y costs at most 2 roundings beside the row's common factor, which the
    quotient loses, the scale 2 + 2 (of the largest y, the constant and the product), its reciprocal and the product one each:
    8 in all, 2^-24 each.  Around a border either neighbour is right: off by half a step and 8 * 2^-24 of the value."""
    s = _blocks(y)
    assert ((scale.cpu().double() - s).abs() <= scale_rel * s).all()
    v = y / s.t().repeat_interleave(128, 1)[:, :y.shape[1]]
    slack = 8 * 2.0 ** -24 * v.abs()
    step = torch.exp2(torch.floor(torch.log2((v.abs() + slack).clamp_min(2.0 ** -6))) - 3)
    off = (q.cpu().double() - v).abs()
    assert (off <= step / 2 + slack).all(), (off - step / 2).max()
    assert q.dtype == E4M3 and q.is_contiguous() and tuple(scale.shape) == (-(-y.shape[1] // 128), y.shape[0])


@pytest.mark.parametrize("M,d", [(1, 16), (3, 112), (1, 128), (5, 144), (2, 512), (9, 528), (4, 1024), (7, 2048), (33, 4096),
                                 (1, 8192), (300, 5504), (2, 8208), (3, 16384), (2, 32768), (1, 30000)])
@pytest.mark.parametrize("ht,dt", [("fp32", "fp32"), ("bf16", "bf16"), ("fp32", "bf16"), ("bf16", "fp32"), ("fp32", None),
                                   ("bf16", None)])
def test_add_norm(M, d, ht, dt):
    amd = _amd()
    print(f"add_norm M={M} d={d} {ht} {dt}", flush=True)
    h = _normal((M, d), 3.0, 11, d).to(TYPES[ht])
    delta = _normal((M, d), 1.0, 12, d).to(TYPES[dt]) if dt else None
    gain = (1 + 0.3 * _normal((d,), 1.0, 13, d)).bfloat16()
    hd = h.cuda()
    q, scale = amd.add_norm_fp8(hd, delta.cuda() if dt else None, gain.cuda(), EPS)
    want = h if delta is None else (h.float() + delta.float()).to(TYPES[ht])
    assert torch.equal(hd.cpu(), want)                     # one fp32 addition, one rounding
    x = want.double()
    y = x / torch.sqrt(x.square().mean(dim=1, keepdim=True) + EPS) * gain.double()
    # the row's factor: 8 + 6 + up to 64 sequential additions of squares, each 2^-24, halved by the root, and 4 roundings more
    _check_rows(q, scale, y, ((8 + 6 + 64) / 2 + 4 + 4) * 2.0 ** -24)


def test_rows_do_not_depend_on_their_number():
    amd = _amd()
    for d in (144, 2048, 8192, 10000):
        h = _normal((70, d), 2.0, 14, d).cuda()
        gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
        q, s = amd.add_norm_fp8(h.clone(), None, gain, EPS)
        for m in (0, 69):
            q1, s1 = amd.add_norm_fp8(h[m:m + 1].clone(), None, gain, EPS)
            assert torch.equal(q1.view(torch.uint8)[0], q.view(torch.uint8)[m]) and torch.equal(s1[:, 0], s[:, m])


def test_strided_rows_and_a_row_for_all():
    """Rows inside wider ones, at odd addresses; what lies between them stays as it was."""
    amd = _amd()
    M, d = 6, 272
    for t in (torch.float32, torch.bfloat16):
        big = _normal((M, d + 37), 1.0, 15, 1).to(t).cuda()
        keep = big.clone()
        h = big[:, 3:3 + d]
        delta = _normal((1, d), 1.0, 15, 2).to(t).cuda().expand(M, d)
        gain = _normal((d + 1,), 1.0, 15, 3).bfloat16().cuda()[1:]
        want = (h.float() + delta.float()).to(t)
        ref = amd.add_norm_fp8(want.clone(), None, gain, EPS)
        got = amd.add_norm_fp8(h, delta, gain, EPS)
        assert torch.equal(h, want) and torch.equal(big[:, :3], keep[:, :3]) and torch.equal(big[:, 3 + d:], keep[:, 3 + d:])
        for a, b in zip(got, ref):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        a, b = amd.quant_fp8(h), amd.quant_fp8(h.contiguous())
        assert torch.equal(a[0].view(torch.uint8), b[0].view(torch.uint8)) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("M,K", [(1, 16), (2, 128), (7, 28672), (130, 1360), (1, 32768), (65, 11008)])
@pytest.mark.parametrize("t", ["fp32", "bf16"])
def test_quant(M, K, t):
    amd = _amd()
    x = (_normal((M, K), 1.0, 16, K) * 10.0 ** _normal((M, 1), 2.0, 17, K)).to(TYPES[t])
    q, scale = amd.quant_fp8(x.cuda())
    _check_rows(q, scale, x.double(), 2 * 2.0 ** -24)      # the constant and the product


@pytest.mark.parametrize("N,K", [(16, 16), (144, 272), (256, 128), (2064, 1040)])
def test_quant_weight(N, K):
    amd = _amd()
    w = _normal((N, K), 0.02, 18, N).bfloat16()
    q, scale = amd.quant_weight_fp8(w.cuda())
    s = torch.stack([_blocks(w.double()[n:n + 128].abs().amax(dim=0, keepdim=True))[:, 0] for n in range(0, N, 128)])
    assert ((scale.cpu().double() - s).abs() <= 2 * 2.0 ** -24 * s).all()
    v = w.double() / s.repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    slack = 4 * 2.0 ** -24 * v.abs()
    step = torch.exp2(torch.floor(torch.log2((v.abs() + slack).clamp_min(2.0 ** -6))) - 3)
    assert ((q.cpu().double() - v).abs() <= step / 2 + slack).all()


def test_zeros_infinities_and_nan():
    amd = _amd()
    x = torch.ones((4, 384), device="cuda")
    x[0] = 0
    x[1, 130] = float("nan")
    x[2, 5] = float("inf")
    x[3, :128] = 1e-40                                    # below the least scale
    q, s = amd.quant_fp8(x)
    v = q.float() * s.t().repeat_interleave(128, 1)
    assert (v[0] == 0).all() and torch.isfinite(s[:, 0]).all() and (s[:, 0] > 0).all()
    assert v[1].isnan().sum() == 1 and v[1, 130].isnan() and torch.isfinite(s[:, 1]).all()
    assert v[2, :128].isnan().all() and torch.isfinite(v[2, 128:]).all()
    assert (v[3, :128] == 0).all() and ((v[3, 128:] - 1).abs() < 2.0 ** -4).all()
    gain = torch.ones(384, dtype=torch.bfloat16, device="cuda")
    q, s = amd.add_norm_fp8(x, None, gain, EPS)
    v = q.float() * s.t().repeat_interleave(128, 1)
    assert (v[0] == 0).all() and v[1].isnan().all() and v[2, 5].isnan() and torch.isfinite(v[3]).all()


def test_another_stream_and_a_captured_call():
    amd = _amd()
    h = _normal((5, 2048), 1.0, 19, 1).cuda()
    gain = torch.ones(2048, dtype=torch.bfloat16, device="cuda")
    ref = amd.add_norm_fp8(h.clone(), None, gain, EPS)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        a = amd.add_norm_fp8(h.clone(), None, gain, EPS)
    st.synchronize()
    assert torch.equal(a[1], ref[1])
    x = h.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        q, s = amd.add_norm_fp8(x, h, gain, EPS)
    for rep in range(3):                                   # x = (1 + rep + 1) h
        x.copy_(h * (1 + rep))
        g.replay()
        torch.cuda.synchronize()
        want = amd.add_norm_fp8(h * (1 + rep), h, gain, EPS)
        assert torch.equal(s, want[1]) and torch.equal(q.view(torch.uint8), want[0].view(torch.uint8))
