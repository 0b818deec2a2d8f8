"""The product of e4m3 rows and weights with scales per block of 128, against 64 bits (run with -m gpu)."""
import pytest
import torch

import synth
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]
E4M3 = torch.float8_e4m3fn


def _normal(shape, std, seed, tensor_id):
    return synth.normal_tensor(shape, std, seed, tensor_id, torch.float32)


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _values(shape, seed):
    """e4m3 values over the whole range of the type."""
    return (_normal(shape, 60.0, seed, shape[0] * 7 + shape[1])).clamp(-448, 448).to(E4M3)


def _scales(shape, seed):
    return torch.exp2(_normal(shape, 2.0, seed, shape[0] * 5 + shape[1]) - 8).float()


def _operands(M, N, K, mats=1):
    kb = -(-K // 128)
    x, xs = _values((M, K), 31), _scales((kb, M), 32)
    ws = [(_values((N // mats, K), 33 + i), _scales((-(-(N // mats) // 128), kb), 35 + i)) for i in range(mats)]
    return x, xs, ws


def _wide(t, dev):
    return t.to(dev).double()


def _definition(x, xs, ws, dev):
    """x W^T in 64 bits and the same of the magnitudes, per matrix."""
    K = x.shape[1]
    xf = _wide(x, dev) * _wide(xs, dev).t().repeat_interleave(128, 1)[:, :K]
    out = []
    for q, s in ws:
        w = _wide(q, dev) * _wide(s, dev).repeat_interleave(128, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :K]
        w = w.t().contiguous()
        out.append(((xf @ w).cpu(), (xf.abs() @ w.abs()).cpu()))
    return out


def _bound(K, magnitude):
    """fp32 sums: 128 products in a block, each addition off by at most 2^-23 of the magnitudes (truncation counted), the product
    with the scales (2 roundings) and ceil(K / 128) + 8 additions of blocks."""
    return (128 * 2 + 2 + (-(-K // 128) + 8)) * 2.0 ** -24 * magnitude


def _bound16(M, K, magnitude):
    """Before a rounding to bf16.  From 33 rows on the 8-bit matrix instruction adds 8 products at a time aligned to the largest of
    them; a product 2^-12 of it counts in full, so each is off by less than 2^-13 of the largest: 8 of them 2^-10."""
    return _bound(K, magnitude) + (2.0 ** -10 * magnitude if M > 32 else 0)


def _pack(amd, ws, interleave=False):
    return amd.pack_weights_fp8([(q.cuda(), s.cuda()) for q, s in ws], interleave=interleave)


SHAPES = [(1, 16, 16), (1, 2048, 2048), (2, 48, 144), (5, 2064, 272), (7, 8192, 1024), (8, 272, 2048), (9, 256, 5504), (16, 512, 4096),
          (17, 768, 1040), (31, 1040, 640), (32, 2048, 128), (33, 144, 256), (48, 1024, 1040), (64, 2048, 2048), (65, 272, 640),
          (100, 4096, 1024), (129, 400, 272), (200, 2064, 2048), (255, 528, 4096), (513, 1040, 1168), (600, 2048, 1024),
          (1023, 768, 256), (1030, 4112, 144)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("kind", ["fp32", "bf16", "swiglu"])
def test_matches_definition(M, N, K, kind):
    amd = _amd()
    print(f"gemm_fp8 M={M} N={N} K={K} {kind}", flush=True)
    if kind == "swiglu":
        N = -(-N // 32) * 32
    x, xs, ws = _operands(M, N, K, 2 if kind == "swiglu" else 1)
    ref = _definition(x, xs, ws, "cpu")
    w = _pack(amd, ws, kind == "swiglu")
    got = amd.gemm_fp8(x.cuda(), xs.cuda(), w, 2 if kind == "swiglu" else 0, torch.float32 if kind == "fp32" else torch.bfloat16)
    assert got.dtype == (torch.float32 if kind == "fp32" else torch.bfloat16)
    got = got.cpu().double()
    if kind == "swiglu":
        (g, gm), (u, um) = ref
        want = g * torch.sigmoid(g) * u
        dg, du = _bound16(M, K, gm), _bound16(M, K, um)
        # |silu'| <= 1.1; exp, quotient and products: 2^-20 of the value and |g| 2^-23 from the exponent; one rounding to bf16
        tol = 1.1 * dg * (u.abs() + du) + (g * torch.sigmoid(g)).abs() * du + (2.0 ** -20 + g.abs() * 2.0 ** -23 + 2.0 ** -8) * want.abs()
        assert got.shape == (M, N // 2)
    elif kind == "fp32":
        want, mag = ref[0]
        tol = _bound(K, mag)
    else:
        want, mag = ref[0]
        tol = _bound16(M, K, mag) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    off = (got - want).abs()
    assert (off <= tol + 1e-30).all(), (off - tol).max()
    if kind == "bf16":                                    # and as a whole: a rounding to bf16 is at most 2^-8 of each value
        assert off.norm() <= 2.0 ** -8 * want.norm()


@pytest.mark.parametrize("M,N,K", [(7, 8192, 28672), (40, 12288, 4096), (300, 4096, 11008), (2048, 2048, 8192)])
def test_wide_matrices(M, N, K):
    amd = _amd()
    x, xs, ws = _operands(M, N, K)
    (want, mag), = _definition(x, xs, ws, "cuda")
    w = _pack(amd, ws)
    got = amd.gemm_fp8(x.cuda(), xs.cuda(), w, 0, torch.float32).cpu().double()
    assert ((got - want).abs() <= _bound(K, mag)).all()
    got = amd.gemm_fp8(x.cuda(), xs.cuda(), w).cpu().double()
    assert ((got - want).abs() <= _bound16(M, K, mag) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()).all()


@pytest.mark.parametrize("M", [3, 40, 700])
def test_concatenated_matrices_and_rows_that_are_nan(M):
    """Matrices whose blocks of 128 rows do not line up, one behind the other; a NaN row and an infinite scale stay in their rows,
    also beside the zeros that fill the last block of columns."""
    amd = _amd()
    K = 272
    x, xs, _ = _operands(M, 16, K)
    mats = [(_values((n, K), 40 + n), _scales((-(-n // 128), 3), 41 + n)) for n in (144, 16, 272)]
    w = _pack(amd, mats)
    assert (w.N, w.K) == (432, K)
    want = torch.cat([y for y, _ in _definition(x, xs, mats, "cpu")], 1)
    mag = torch.cat([m for _, m in _definition(x, xs, mats, "cpu")], 1)
    xd, sd = x.cuda(), xs.cuda()
    got = amd.gemm_fp8(xd, sd, w, 0, torch.float32).cpu().double()
    assert ((got - want).abs() <= _bound(K, mag)).all()
    half = amd.gemm_fp8(xd, sd, w)
    xd[1] = float("nan")
    sd[2, 2] = float("inf")
    bad = amd.gemm_fp8(xd, sd, w, 0, torch.float32).cpu().double()
    assert bad[1].isnan().all() and not torch.isfinite(bad[2]).any()
    rest = [m for m in range(M) if m not in (1, 2)]
    assert torch.equal(bad[rest], got[rest])
    bad = amd.gemm_fp8(xd, sd, w)
    assert bad[1].isnan().all() and not torch.isfinite(bad[2]).any()
    assert torch.equal(bad[rest], half[rest])


def test_rows_up_to_32_do_not_depend_on_their_number():
    amd = _amd()
    x, xs, ws = _operands(32, 2064, 1168)
    w = _pack(amd, ws)
    full = amd.gemm_fp8(x.cuda(), xs.cuda(), w)
    for m in (1, 2, 7, 8, 9, 16, 17, 31):
        part = amd.gemm_fp8(x[:m].cuda(), xs[:, :m].contiguous().cuda(), w)
        assert torch.equal(part, full[:m]), m


def test_streams_graphs_and_repeats():
    amd = _amd()
    for M in (5, 96, 600):
        for dtype in (torch.float32, torch.bfloat16):
            x, xs, ws = _operands(M, 1040, 2064)
            w, xd, sd = _pack(amd, ws), x.cuda(), xs.cuda()
            ref = amd.gemm_fp8(xd, sd, w, 0, dtype)
            st = torch.cuda.Stream()
            st.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(st):
                a = amd.gemm_fp8(xd, sd, w, 0, dtype)
            b = amd.gemm_fp8(xd, sd, w, 0, dtype)             # both at once
            torch.cuda.synchronize()
            assert torch.equal(a, ref) and torch.equal(b, ref)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                y = amd.gemm_fp8(xd, sd, w, 0, dtype)
            for rep in range(3):
                sd.copy_(xs.cuda() * 2.0 ** rep)              # a power of two scales every sum exactly
                g.replay()
                torch.cuda.synchronize()
                assert torch.equal(y, ref * 2.0 ** rep) and torch.equal(amd.gemm_fp8(xd, sd, w, 0, dtype), y)


def test_refusals():
    amd = _amd()
    x, xs, ws = _operands(3, 64, 128)
    w, xd, sd = _pack(amd, ws), x.cuda(), xs.cuda()
    with pytest.raises(ValueError):
        amd.gemm_fp8(xd, sd.t().contiguous(), w)
    with pytest.raises(ValueError):
        amd.gemm_fp8(xd[:, :64].contiguous(), sd, w)
    with pytest.raises(ValueError):
        amd.gemm_fp8(xd.float(), sd, w)
    with pytest.raises(ValueError):
        amd.gemm_fp8(xd, sd, w, 2)                        # not interleaved
    with pytest.raises(ValueError):
        amd.gemm_fp8(xd, sd, w, 0, torch.float16)
    with pytest.raises(amd.SpecError):
        amd.gemm_fp8(xd, sd, w, 1)
    with pytest.raises(amd.SpecError):
        amd.gemm_fp8(xd[:0], sd[:, :0].contiguous(), w)
