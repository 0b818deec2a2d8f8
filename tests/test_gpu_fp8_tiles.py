"""Every tile of the many-row product, with rows, panels and columns that end inside one, against 64 bits (run with -m gpu); each
case asserts the tile it takes."""
import ctypes as C

import pytest
import torch

from tests.test_gpu_fp8_gemm import _bound, _bound16, _definition, _operands, _pack
from tests.util import gpu_available


def _tile(M, N, K, exact):
    import paper_2408_11850_amd as amd
    amd.load_library()
    f = C.CDLL(amd.LIB_PATH)._Z8fp8_tileiiib
    f.restype, f.argtypes = C.c_int, [C.c_int, C.c_int, C.c_int, C.c_bool]
    return f(M, N // 16, -(-K // 128), exact)


# tile -> shapes (M, N, K)
BF16 = {0: [(4000, 4096, 272), (3841, 4080, 144), (4095, 4064, 128)], 1: [(2040, 6144, 272), (1793, 6080, 144)],
        2: [(1000, 8192, 400), (897, 8160, 528)], 3: [(1000, 4096, 272), (897, 4064, 144), (1024, 4096, 128)],
        4: [(33, 48, 16), (64, 64, 128), (65, 4112, 272), (200, 1040, 400)]}
FP32 = {2: [(1000, 8192, 400), (897, 8160, 528)], 3: [(1000, 4096, 272), (897, 4064, 144)], 4: [(33, 48, 16), (65, 4112, 272)]}


def _cases(table):
    return [(tile, *shape) for tile, shapes in table.items() for shape in shapes]


def test_the_shapes_reach_every_tile():
    """Host logic, no GPU needed."""
    assert {t for t, *_ in _cases(BF16)} == {0, 1, 2, 3, 4} and {t for t, *_ in _cases(FP32)} == {2, 3, 4}
    for exact, table in ((False, BF16), (True, FP32)):
        for tile, M, N, K in _cases(table):
            assert _tile(M, N, K, exact) == tile, (M, N, K, exact)


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs a GPU")
@pytest.mark.parametrize("tile,M,N,K", _cases(BF16))
def test_bf16_results(tile, M, N, K):
    import paper_2408_11850_amd as amd
    print(f"gemm_fp8 tile {tile} M={M} N={N} K={K}", flush=True)
    x, xs, ws = _operands(M, N, K)
    (want, mag), = _definition(x, xs, ws, "cuda")
    w = _pack(amd, ws)
    got = amd.gemm_fp8(x.cuda(), xs.cuda(), w)
    off = (got.cpu().double() - want).abs()
    assert (off <= _bound16(M, K, mag) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()).all()
    assert off.norm() <= 2.0 ** -8 * want.norm()
    assert torch.equal(amd.gemm_fp8(x.cuda(), xs.cuda(), w), got)


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs a GPU")
@pytest.mark.parametrize("tile,M,N,K", _cases(FP32))
def test_fp32_results(tile, M, N, K):
    import paper_2408_11850_amd as amd
    print(f"gemm_fp8 fp32 tile {tile} M={M} N={N} K={K}", flush=True)
    x, xs, ws = _operands(M, N, K)
    (want, mag), = _definition(x, xs, ws, "cuda")
    got = amd.gemm_fp8(x.cuda(), xs.cuda(), _pack(amd, ws), 0, torch.float32)
    assert ((got.cpu().double() - want).abs() <= _bound(K, mag)).all()


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs a GPU")
@pytest.mark.parametrize("tile,M,N,K", [c for c in _cases(BF16) if c[2] % 32 == 0])
def test_gate_up(tile, M, N, K):
    import paper_2408_11850_amd as amd
    print(f"gemm_fp8 gate/up tile {tile} M={M} N={N} K={K}", flush=True)
    x, xs, ws = _operands(M, N, K, 2)
    (g, gm), (u, um) = _definition(x, xs, ws, "cuda")
    want = g * torch.sigmoid(g) * u
    dg, du = _bound16(M, K, gm), _bound16(M, K, um)
    tol = 1.1 * dg * (u.abs() + du) + (g * torch.sigmoid(g)).abs() * du + (2.0 ** -20 + g.abs() * 2.0 ** -23 + 2.0 ** -8) * want.abs()
    got = amd.gemm_fp8(x.cuda(), xs.cuda(), _pack(amd, ws, True), 2).cpu().double()
    assert ((got - want).abs() <= tol + 1e-30).all()


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs a GPU")
@pytest.mark.parametrize("M,N,K", [(8, 8208, 272), (9, 8208, 400), (16, 8208, 272), (17, 8208, 272), (32, 8208, 1040), (17, 16432, 272),
                                   (32, 16416, 400), (12, 8176, 272), (32, 8176, 272)])
@pytest.mark.parametrize("kind", ["fp32", "bf16", "swiglu"])
def test_few_rows_of_wide_matrices(M, N, K, kind):
    """Panels taken one, two and four at a time, the last of them not whole."""
    import paper_2408_11850_amd as amd
    if kind == "swiglu":
        N = -(-N // 32) * 32
    print(f"gemm_fp8 M={M} N={N} K={K} {kind}", flush=True)
    x, xs, ws = _operands(M, N, K, 2 if kind == "swiglu" else 1)
    ref = _definition(x, xs, ws, "cuda")
    w = _pack(amd, ws, kind == "swiglu")
    got = amd.gemm_fp8(x.cuda(), xs.cuda(), w, 2 if kind == "swiglu" else 0, torch.float32 if kind == "fp32" else torch.bfloat16)
    got = got.cpu().double()
    if kind == "swiglu":
        (g, gm), (u, um) = ref
        want = g * torch.sigmoid(g) * u
        dg, du = _bound(K, gm), _bound(K, um)
        tol = 1.1 * dg * (u.abs() + du) + (g * torch.sigmoid(g)).abs() * du + (2.0 ** -20 + g.abs() * 2.0 ** -23 + 2.0 ** -8) * want.abs()
    else:
        want, mag = ref[0]
        tol = _bound(K, mag) if kind == "fp32" else _bound(K, mag) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    assert ((got - want).abs() <= tol + 1e-30).all()
    one = amd.gemm_fp8(x[:1].cuda(), xs[:, :1].contiguous().cuda(), w, 2 if kind == "swiglu" else 0,
                       torch.float32 if kind == "fp32" else torch.bfloat16)
    assert torch.equal(one.cpu().double(), got[:1])
