"""Rows rotated, rounded to e4m3 and stored in pages, against 64 bits (run with -m gpu)."""
import numpy as np
import pytest
import torch

from oracle import cache8
from tests.cache8 import EPS, bf16, codes, make, normal, same_codes, starts_of, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _rows(rng, n, kv, d, dtype):
    x = normal(rng, n, kv, d) * np.exp(normal(rng, n, kv, 1))
    return x if dtype is torch.float32 else bf16(x)


def _gpu(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda().to(dtype)


def _same(g, c):
    """Codes, scales and everything else that was there."""
    assert np.array_equal(g.scale.cpu().numpy(), c.scale)
    assert same_codes(codes(g.k), c.k) and same_codes(codes(g.v), c.v)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kv,d", [(1, 64), (3, 128), (8, 128)])
@pytest.mark.parametrize("rows,lengths", [([1], [1]), ([1], [64]), ([1], [65]), ([2], [65]), ([64], [64]), ([64], [100]), ([200], [333]),
                                          ([1, 0, 7, 65], [5, 9, 7, 130]), ([3, 130], [67, 130])])
def test_codes_without_rotation(rows, lengths, kv, d, dtype):
    """Powers of two scale exactly: codes and scales are those of the definition bit for bit, and nothing else changes."""
    amd, rng = _amd(), np.random.default_rng(sum(rows) + kv)
    c = make(rng, lengths, kv, d)
    g = to_gpu(amd, c, table_pad=1)
    start = starts_of(rows)
    n = int(start[-1])
    k, v = _rows(rng, n + 2, kv, d, dtype), _rows(rng, n + 2, kv, d, dtype)
    c.append(start, k, v)
    assert amd.append_fp8(g, _gpu(k, dtype), _gpu(v, dtype), rows=torch.from_numpy(start).cuda()) is None
    _same(g, c)


@pytest.mark.parametrize("d", [64, 128])
def test_one_by_one_scales_only_grow(d):
    """Tokens that grow move the codes before them; smaller ones keep the scale."""
    amd, rng = _amd(), np.random.default_rng(7)
    c = make(rng, [0, 0], 2, d, spare=6, width=2)
    c.table[:] = [[0, 1], [2, 3]]
    g = to_gpu(amd, c)
    for i in range(70):
        level = 2.0 ** (rng.integers(-12, 12) if i % 3 else -20)
        k, v = bf16(normal(rng, 2, 2, d) * level), bf16(normal(rng, 2, 2, d) / level)
        c.length += 1
        g.length += 1
        c.append([0, 1, 2], k, v)
        amd.append_fp8(g, _gpu(k, torch.bfloat16), _gpu(v, torch.bfloat16))
        _same(g, c)


def test_a_cut_sequence_goes_on():
    """After a rollback rows take the places of those that were dropped; a page begun anew forgets its scale."""
    amd, rng = _amd(), np.random.default_rng(8)
    c = make(rng, [60], 2, 128, spare=4, width=3)
    c.table[0] = [0, 1, 2]
    g = to_gpu(amd, c)
    for length, m in ((70, 10), (66, 3), (65, 1), (80, 16), (62, 2), (130, 68)):
        k, v = bf16(normal(rng, m, 2, 128) * 50), bf16(normal(rng, m, 2, 128))
        c.length[:], g.length[:] = length, length
        c.append([0, m], k, v)
        amd.append_fp8(g, _gpu(k, torch.bfloat16), _gpu(v, torch.bfloat16))
        _same(g, c)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (9, 3, 128), (64, 8, 128)])
@pytest.mark.parametrize("theta,far", [(10000.0, 0), (500000.0, 100000), (10000.0, 2 ** 30)])
def test_rotation(heads, kv, d, theta, far, dtype):
    """q: rotated in fp32 by an angle off by less than 2^-21, rounded to bf16.  k: the code's value within half a step (2^-4 of it, or
    2^-10 of the scale where it is denormal); the scale by the largest of the rotated values, which the test keeps off its borders."""
    amd, rng = _amd(), np.random.default_rng(heads + far)
    rows, lengths = [1, 70, 3], [40, 70, 131]
    c = make(rng, lengths, kv, d)
    g = to_gpu(amd, c)
    start = starts_of(rows)
    n = int(start[-1])
    k, v, q = (_rows(rng, n, h, d, dtype) for h in (kv, kv, heads))
    position = np.array([far + 5, far, far + 77], np.int32)
    at = np.concatenate([p + np.arange(m) for p, m in zip(position if far else np.array(lengths) - rows, rows)])
    got = amd.append_fp8(g, _gpu(k, dtype), _gpu(v, dtype), _gpu(q, dtype), torch.from_numpy(start).cuda(), theta,
                         torch.from_numpy(position).cuda() if far else None)
    before = cache8.Cache(c.k, c.v, c.scale, c.table, c.length)
    c.append(start, k, v, theta, position if far else None)
    want = cache8.rotate(q.astype(np.float64), at, theta)
    half = d // 2
    both = np.abs(q).astype(np.float64)
    both = np.concatenate([both[..., :half] + both[..., half:]] * 2, -1)
    slack = both * (2.0 ** -21 + 3 * EPS)
    assert got.dtype is torch.bfloat16 and got.shape == (n, heads, d)
    assert (np.abs(got.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 1.01 * slack + 1e-38).all()
    assert np.array_equal(g.scale.cpu().numpy()[..., 1], c.scale[..., 1]) and same_codes(codes(g.v), c.v)
    scale = g.scale.cpu().numpy()
    apart = scale[..., 0] != c.scale[..., 0]
    assert apart.mean() < 1e-2                              # only where a largest value lies on a border
    kr = cache8.rotate(k.astype(np.float64), at, theta)
    both = np.abs(k).astype(np.float64)
    both = np.concatenate([both[..., :half] + both[..., half:]] * 2, -1) * (2.0 ** -21 + 3 * EPS)
    mine = codes(g.k)
    touched = np.zeros(mine.shape, bool)
    for s, (m, length) in enumerate(zip(rows, lengths)):
        for j in range(m):
            p = length - m + j
            page, row = c.table[s, p // 64], start[s] + j
            value = cache8.DECODE[mine[page, :, p % 64]] * scale[page, :, 0, None]
            assert (np.abs(value - kr[row]) <= 2.0 ** -4 * np.abs(kr[row]) + 2.0 ** -10 * scale[page, :, 0, None] + 1.1 * both[row]).all()
            touched[page, :, :p % 64 + 1] = True
    assert np.array_equal(mine[~touched], before.k[~touched])


def test_values_that_are_not_finite():
    """Their token gets a NaN key and the value 0 in that head; scales, other tokens and other heads do not see them."""
    amd, rng = _amd(), np.random.default_rng(5)
    c = make(rng, [70], 4, 128)
    g = to_gpu(amd, c)
    k, v = normal(rng, 70, 4, 128), normal(rng, 70, 4, 128)
    k[3, 0, 5], v[10, 1, 100], k[64, 2, 127], v[69, 3, 0], v[20, 0, 1] = np.nan, np.inf, -np.inf, 2.0 ** 120, -np.nan
    k[30, 3, :] = 1.9999 * 2.0 ** 119                       # finite still
    c.append([0, 70], k, v)
    with np.errstate(invalid="ignore"):
        amd.append_fp8(g, _gpu(k, torch.float32), _gpu(v, torch.float32))
    _same(g, c)
    assert np.isnan(cache8.DECODE[codes(g.k)[c.table[0, 0], 0, 3]]).all() and not np.isnan(cache8.DECODE[codes(g.v)]).any()


def test_tiny_and_zero_values():
    amd, rng = _amd(), np.random.default_rng(6)
    c = make(rng, [3, 3, 3], 1, 64)
    g = to_gpu(amd, c)
    k, v = np.zeros((9, 1, 64), np.float32), normal(rng, 9, 1, 64)
    v[3:6] *= 2.0 ** -120
    v[6:] = np.float32(1e-45)
    k[5, 0, 7] = 448 * 2.0 ** -100
    k[8, 0, 9] = np.nextafter(np.float32(448 * 2.0 ** -3), np.float32(1e9))
    c.append([0, 3, 6, 9], k, v)
    amd.append_fp8(g, _gpu(k, torch.float32), _gpu(v, torch.float32))
    _same(g, c)


def test_nothing_is_stored_where_there_is_no_page():
    """Page ids out of range, rows in front of entry 0, lengths beyond the table: q is rotated all the same."""
    amd, rng = _amd(), np.random.default_rng(10)
    c = make(rng, [100, 2, 100, 0], 2, 64, width=2)
    c.table[0] = [-1, 10 ** 9]
    c.length[2] = 129
    c.length[3] = 2 ** 31 - 1
    g = to_gpu(amd, c)
    start = starts_of([50, 5, 3, 4])
    k, v, q = (_rows(rng, 62, h, 64, torch.bfloat16) for h in (2, 2, 4))
    c.append(start, k, v)
    got = amd.append_fp8(g, *(_gpu(x, torch.bfloat16) for x in (k, v, q)), rows=torch.from_numpy(start).cuda())
    _same(g, c)
    assert np.array_equal(got.float().cpu().numpy(), q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_slices_of_one_projection_and_q_in_place(dtype):
    amd, rng = _amd(), np.random.default_rng(11)
    heads, kv, d, n = 4, 2, 64, 7
    c = make(rng, [n], kv, d)
    wide = _gpu(_rows(rng, n, 1, (heads + 2 * kv) * d + 3, dtype), dtype)[:, 0, 1:]          # odd addresses and strides
    q, k, v = (wide[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
    g, g2 = to_gpu(amd, c), to_gpu(amd, c)
    a = amd.append_fp8(g, k, v, q, theta=100.0)
    b = amd.append_fp8(g2, k.contiguous(), v.contiguous(), q.contiguous(), theta=100.0)
    assert torch.equal(a, b) and torch.equal(g.k.view(torch.uint8), g2.k.view(torch.uint8)) and torch.equal(g.v.view(torch.uint8), g2.v.view(torch.uint8))
    if dtype is torch.bfloat16:
        own = q.contiguous()
        amd.check(amd.load_library().spec_append_quant(g.ref, k.data_ptr(), k.stride(0), v.data_ptr(), v.stride(0), amd.SPEC_BF16, None, n,
                                                       own.data_ptr(), heads * d, heads, 100.0, None, own.data_ptr(),
                                                       torch.cuda.current_stream().cuda_stream))
        assert torch.equal(own, a)
