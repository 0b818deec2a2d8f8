"""Eviction where the scales of old and new pages are further apart than fp32's exponents, bit for bit (run with -m gpu)."""
import numpy as np
import pytest
import torch

from oracle import cache8
from tests.cache8 import codes, make, normal, same_codes, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _evict(change, kv, d, lengths=(300, 130), budget=130, sinks=4, recent=20):
    amd, rng = _amd(), np.random.default_rng(3)
    c = make(rng, lengths, kv, d)
    to = make(rng, [192] * len(lengths), kv, d, width=3)
    change(c, rng)
    weight = rng.random((len(lengths), kv, c.table.shape[1] * 64)).astype(np.float32)
    g, o = to_gpu(amd, c), to_gpu(amd, to)
    kept = amd.evict_fp8(g, torch.from_numpy(weight).cuda(), o, budget, sinks, recent)
    want, _ = cache8.evict(c, weight, to, budget, sinks, recent)
    assert np.array_equal(kept.cpu().numpy(), want) and np.array_equal(o.scale.cpu().numpy(), to.scale)
    assert same_codes(codes(o.k), to.k) and same_codes(codes(o.v), to.v)
    return to


def _zeros(rng, shape):
    return np.where(rng.random(shape) < 0.5, 0, 0x80).astype(np.uint8)


@pytest.mark.parametrize("kv,d", [(2, 64), (3, 128)])
@pytest.mark.parametrize("exponent", [27, 28, 60, 112])
def test_zeros_of_pages_with_large_scales(exponent, kv, d):
    """New pages of nothing but zeros have the least scale, 2^-100; zeros stay zeros."""
    def change(c, rng):
        c.k, c.v = _zeros(rng, c.k.shape), _zeros(rng, c.v.shape)
        c.scale[:] = 2.0 ** exponent
    to = _evict(change, kv, d)
    assert (cache8.DECODE[to.k[to.table[0, :2]]] == 0).all() and (to.scale[to.table[0, 0]] == 2.0 ** -100).all()


@pytest.mark.parametrize("kv,d", [(2, 64), (3, 128)])
def test_zeros_beside_small_values(kv, d):
    """Every other page holds zeros at 2^112, the others ordinary codes at 2^-50: zeros and codes share the new pages."""
    def change(c, rng):
        for s in range(2):
            for i, page in enumerate(c.table[s, :-1]):
                if i % 2:
                    c.k[page], c.v[page], c.scale[page] = _zeros(rng, c.k[page].shape), _zeros(rng, c.v[page].shape), 2.0 ** 112
                else:
                    c.scale[page] = 2.0 ** -50
    _evict(change, kv, d)


@pytest.mark.parametrize("d", [64, 128])
def test_nan_keys_beside_zeros_of_a_large_scale(d):
    """NaN keys stay NaN keys, and nothing else becomes one."""
    def change(c, rng):
        c.k, c.v = _zeros(rng, c.k.shape), _zeros(rng, c.v.shape)
        c.scale[:] = 2.0 ** 100
        c.k[:, :, 7] = 127
    _evict(change, 2, d)


@pytest.mark.parametrize("d", [64, 128])
def test_a_large_token_that_is_evicted(d):
    """Its page's other tokens are rounded to 0 and stay so, and the rows that see them are finite."""
    amd, rng = _amd(), np.random.default_rng(5)
    cache = lambda ids: amd.Fp8Cache(torch.zeros(2, 1, 64, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
                                     torch.zeros(2, 1, d, 64, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
                                     torch.zeros(2, 1, 2, device="cuda"), torch.tensor([ids], dtype=torch.int32, device="cuda"),
                                     torch.tensor([64], dtype=torch.int32, device="cuda"))
    g, o = cache([1]), cache([0])
    k, v = normal(rng, 64, 1, d), normal(rng, 64, 1, d)
    k[7, 0, 3], v[7, 0, 5] = 2.0 ** 40, -2.0 ** 40
    amd.append_fp8(g, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda())
    weight = torch.rand(1, 1, 64, device="cuda") + 1
    weight[0, 0, 7] = 0
    kept = amd.evict_fp8(g, weight, o, 63)
    assert (kept[0, 0].cpu().numpy() == np.delete(np.arange(64), 7)).all()
    assert ((codes(o.k)[0, 0, :63] & 127) == 0).all() and ((codes(o.v)[0, 0, :, :63] & 127) == 0).all()
    out, lse = amd.attend_fp8(o, torch.from_numpy(normal(rng, 1, 4, d)).cuda().to(torch.bfloat16), want_lse=True)
    assert (out == 0).all() and ((lse - float(np.log(63))).abs() <= 1e-6).all()
