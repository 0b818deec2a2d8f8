"""Eviction from the paged 8-bit cache by the weight of its entries, bit for bit (run with -m gpu)."""
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


def _weights(rng, kind, shape):
    w = np.exp(2 * normal(rng, *shape)).astype(np.float32)
    if kind == "few":
        w = np.round(w).astype(np.float32)                   # many equal ones
    elif kind == "zero":
        w = np.where(rng.random(shape) < 0.9, 0, w).astype(np.float32)
    elif kind == "flat":
        w[:] = 0.25
    elif kind == "odd":
        for x in (np.nan, np.inf, -np.inf, -0.0, 0.0, -1.5, -np.nan, 1e-45):
            w[rng.random(shape) < 0.08] = x
    return w


def _run(lengths, kv, d, budget, sinks, recent, kind="any", seed=1, change=None, one_pool=False):
    amd, rng = _amd(), np.random.default_rng(seed)
    c = make(rng, lengths, kv, d, junk=True)
    width = -(-budget // 64) + 1
    to = make(rng, [64 * width] * len(lengths), kv, d, width=width, junk=True)
    if change:
        change(c, to)
    weight = _weights(rng, kind, (len(lengths), kv, c.table.shape[1] * 64 + 1))
    if one_pool:                                             # pages of the same pool, another table
        n = c.k.shape[0]
        c.k, c.v, c.scale = (np.concatenate([a, b]) for a, b in ((c.k, to.k), (c.v, to.v), (c.scale, to.scale)))
        to.k, to.v, to.scale = c.k, c.v, c.scale
        to.table = to.table + n
        g = to_gpu(amd, c)
        o = amd.Fp8Cache(g.k, g.v, g.scale, torch.from_numpy(to.table).cuda(), torch.from_numpy(to.length).cuda())
    else:
        g, o = to_gpu(amd, c, table_pad=1), to_gpu(amd, to, table_pad=2)
    left = torch.full((len(lengths), kv, budget + 2), -5.0, device="cuda")
    kept = amd.evict_fp8(g, torch.from_numpy(weight).cuda(), o, budget, sinks, recent, to_weight=left)
    want, want_left = cache8.evict(c, weight, to, budget, sinks, recent)
    assert np.array_equal(kept.cpu().numpy(), want)
    got_left = left.cpu().numpy()
    assert np.array_equal(np.where(want >= 0, got_left[..., :budget], 0), want_left, equal_nan=True)
    assert (got_left[..., :budget][want < 0] == -5).all() and (got_left[..., budget:] == -5).all()
    assert np.array_equal(o.length.cpu().numpy(), to.length)
    assert np.array_equal(o.scale.cpu().numpy(), to.scale)
    assert same_codes(codes(o.k), to.k) and same_codes(codes(o.v), to.v)
    return kept


@pytest.mark.parametrize("kind", ["any", "few", "zero", "flat", "odd"])
@pytest.mark.parametrize("lengths,budget,sinks,recent", [
    ([300, 200, 129], 128, 4, 32), ([300], 100, 0, 0), ([500, 64, 101], 65, 0, 65), ([200], 64, 64, 0), ([130], 1, 0, 0),
    ([130], 1, 1, 0), ([65], 64, 1, 62), ([1500], 700, 10, 300), ([64, 63, 1, 0], 64, 4, 4), ([5000, 2049], 2048, 4, 1)])
def test_what_is_kept(lengths, budget, sinks, recent, kind):
    _run(lengths, 2, 64, budget, sinks, recent, kind)


@pytest.mark.parametrize("kv,d", [(1, 128), (5, 128), (3, 64)])
@pytest.mark.parametrize("one_pool", [False, True])
def test_codes_move_to_new_scales(kv, d, one_pool):
    """Source pages of scales up to 2^12 apart: codes become denormal, or nothing."""
    def spread(c, to):
        c.scale[:] = 2.0 ** np.random.default_rng(2).integers(-10, 3, c.scale.shape)
    _run([700, 333], kv, d, 200, 4, 20, change=spread, one_pool=one_pool)


def test_scales_at_their_ends():
    def ends(c, to):
        c.scale[::2], c.scale[1::2] = 2.0 ** -100, 2.0 ** 112
    _run([300], 2, 128, 130, 4, 20, change=ends)


def test_nan_keys_zeros_and_pages_that_are_none():
    def odd(c, to):
        c.k[c.table[0, 1], 0, 3:9] = 127
        c.v[c.table[0, 1], 0, :, 3:9] = 0
        c.k[c.table[0, 0]] = 0
        c.v[c.table[0, 0]] = 0x80
        c.table[0, 2] = -1
        c.table[1, 0] = 10 ** 6
        to.table[1, 1] = -1
        to.table[0, 0] = 2 ** 31 - 1
    _run([300, 300], 2, 128, 200, 4, 20, change=odd)


def test_lengths_beyond_the_table_and_negative_ones():
    def change(c, to):
        c.length[:] = [64 * c.table.shape[1] + 1, 2 ** 31 - 1, 150]
    _run([150, 150, 150], 2, 64, 100, 4, 20, change=change)
