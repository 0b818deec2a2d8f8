"""The oracle of the paged 8-bit cache against itself and against torch: codes, scales, rotation, attention, weights, eviction."""
import math

import numpy as np
import pytest
import torch

from oracle import cache8
from tests.cache8 import make, normal, starts_of


def test_codes_are_torchs():
    x = np.concatenate([normal(np.random.default_rng(0), 20000) * s for s in (1e-4, 1e-2, 1, 60)])
    x = np.clip(np.concatenate([x, [0.0, -0.0, 448, -448, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9, 17, 19, np.nan]]), -448, 448).astype(np.float32)
    t = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(cache8.encode(x) & 127, t & 127) and np.array_equal(cache8.encode(x)[~np.isnan(x)], t[~np.isnan(x)])
    assert np.array_equal(cache8.DECODE, torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)


def test_exponents_are_the_least():
    for top in (448.0, 448.0001, 449, 224, 224.0001, 1.0, 1.75, 1.7500001, 3e30, 448 * 2.0 ** -100, 1e-40, 0.0):
        e = cache8.exponent(top)
        assert top <= 448 * 2.0 ** e and (e == -100 or top > 448 * 2.0 ** (e - 1))


def test_rotation_keeps_norms_and_relative_positions():
    rng = np.random.default_rng(1)
    x, y = normal(rng, 1, 1, 64), normal(rng, 1, 1, 64)
    a, b = cache8.rotate(x, [7], 10000.0), cache8.rotate(y, [19], 10000.0)
    c, d = cache8.rotate(x, [1007], 10000.0), cache8.rotate(y, [1019], 10000.0)
    assert abs((a ** 2).sum() - (x.astype(np.float64) ** 2).sum()) < 1e-10 and abs((a * b).sum() - (c * d).sum()) < 1e-9
    z = cache8.rotate(x, [3], 10000.0)[0, 0]                # element 0 turns with element 32, by 3
    assert math.isclose(z[0], float(x[0, 0, 0]) * math.cos(3) - float(x[0, 0, 32]) * math.sin(3), rel_tol=1e-12)


def test_append_gives_back_what_it_was_given():
    rng = np.random.default_rng(2)
    c = make(rng, [0, 0], 2, 64, spare=9, width=3)
    c.table[:] = [[0, 5, 2], [4, 1, 3]]
    c.length[:] = [150, 70]
    k, v = normal(rng, 220, 2, 64), normal(rng, 220, 2, 64)
    c.append([0, 150, 220], k, v)
    for s, (a, b) in enumerate(((0, 150), (150, 220))):
        for h in range(2):
            for got, want in zip(c.entries(s, h), (k[a:b, h], v[a:b, h])):
                step = np.concatenate([np.full(64, 2.0 ** cache8.exponent(np.abs(want[i:i + 64]).max())) for i in range(0, b - a, 64)])[:b - a, None]
                assert (np.abs(got - want) <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * step)).all()


def test_one_by_one_is_all_at_once_but_for_denormal_codes():
    rng = np.random.default_rng(3)
    k, v = normal(rng, 64, 1, 64), normal(rng, 64, 1, 64)
    one, all_ = (make(rng, [0], 1, 64, width=1) for _ in range(2))
    for c in (one, all_):
        c.table[0, 0], c.k[:], c.v[:] = 0, 0, 0
    for i in range(64):
        one.length[0] = i + 1
        one.append([0, 1], k[i:i + 1], v[i:i + 1])
    all_.length[0] = 64
    all_.append([0, 64], k, v)
    assert np.array_equal(one.scale[0], all_.scale[0])
    a, b = cache8.DECODE[one.k[0]], cache8.DECODE[all_.k[0]]
    assert np.array_equal(a[np.abs(b) >= 2.0 ** -6], b[np.abs(b) >= 2.0 ** -6]) and np.abs(a - b).max() <= 2.0 ** -9


@pytest.mark.parametrize("window,sinks", [(0, 0), (5, 0), (5, 2), (1, 0)])
def test_attention_is_the_softmax_over_what_is_seen(window, sinks):
    rng = np.random.default_rng(4)
    c = make(rng, [20, 9], 2, 64)
    q = normal(rng, 7, 4, 64)
    out, lse, mass, _ = cache8.attend(c, [0, 4, 7], q, 0.125, window, sinks)
    k, v = c.entries(0, 1)
    for j in range(4):                                      # head 3 reads KV head 1
        p = 16 + j
        seen = [e for e in range(p + 1) if not window or e > p - window or e < sinks]
        w = np.exp(q[j, 3].astype(np.float64) @ k[seen].T * 0.125)
        assert np.allclose(out[j, 3], w @ v[seen] / w.sum(), rtol=1e-12) and math.isclose(lse[j, 3], math.log(w.sum()), rel_tol=1e-12)
    assert (mass >= np.abs(out) - 1e-12).all()


def test_weights_add_up_and_new_entries_begin_at_zero():
    rng = np.random.default_rng(5)
    c = make(rng, [30, 12], 2, 64)
    q = normal(rng, 8, 6, 64)
    start = starts_of([5, 3])
    _, lse, _, _ = cache8.attend(c, start, q, 0.125)
    w, _ = cache8.weigh(c, start, q, lse, np.full((2, 2, 128), 100.0), 0.125)
    assert np.allclose(w[0, :, :30].sum(1), 25 * 100 + 5 * 3) and np.allclose(w[1, :, :12].sum(1), 9 * 100 + 3 * 3)
    assert (w[0, :, 30:] == 100).all() and (w[0, :, 25:30] < 15).all()


def test_eviction_keeps_ends_and_the_heaviest():
    rng = np.random.default_rng(6)
    c, to = make(rng, [10, 3], 1, 64), make(rng, [64, 64], 1, 64, width=1)
    w = np.zeros((2, 1, 64), np.float32)
    w[0, 0, :10] = [9, 0, 5, 5, 1, 5, np.nan, -np.inf, 7, 0]
    kept, left = cache8.evict(c, w, to, 6, 1, 2)
    assert kept[0, 0].tolist() == [0, 2, 3, 5, 8, 9] and kept[1, 0].tolist() == [0, 1, 2, -1, -1, -1] and to.length.tolist() == [6, 3]
    assert np.array_equal(to.entries(0, 0, 6)[0][[1, 4]], c.entries(0, 0)[0][[2, 8]])
    kept, _ = cache8.evict(c, w, to, 9, 1, 1)
    assert kept[0, 0].tolist() == [0, 1, 2, 3, 4, 5, 7, 8, 9]          # -inf before NaN
