"""Helpers of the tests of the paged 8-bit cache: random caches on both sides, and how far results may be from 64 bits."""
import numpy as np
import torch

from oracle import cache8

EPS = 2.0 ** -24                 # half a step of fp32, relative
NAN_CODE = 127


def normal(rng, *shape):
    return rng.standard_normal(shape).astype(np.float32)


def bf16(x):
    """float32 array rounded to bf16."""
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16).float().numpy()


def make(rng, lengths, kv, d, spare=3, width=None, junk=False):
    """Random caches: oracle side.  Pages in random order; slots behind an end hold codes too (junk: any byte, NaN among them)."""
    pages = [-(-max(n, 0) // 64) for n in lengths]
    width = max(max(pages), 1) + 1 if width is None else width
    total = sum(min(p, width) for p in pages) + spare
    ids = rng.permutation(total)
    table, at = np.full((len(lengths), width), -7, np.int32), 0
    for s, p in enumerate(pages):
        p = min(p, width)
        table[s, :p] = ids[at:at + p]
        at += p
    k = cache8.encode(np.clip(normal(rng, total, kv, 64, d) * 40, -448, 448))
    v = cache8.encode(np.clip(normal(rng, total, kv, d, 64) * 40, -448, 448))
    if junk:
        used = np.zeros((total, 64), bool)
        for s, n in enumerate(lengths):
            for i in range(min(max(n, 0), width * 64)):
                used[table[s, i // 64], i % 64] = True
        k = np.where(used[:, None, :, None], k, rng.integers(0, 256, k.shape).astype(np.uint8))
        v = np.where(used[:, None, None, :], v, rng.integers(0, 256, v.shape).astype(np.uint8))
        k[~used[:, None, :, None] & (rng.random(k.shape) < 0.2)] = NAN_CODE
        v[~used[:, None, None, :] & (rng.random(v.shape) < 0.2)] = NAN_CODE
    scale = 2.0 ** rng.integers(-7, -3, (total, kv, 2)).astype(np.float32)
    return cache8.Cache(k, v, scale.astype(np.float32), table, np.asarray(lengths, np.int32))


def to_gpu(amd, c, table_pad=0):
    code = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda().view(torch.float8_e4m3fn)
    table = torch.from_numpy(np.pad(c.table, ((0, 0), (0, table_pad)), constant_values=-3)).cuda()[:, :c.table.shape[1]]
    return amd.Fp8Cache(code(c.k), code(c.v), torch.from_numpy(c.scale.copy()).cuda(), table, torch.from_numpy(c.length.copy()).cuda())


def starts_of(rows):
    return np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)


def codes(t):
    return t.view(torch.uint8).cpu().numpy()


def same_codes(got, want):
    """Equal as values: a zero's sign does not count, NaN equals NaN."""
    return np.array_equal(cache8.DECODE[got], cache8.DECODE[want], equal_nan=True)


def check_attention(got, lse, want, want_lse, mass, size, d, n):
    """Derived bound: a score is a sum of d exact products in fp32, off by (d + 2) steps of its magnitudes, and its base-2 form by two
    more, so a weight by e = exp(that) - 1 and the hardware exponential's 2^-23, relative; weights and their sum each.  Weights for the product with
    the values are rounded to bf16 (2^-8), sums over n entries are in fp32, the result is bf16 (2^-8)."""
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    worst = np.where(np.isfinite(size), size, 0)
    off = np.expm1((d + 5) * EPS * 1.05 * worst) + 4 * EPS * 2 + (n + 8) * EPS
    bound = (2.0 ** -8 + 2.2 * off[..., None]) * mass * 1.01 + 2.0 ** -8 * np.abs(want) + 1e-37
    assert (np.abs(got - want) <= bound)[fine].all(), float((np.abs(got - want) / bound)[fine].max())
    if lse is not None:
        assert np.array_equal(np.isnan(lse), np.isnan(want_lse)) and np.array_equal(np.isneginf(lse), np.isneginf(want_lse))
        there = np.isfinite(want_lse)
        room = off + 8 * EPS * (np.abs(np.where(there, want_lse, 0)) + 1 + worst)
        with np.errstate(invalid="ignore"):
            assert (np.abs(lse - want_lse) <= room)[there].all()


# (rows, lengths, heads, kv): prompts, drafts and single tokens in one batch, so many rows that sequences of few and of many have kernels of their own
MIXED = [([600, 1, 0, 5, 40, 41, 1], [700, 900, 0, 77, 300, 41, 2000], 8, 2), ([150, 3, 8, 9, 0, 1], [150, 500, 1000, 9, 64, 640], 40, 2),
         ([1] * 60 + [500], [130] * 60 + [600], 8, 2), ([1050] + [1] * 15, [1050] + [65] * 15, 32, 16), ([0, 257, 0, 257, 32, 33, 0], [9, 300, 0, 257, 90, 600, 1], 8, 2)]
