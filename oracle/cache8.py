"""A paged cache of keys and values in e4m3 in plain NumPy, in 64 bits: append, attention, weights of its entries, eviction."""
from __future__ import annotations

import math

import numpy as np

PAGE = 64
LEAST = -100


def _decode():
    t = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        t[c] = np.nan if c & 127 == 127 else -x if c & 128 else x
    return t


DECODE = _decode()


def encode(x):
    """e4m3 codes of values up to 448, nearest, ties to even; a NaN is 0x7f."""
    x = np.asarray(x, np.float64)
    step = 2.0 ** (np.maximum(np.frexp(x)[1] - 1, -6) - 3.0)
    v = np.abs(np.rint(x / step) * step)
    code = np.searchsorted(DECODE[:127], np.where(np.isnan(v), 0, v)).astype(np.uint8)
    return np.where(np.isnan(v), 127, code | (np.signbit(x) << 7)).astype(np.uint8)


def exponent(top):
    e = LEAST
    while top > 448.0 * 2.0 ** e:
        e += 1
    return e


def rotate(x, pos, theta):
    """[rows][heads][d] by positions [rows]."""
    if not theta:
        return x
    half = x.shape[-1] // 2
    angle = np.asarray(pos, np.float64)[:, None, None] * theta ** (-np.arange(half) / half)
    a, b = x[..., :half], x[..., half:]
    return np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], -1)


class Cache:
    """k [pages][heads][64][d], v [pages][heads][d][64] codes, scale [pages][heads][2], table [seqs][width], length [seqs]."""

    def __init__(self, k, v, scale, table, length):
        self.k, self.v, self.scale, self.table, self.length = (np.array(a) for a in (k, v, scale, table, length))

    def entries(self, s, h, n=None):
        """Keys and values [n][d] of a sequence's head."""
        n = int(self.length[s]) if n is None else n
        k, v = np.empty((n, self.k.shape[3])), np.empty((n, self.k.shape[3]))
        for i in range(0, n, PAGE):
            page, m = int(self.table[s, i // PAGE]), min(PAGE, n - i)
            if not 0 <= page < self.k.shape[0]:
                k[i:i + m], v[i:i + m] = np.nan, 0
                continue
            k[i:i + m] = DECODE[self.k[page, h, :m]] * float(self.scale[page, h, 0])
            v[i:i + m] = DECODE[self.v[page, h, :, :m]].T * float(self.scale[page, h, 1])
        return k, v

    def append(self, starts, k, v, theta=0.0, position=None):
        for s in range(len(self.length)):
            a, b, n = int(starts[s]), int(starts[s + 1]), int(self.length[s])
            if n > self.table.shape[1] * PAGE or a == b:
                continue
            first = n - (b - a)
            pos = (first if position is None else int(position[s])) + np.arange(b - a)
            kr, vr = rotate(np.asarray(k[a:b], np.float64), pos, theta), np.asarray(v[a:b], np.float64)
            for h in range(kr.shape[1]):
                bad = ~((np.abs(kr[:, h]) < 2.0 ** 120).all(1) & (np.abs(vr[:, h]) < 2.0 ** 120).all(1))
                kh, vh = np.where(bad[:, None], np.nan, kr[:, h]), np.where(bad[:, None], 0.0, vr[:, h])
                for p in range(max(first, 0) // PAGE, -(-n // PAGE)):
                    page, lo, hi = int(self.table[s, p]), max(first, p * PAGE), min(n, (p + 1) * PAGE)
                    if not 0 <= page < self.k.shape[0]:
                        continue
                    for w, x in ((0, kh[lo - first:hi - first]), (1, vh[lo - first:hi - first])):
                        codes = self.k[page, h] if w == 0 else self.v[page, h].T
                        top = np.abs(np.where(np.isnan(x), 0, x)).max()
                        e, slot = exponent(top), lo - p * PAGE
                        if slot:
                            was = math.frexp(float(self.scale[page, h, w]))[1] - 1
                            e = max(e, was)
                            if e != was:
                                codes[:slot] = encode(DECODE[codes[:slot]] * 2.0 ** (was - e))
                        codes[slot:slot + hi - lo] = encode(x * 2.0 ** -e)
                        self.scale[page, h, w] = 2.0 ** e


def visible(first, rows, n, window, sinks):
    """[rows][n]: which entries row j, at entry first + j, sees."""
    pos, p = first + np.arange(rows)[:, None], np.arange(n)[None]
    return (p <= pos) & ((p > pos - window) | (p < sinks) if window else True)


def attend(cache, starts, q, scale, window=0, sinks=0):
    """(out, lse, sum of p |v|, largest sum of |q| |k| * scale that a row sees) of rows [n][heads][d] in 64 bits; rows of no sequence 0."""
    n_rows, heads, d = q.shape
    kv = cache.k.shape[1]
    out, lse = np.zeros(q.shape), np.zeros((n_rows, heads))
    mass, size = np.zeros(q.shape), np.zeros((n_rows, heads))
    for s in range(len(cache.length)):
        a, b = int(starts[s]), int(starts[s + 1])
        n = int(cache.length[s])
        if n > cache.table.shape[1] * PAGE:
            out[a:b], lse[a:b] = np.nan, np.nan
            continue
        see = visible(n - (b - a), b - a, n, window, sinks)
        for h in range(heads):
            k, v = cache.entries(s, h // (heads // kv))
            if not n:
                lse[a:b, h] = -np.inf
                continue
            with np.errstate(invalid="ignore", divide="ignore"):
                x = np.where(see, q[a:b, h].astype(np.float64) @ k.T * scale, -np.inf)
                top = x.max(1, keepdims=True)
                p = np.exp(x - np.where(see.any(1, keepdims=True), top, 0))
                total = p.sum(1, keepdims=True)
                any_seen = see.any(1, keepdims=True)
                out[a:b, h] = np.where(any_seen, p @ v / total, 0)
                mass[a:b, h] = np.where(any_seen, p @ np.abs(v) / total, 0)
                lse[a:b, h] = np.where(any_seen, top + np.log(total), -np.inf)[:, 0]
                size[a:b, h] = np.where(see, np.abs(q[a:b, h].astype(np.float64)) @ np.abs(k).T * scale, 0).max(1)
    return out, lse, mass, size


def weigh(cache, starts, q, lse, weight, scale, window=0, sinks=0):
    """(weight, added weight times the largest exponent's size) after the rows' attention."""
    weight, heads, kv = np.array(weight, np.float64), q.shape[1], cache.k.shape[1]
    G = heads // kv
    slack = np.zeros(weight.shape)
    for s in range(len(cache.length)):
        a, b, n = int(starts[s]), int(starts[s + 1]), int(cache.length[s])
        if n > cache.table.shape[1] * PAGE or a == b:
            continue
        see = visible(n - (b - a), b - a, n, window, sinks)
        for h in range(kv):
            weight[s, h, max(n - (b - a), 0):n] = 0
            k = cache.entries(s, h)[0]
            for g in range(h * G, (h + 1) * G):
                x = q[a:b, g].astype(np.float64) @ k.T * scale
                size = np.abs(q[a:b, g].astype(np.float64)) @ np.abs(k).T * scale + np.abs(lse[a:b, g])[:, None]
                p = np.where(see, np.exp(np.where(see, x - lse[a:b, g].astype(np.float64)[:, None], 0)), 0)
                weight[s, h, :n] += p.sum(0)
                slack[s, h, :n] += np.where(see, p * size, 0).sum(0)
    return weight, slack


def evict(cache, weight, to, budget, sinks, recent):
    """Fills `to`; returns kept [seqs][heads][budget] and their weights (0 behind the last)."""
    kv, d = cache.k.shape[1], cache.k.shape[3]
    kept, left = np.full((len(cache.length), kv, budget), -1, np.int32), np.zeros((len(cache.length), kv, budget), np.float32)
    for s in range(len(cache.length)):
        n = int(cache.length[s])
        if n > cache.table.shape[1] * PAGE:
            to.length[s] = (2 ** 31 - 1) // 2
            continue
        to.length[s] = min(n, budget)
        for h in range(kv):
            keep = list(range(n))
            if n > budget:
                rank = {p: -np.inf if np.isnan(weight[s, h, p]) else float(weight[s, h, p]) for p in range(sinks, n - recent)}
                rank = {p: (r, not np.isnan(weight[s, h, p])) for p, r in rank.items()}          # a NaN is below -inf
                middle = sorted(rank, key=lambda p: (-rank[p][0], -rank[p][1], p))[:budget - sinks - recent]
                keep = sorted(list(range(sinks)) + middle + list(range(n - recent, n)))
            kept[s, h, :len(keep)], left[s, h, :len(keep)] = keep, weight[s, h, keep]
            k, v = cache.entries(s, h)
            for i in range(0, len(keep), PAGE):
                part, page = keep[i:i + PAGE], int(to.table[s, i // PAGE])
                if not 0 <= page < to.k.shape[0]:
                    continue
                for w, x in ((0, k[part]), (1, v[part])):
                    e = exponent(np.abs(np.where(np.isnan(x), 0, x)).max())
                    codes = to.k[page, h] if w == 0 else to.v[page, h].T
                    codes[:len(part)] = encode(x * 2.0 ** -e)
                    to.scale[page, h, w] = 2.0 ** e
    return kept, left
