"""Oracle: rows truncated by top-k, top-p and min-p, and draws from them (test infrastructure only).

With z = logit * logit_scale / temperature and w = exp(z - max z), ids in the order of falling logits, equal ones by rising id:
of the first k ids the shortest prefix that holds at least top_p of their mass (at least one id), and of that the ids with
w >= min_p.  Everything in float64; the parameters are the float32 values the library is given.
"""
from __future__ import annotations

import numpy as np

from . import sampling


def weights(logits, temperature=1.0, logit_scale=1.0, top_k=0, top_p=1.0, min_p=0.0) -> np.ndarray:
    """w of the kept ids, 0 elsewhere; one-hot at the lowest arg-max if temperature == 0; NaN without a distribution."""
    x = np.asarray(logits, dtype=np.float32).astype(np.float64)
    f = lambda v: float(np.float32(v))
    out = np.zeros_like(x)
    if temperature == 0.0:
        y = np.where(np.isnan(x), -np.inf, x)
        out[int(np.argmax(y))] = 1.0
        return out
    if not np.isfinite(x).any() or np.isnan(x).any() or (x == np.inf).any():
        return np.full_like(x, np.nan)
    w = np.exp((x - x.max()) * (f(logit_scale) / f(temperature)))
    order = np.argsort(-x, kind="stable")
    if 0 < top_k < x.size:
        order = order[:top_k]
    if f(top_p) < 1.0:
        mass = np.cumsum(w[order])
        order = order[:int(np.argmax(mass >= f(top_p) * mass[-1])) + 1]
    order = order[w[order] >= f(min_p)]
    out[order] = w[order]
    return out


def row(logits, u: float, **how):
    """(token, distribution); token -1 and NaN without a distribution."""
    w = weights(logits, **how)
    if np.isnan(w).any():
        return -1, w
    return sampling.sample(w, min(max(u, 0.0), 1.0 - 2.0 ** -53)), w / w.sum()
