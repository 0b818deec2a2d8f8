"""Attention over a paged cache of keys and values in e4m3, its append, its entries' weights and eviction (see include/spec.h).

Argument marshalling only.  Every call runs on the current stream of the cache's device; the results are that device's.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from . import PAGE_TOKENS, SPEC_BF16, SPEC_F32, QuantCacheDesc, load_library
from .binding import call_on, need

_TYPES = {torch.float32: SPEC_F32, torch.bfloat16: SPEC_BF16}
E4M3 = torch.float8_e4m3fn


class Fp8Cache:
    """Keys and values of several sequences in pages of 64 entries; the tensors stay the caller's.

    k e4m3 [n_pages][heads][64][d]; v e4m3 [n_pages][heads][d][64]; scale fp32 [n_pages][heads][2] (of the keys, of the values);
    table int32 [n_seqs][max_pages] (any row stride); length int32 [n_seqs], the entries of every sequence with the rows of the
    calls that follow.  All contiguous but the table's rows, on one GPU.  How calls are split goes by the table's width, so that a table
    for the longest text is better given as far as it is needed, table[:, :n].  Their values may change at any time, as the calls on a stream see
    them; other tensors need another Fp8Cache."""

    __slots__ = ("k", "v", "scale", "table", "length", "device", "heads", "d", "n_seqs", "capacity", "desc", "ref", "sizes")

    def __init__(self, k: torch.Tensor, v: torch.Tensor, scale: torch.Tensor, table: torch.Tensor, length: torch.Tensor):
        need(k.is_cuda and k.dtype is E4M3 and k.dim() == 4 and k.shape[2] == PAGE_TOKENS and k.is_contiguous(),
             "k: contiguous e4m3 [n_pages][heads][64][d] on a GPU is wanted")
        n_pages, heads, _, d = k.shape
        need(v.dtype is E4M3 and v.shape == (n_pages, heads, d, PAGE_TOKENS) and v.is_contiguous() and v.device == k.device,
             "v: contiguous e4m3 [n_pages][heads][d][64] on the device of k is wanted")
        need(scale.dtype is torch.float32 and scale.shape == (n_pages, heads, 2) and scale.is_contiguous() and scale.device == k.device,
             "scale: contiguous float32 [n_pages][heads][2] on the device of k is wanted")
        need(table.dtype is torch.int32 and table.dim() == 2 and table.shape[1] > 0 and (table.stride(1) == 1 or table.shape[1] == 1) and
             table.device == k.device, "table: int32 [n_seqs][max_pages] on the device of k is wanted")
        need(length.dtype is torch.int32 and length.shape == table.shape[:1] and length.is_contiguous() and length.device == k.device,
             "length: int32 [n_seqs] on the device of k is wanted")
        ld = table.stride(0) if table.shape[0] > 1 else table.shape[1]
        need(not (n_pages >> 31 or heads >> 31 or table.shape[0] >> 31 or table.shape[1] >> 31 or ld >> 31), "sizes below 2^31 are wanted")
        self.k, self.v, self.scale, self.table, self.length = k, v, scale, table, length
        self.device, self.heads, self.d, self.n_seqs, self.capacity = k.get_device(), heads, d, table.shape[0], table.shape[1] * PAGE_TOKENS
        self.desc = QuantCacheDesc(k.data_ptr(), v.data_ptr(), scale.data_ptr(), table.data_ptr(), length.data_ptr(), n_pages, heads, d,
                                   table.shape[0], table.shape[1], ld)
        self.ref = C.byref(self.desc)
        self.sizes = {}                                        # workspaces' sizes by what they depend on: asking takes 2 us

    def _work(self, call: str, start, n: int, heads: int, window: int, sinks: int, like: torch.Tensor) -> Optional[torch.Tensor]:
        key = (call, start is None, n, heads, window, sinks)
        size = self.sizes.get(key)
        if size is None:
            ask = getattr(load_library(), call + "_workspace_bytes")
            size = self.sizes[key] = ask(self.ref, start, n, heads, window, sinks)
            if len(self.sizes) > 256:                          # prompts of ever other lengths
                self.sizes.clear()
        return like.new_empty(size, dtype=torch.uint8) if size else None

    def _rows(self, x: torch.Tensor, heads: int, name: str) -> int:
        """Row stride of [n][heads][d] on this cache's device."""
        if x.dim() != 3 or x.get_device() != self.device:
            raise ValueError(f"{name}: [rows][heads][d] of the cache's d on its device is wanted")
        n, h, d = x.shape                                      # once: a look at a tensor's attribute takes 0.1 us
        ld, apart, one = x.stride()
        if d != self.d or not heads or (heads > 0 and h != heads):
            raise ValueError(f"{name}: [rows][heads][d] of the cache's d on its device is wanted")
        if one != 1 or (apart != d and h != 1):
            raise ValueError(f"{name}: the heads of a row have to be neighbours")
        if (n | h) >> 31:                                      # ctypes would keep the low 32 bits
            raise ValueError(f"{name}: rows and heads below 2^31 are wanted")
        return ld if n > 1 else h * d

    def _starts(self, rows: Optional[torch.Tensor]):
        if rows is None:
            return None
        if not (rows.dtype is torch.int32 and rows.shape == (self.n_seqs + 1,) and rows.is_contiguous() and rows.get_device() == self.device):
            raise ValueError("rows: int32 [n_seqs + 1] on the cache's device is wanted")
        return rows.data_ptr()

    def _weights(self, w: torch.Tensor, least: int, name: str) -> int:
        if not (w.dtype is torch.float32 and w.dim() == 3 and w.shape[:2] == (self.n_seqs, self.heads) and w.shape[2] >= least and
                w.is_contiguous() and w.get_device() == self.device):
            raise ValueError(f"{name}: contiguous float32 [n_seqs][heads][{least} or more] on the cache's device is wanted")
        return w.shape[2]


def _int32(value: int, name: str) -> int:
    if not 0 <= value < 1 << 31:                               # ctypes would keep the low 32 bits
        raise ValueError(f"{name}: a number from 0 on, below 2^31, is wanted")
    return value


def append_fp8(cache: Fp8Cache, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None, rows: Optional[torch.Tensor] = None,
               theta: float = 0.0, position: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
    """Stores k and v [n][heads][d] (float32 or bfloat16, any row stride) as the last entries of their sequences, which cache.length
    counts already.

    rows int32 [n_seqs + 1]: where every sequence's rows begin (None: as many for each).  theta > 0: k and q are rotated by their
    position, position int32 [n_seqs] + j or (None) the entry's number.  Returns q [n][query heads][d], rotated, in bfloat16."""
    ldk, ldv = cache._rows(k, cache.heads, "k"), cache._rows(v, cache.heads, "v")
    n = k.shape[0]
    if k.dtype not in _TYPES or v.dtype is not k.dtype or v.shape[0] != n:
        raise ValueError("k, v: as many rows of float32 or bfloat16, of one type, are wanted")
    out, ldq, heads = None, 0, 0
    if q is not None:
        ldq, heads = cache._rows(q, -1, "q"), q.shape[1]
        if q.dtype is not k.dtype or q.shape[0] != n:
            raise ValueError("q: as many rows as k, of its type, are wanted")
        out = q.new_empty(n, heads, cache.d, dtype=torch.bfloat16)
    if position is not None and not (position.dtype is torch.int32 and position.shape == (cache.n_seqs,) and position.is_contiguous() and
                                     position.get_device() == cache.device):
        raise ValueError("position: int32 [n_seqs] on the cache's device is wanted")
    call_on(cache.device, load_library().spec_append_quant, cache.ref, k.data_ptr(), ldk, v.data_ptr(), ldv, _TYPES[k.dtype],
            cache._starts(rows), n, q.data_ptr() if q is not None else None, ldq, heads, theta,
            position.data_ptr() if position is not None else None, out.data_ptr() if out is not None else None)
    return out


def attend_fp8(cache: Fp8Cache, q: torch.Tensor, rows: Optional[torch.Tensor] = None, scale: Optional[float] = None, window: int = 0,
               sinks: int = 0, want_lse: bool = False, out: Optional[torch.Tensor] = None,
               lse: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(out, lse): attention of the last rows of every sequence, q bfloat16 [n][query heads][d] at any row stride that is a multiple
    of 8, over the cache.

    Row j of a sequence's M sees its entries up to len - M + j; with a window the last `window` of those and the first `sinks`
    entries.  scale: None is d ** -0.5.  out bfloat16 [n][query heads][d], lse float32 [n][query heads], made where they are not
    given (lse only if wanted)."""
    ldq = cache._rows(q, -1, "q")
    n, heads, d = q.shape
    if q.dtype is not torch.bfloat16:
        raise ValueError("q: bfloat16 is wanted")
    start = cache._starts(rows)
    _int32(window, "window"), _int32(sinks, "sinks")
    if out is None:
        out = q.new_empty(n, heads, d)
    elif not (out.dtype is torch.bfloat16 and out.shape == q.shape and out.is_contiguous() and out.get_device() == cache.device):
        raise ValueError("out: contiguous bfloat16 of the shape of q on its device is wanted")
    if lse is not None:
        if not (lse.dtype is torch.float32 and lse.shape == (n, heads) and lse.is_contiguous() and lse.get_device() == cache.device):
            raise ValueError("lse: contiguous float32 [n][query heads] on the device of q is wanted")
    elif want_lse:
        lse = q.new_empty(n, heads, dtype=torch.float32)
    lib = load_library()
    work = cache._work("spec_attend_quant", start, n, heads, window, sinks, q)
    call_on(cache.device, lib.spec_attend_quant, cache.ref, q.data_ptr(), ldq, start, n, heads, d ** -0.5 if scale is None else scale,
            window, sinks, out.data_ptr(), lse.data_ptr() if lse is not None else None, work.data_ptr() if work is not None else None)
    return out, lse


def weigh_fp8(cache: Fp8Cache, q: torch.Tensor, lse: torch.Tensor, weight: torch.Tensor, rows: Optional[torch.Tensor] = None,
              scale: Optional[float] = None, window: int = 0, sinks: int = 0) -> torch.Tensor:
    """Adds to weight (float32 [n_seqs][heads][64 * max_pages or more], returned) what every entry got of the attention of attend_fp8's
    rows: the sum of exp(scale * q k - lse) over rows and the query heads of a KV head.  The rows' own entries start from 0."""
    ldq = cache._rows(q, -1, "q")
    n, heads, d = q.shape
    if q.dtype is not torch.bfloat16:
        raise ValueError("q: bfloat16 is wanted")
    if not (lse.dtype is torch.float32 and lse.shape == (n, heads) and lse.is_contiguous() and lse.get_device() == cache.device):
        raise ValueError("lse: contiguous float32 [n][query heads] on the device of q is wanted")
    ldw, start = cache._weights(weight, cache.capacity, "weight"), cache._starts(rows)
    _int32(window, "window"), _int32(sinks, "sinks")
    lib = load_library()
    work = cache._work("spec_weigh_quant", start, n, heads, window, sinks, q)
    call_on(cache.device, lib.spec_weigh_quant, cache.ref, q.data_ptr(), ldq, lse.data_ptr(), start, n, heads,
            d ** -0.5 if scale is None else scale, window, sinks, weight.data_ptr(), ldw, work.data_ptr() if work is not None else None)
    return weight


def evict_fp8(cache: Fp8Cache, weight: torch.Tensor, to: Fp8Cache, budget: int, sinks: int = 0, recent: int = 0,
              to_weight: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Moves `budget` entries of every sequence and head of `cache` to the pages of `to`: the first `sinks`, the last `recent`, and
    between them those of the largest weight.

    to: the same heads and sequences, pages that `cache` does not use (the pools may be the same); its length is set.  to_weight
    float32 [n_seqs][heads][budget or more] gets the weights of what is kept (None: made, and not returned).  Returns the numbers of the kept
    entries, int32 [n_seqs][heads][budget], -1 behind the last."""
    ldw = cache._weights(weight, cache.capacity, "weight")
    _int32(budget, "budget"), _int32(sinks, "sinks"), _int32(recent, "recent")
    if to.device != cache.device or (to.heads, to.d, to.n_seqs) != (cache.heads, cache.d, cache.n_seqs):
        raise ValueError("to: a cache of the same heads and sequences on the same device is wanted")
    if budget > to.capacity:
        raise ValueError("budget: more than the new table holds")
    kept = weight.new_empty(cache.n_seqs, cache.heads, budget, dtype=torch.int32)
    if to_weight is None:
        to_weight = weight.new_empty(cache.n_seqs, cache.heads, budget)
    ldt = to._weights(to_weight, budget, "to_weight")
    call_on(cache.device, load_library().spec_evict_quant, cache.ref, weight.data_ptr(), ldw, to.ref, budget, sinks, recent,
            kept.data_ptr(), to_weight.data_ptr(), ldt)
    return kept
