"""Workspaces of the calls on a paged 8-bit cache stay small, and a softmax scale is finite to the base 2 too (no GPU is needed)."""
import ctypes as C

import pytest

from tests.test_abi_cache import LSE, OUT, Q, ROWS, W, WORK, _attend, _cache, amd  # noqa: F401


def _sizes(amd, n, heads, window=0, sinks=0, rows=ROWS, **c):
    lib, cache = amd.load_library(), _cache(amd, **c)
    return [f(C.byref(cache), rows, n, heads, window, sinks) for f in (lib.spec_attend_quant_workspace_bytes, lib.spec_weigh_quant_workspace_bytes)]


@pytest.mark.parametrize("by", [2.4e38, 3.4e38])
def test_scales_that_overflow_to_the_base_2_are_refused(amd, by):  # noqa: F811
    assert _attend(amd, by=by) == amd.SPEC_E_INVAL
    cache = _cache(amd)
    assert amd.load_library().spec_weigh_quant(C.byref(cache), Q, 1024, LSE, ROWS, 7, 8, by, 0, 0, W, 256, WORK, None) == amd.SPEC_E_INVAL


@pytest.mark.parametrize("pages", [65, 513, 4097])
@pytest.mark.parametrize("heads,kv", [(64, 8), (32, 32), (32, 4), (8, 1)])
@pytest.mark.parametrize("tokens", [129, 256, 257, 512, 1000, 2048, 10000])
def test_attention_of_single_tokens_needs_little(amd, tokens, heads, kv, pages):  # noqa: F811
    """Parts are for as many tiles of 256 rows as leave compute units free: two for each of 256 of them, with 130 floats a row of 128."""
    size = _sizes(amd, tokens, heads, n_seqs=tokens, n_kv_heads=kv, n_pages=100, max_pages=pages, table_ld=pages)[0]
    assert size <= 2 * 256 * 256 * 130 * 4


@pytest.mark.parametrize("window,sinks", [(1000, 0), (64, 4), (1, 0)])
@pytest.mark.parametrize("n_seqs,n,kv", [(1, 2047, 8), (1, 16384, 1), (3, 6000, 2), (200, 5000, 2)])
def test_weights_under_a_window_do_not_grow_with_the_table(amd, n_seqs, n, kv, window, sinks):  # noqa: F811
    for rows in (ROWS, None) if n % n_seqs == 0 else (ROWS,):
        small, large = (_sizes(amd, n, 8 * kv, window, sinks, rows, n_seqs=n_seqs, n_kv_heads=kv, n_pages=100, max_pages=pages, table_ld=pages)[1]
                        for pages in (2000, 1 << 17))
        assert large == small <= 256 << 20


@pytest.mark.parametrize("pages", [9, 65, 513])
@pytest.mark.parametrize("heads,kv", [(64, 8), (8, 1), (24, 1)])
@pytest.mark.parametrize("tokens", [300, 512, 2048, 10000])
def test_attention_of_single_tokens_is_planned_alike_with_their_rows_and_without(amd, tokens, heads, kv, pages):  # noqa: F811
    """A row of every sequence leaves none for a long one: no launch, and no workspace, for those."""
    with_rows, without = (_sizes(amd, tokens, heads, rows=rows, n_seqs=tokens, n_kv_heads=kv, n_pages=100, max_pages=pages, table_ld=pages) for rows in (ROWS, None))
    assert with_rows[0] == without[0] == 0
