"""Attention weights of the entries of the paged 8-bit cache against 64 bits (run with -m gpu)."""
import numpy as np
import pytest
import torch

from oracle import cache8
from tests.cache8 import EPS, MIXED, bf16, make, normal, starts_of, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _run(lengths, rows, heads, kv, d, window=0, sinks=0, ragged=True, seed=1, change=None, more=0):
    """A term is exp of a score off by (d + 5) steps of its magnitudes and of the logarithm, plus the hardware exponential's two steps; the
    terms are positive and added in fp32, at most rows * group + 32 additions deep."""
    amd, rng = _amd(), np.random.default_rng(seed)
    c = make(rng, lengths, kv, d, junk=True)
    if change:
        change(c)
    start = starts_of(rows)
    n = int(start[-1])
    q = bf16(normal(rng, max(n, 1), heads, d))
    lse = (4 + normal(rng, max(n, 1), heads)).astype(np.float32)
    weight = rng.random((len(lengths), kv, c.table.shape[1] * 64 + more)).astype(np.float32)
    want, slack = cache8.weigh(c, start, q, lse, weight, d ** -0.5, window, sinks)
    w = torch.from_numpy(weight).cuda()
    got = amd.weigh_fp8(to_gpu(amd, c, table_pad=1), torch.from_numpy(q).cuda().to(torch.bfloat16), torch.from_numpy(lse).cuda(), w,
                        torch.from_numpy(start).cuda() if ragged else None, window=window, sinks=sinks)
    assert got is w
    got = got.cpu().numpy()
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(want), np.isnan(got))
    deep = max(rows) * heads // kv + 40
    bound = slack * (d + 5) * EPS * 1.1 + want * (deep + 8) * EPS
    assert (np.abs(got - want) <= bound + 1e-37)[fine].all()
    for s, length in enumerate(c.length):
        if length <= c.table.shape[1] * 64:
            assert np.array_equal(got[s, :, max(int(length), 0):], weight[s, :, max(int(length), 0):])
        else:
            assert np.array_equal(got[s], weight[s])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv", [(4, 4), (8, 1), (6, 2), (40, 2)])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 64), (1, 65), (1, 500), (3, 3), (9, 200), (17, 130), (70, 70), (300, 400)])
def test_sums(m, n, heads, kv, d):
    _run([n, max(m, n - 2)], [m, m], heads, kv, d, ragged=False, more=3)


@pytest.mark.parametrize("window,sinks", [(1, 0), (7, 4), (64, 1), (100, 70), (1000, 5)])
@pytest.mark.parametrize("m", [1, 9, 70, 300])
def test_windows_and_sinks(m, window, sinks):
    _run([500, max(m, 131)], [m, m], 8, 2, 128, window, sinks)
    _run([500], [m], 2, 2, 64, window, sinks)


@pytest.mark.parametrize("rows", [[1, 5, 0, 2, 17], [0, 0, 40, 1, 0], [3, 64, 65, 1, 200], [1, 1, 1, 1, 500]])
def test_ragged_batches(rows):
    lengths = [max(r, n) for r, n in zip(rows, [300, 64, 128, 77, 640])]
    _run(lengths, rows, 8, 2, 128)
    _run(lengths, rows, 4, 4, 64, window=50, sinks=2)


def test_rows_in_front_of_the_first_entry_and_empty_caches():
    _run([3, 0, 5], [6, 2, 5], 4, 2, 128)
    _run([3, 0, 90], [100, 90, 90], 4, 2, 64)


@pytest.mark.parametrize("m", [1, 150])
def test_pages_and_lengths_that_are_none(m):
    def change(c):
        c.table[0, 2] = 10 ** 6
        c.length[1] = 64 * c.table.shape[1] + 1
    _run([400, 300, 200], [m, m, m], 4, 2, 128, change=change)
    def hidden(c):
        c.table[0, 1:5] = -1
    _run([400], [m], 4, 2, 64, window=10, sinks=3, change=hidden) if m == 1 else None


@pytest.mark.parametrize("m", [1, 5, 40, 200])
def test_entries_of_a_page_that_is_none_that_no_row_sees(m):
    """The window begins, and the first entries end, inside such pages: what is hidden there keeps its weight."""
    def change(c):
        first = 600 - m - 30 + 1
        c.table[0, first // 64] = 10 ** 6
        c.table[0, 0] = -5
    _run([600], [m], 8, 2, 128, window=30, sinks=5, change=change)
    _run([600], [m], 4, 4, 64, window=30, sinks=5, change=change)


@pytest.mark.parametrize("window,sinks", [(0, 0), (100, 4)])
@pytest.mark.parametrize("m", [1, 8, 200])
def test_weights_of_an_attention_add_up(m, window, sinks):
    """With the attention's own logarithms every row and head hands out 1: the entries of a KV head get rows * group in all."""
    amd, rng = _amd(), np.random.default_rng(3)
    c = make(rng, [900, 300], 2, 128)
    g = to_gpu(amd, c)
    q = torch.from_numpy(normal(rng, 2 * m, 16, 128)).cuda().to(torch.bfloat16)
    _, lse = amd.attend_fp8(g, q, window=window, sinks=sinks, want_lse=True)
    w = amd.weigh_fp8(g, q, lse, torch.zeros(2, 2, g.capacity, device="cuda"), window=window, sinks=sinks)
    assert ((w.double().sum(2) - 8 * m).abs() <= 8 * m * 1e-4).all()
    again = amd.weigh_fp8(g, q, lse, w.clone(), window=window, sinks=sinks)
    for s, n in enumerate((900, 300)):
        assert torch.allclose(again[s, :, :n - m], 2 * w[s, :, :n - m], rtol=1e-6) and torch.equal(again[s, :, n - m:], w[s, :, n - m:])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("m,n", [(9, 4), (100, 70), (300, 130)])
def test_rows_without_entries_with_their_own_logarithms(m, n, d):
    """Rows in front of entry 0 have -inf as the logarithm of their sum and add nothing; the others hand out 1 each."""
    amd, rng = _amd(), np.random.default_rng(5)
    g = to_gpu(amd, make(rng, [n, 2 * m], 2, d, junk=True))
    q = torch.from_numpy(normal(rng, 2 * m, 8, d)).cuda().to(torch.bfloat16)
    _, lse = amd.attend_fp8(g, q, want_lse=True)
    assert torch.isneginf(lse[:m - n]).all() and torch.isfinite(lse[m - n:]).all()
    w = amd.weigh_fp8(g, q, lse, torch.zeros(2, 2, g.capacity, device="cuda"))
    want = torch.tensor([n * 4.0, m * 4.0], device="cuda", dtype=torch.float64)[:, None]
    assert ((w.double().sum(2) - want).abs() <= want * 1e-4).all()


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("m", [4, 16, 200])
def test_a_row_whose_logarithm_is_none_touches_only_what_it_sees(m, window, value):
    """Row j with NaN: NaN; with +inf: nothing; with -inf: inf, to the entries that it sees, and all others as without it."""
    amd, rng = _amd(), np.random.default_rng(6)
    n, j = 300, m // 2
    g = to_gpu(amd, make(rng, [n], 2, 128, junk=True))
    q = torch.from_numpy(normal(rng, m, 8, 128)).cuda().to(torch.bfloat16)
    _, lse = amd.attend_fp8(g, q, window=window, want_lse=True)
    odd, none = lse.clone(), lse.clone()
    odd[j, 4:] = value
    none[j, 4:] = float("inf")
    got = amd.weigh_fp8(g, q, odd, torch.zeros(1, 2, g.capacity, device="cuda"), window=window)
    without = amd.weigh_fp8(g, q, none, torch.zeros(1, 2, g.capacity, device="cuda"), window=window)
    assert torch.isfinite(without).all()
    last = n - m + j
    seen = torch.zeros(g.capacity, dtype=torch.bool, device="cuda")
    seen[max(0, last - window + 1) if window else 0:last + 1] = True
    assert torch.equal(got[0, 0], without[0, 0]) and torch.equal(got[0, 1][~seen], without[0, 1][~seen])
    if value == float("inf"):
        assert torch.equal(got, without)
    else:
        assert (torch.isnan(got[0, 1][seen]) if value != value else torch.isposinf(got[0, 1][seen])).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 5)])
@pytest.mark.parametrize("rows,lengths,heads,kv", MIXED)
def test_prompts_and_single_tokens_in_one_batch(rows, lengths, heads, kv, window, sinks, d):
    _run(lengths, rows, heads, kv, d, window, sinks)


@pytest.mark.parametrize("window", [0, 1000])
def test_long_and_short_sequences_together_and_alone(window):
    """So many rows that a slice has more than its least number of tiles.  Terms are the same in both; their sums, of up to 16 * 5000 positive
    terms, are off by as many steps at most."""
    amd, rng = _amd(), np.random.default_rng(8)
    rows, lengths = [5000, 3, 70], [5100, 900, 130]
    c = make(rng, lengths, 1, 64)
    g, start = to_gpu(amd, c), starts_of(rows)
    q = torch.from_numpy(normal(rng, int(start[-1]), 16, 64)).cuda().to(torch.bfloat16)
    at = torch.from_numpy(start).cuda()
    _, lse = amd.attend_fp8(g, q, at, window=window, sinks=4, want_lse=True)
    got = amd.weigh_fp8(g, q, lse, torch.zeros(3, 1, g.capacity, device="cuda"), at, window=window, sinks=4)
    for s in range(3):
        one = amd.Fp8Cache(g.k, g.v, g.scale, g.table[s:s + 1], g.length[s:s + 1].clone())
        mine = slice(int(start[s]), int(start[s + 1]))
        want = amd.weigh_fp8(one, q[mine], lse[mine], torch.zeros(1, 1, g.capacity, device="cuda"), window=window, sinks=4)
        assert ((got[s] - want[0]).abs() <= 2 * (16 * 5000 + 80) * EPS * want[0]).all()
        assert abs(float(want.double().sum()) - 16 * rows[s]) <= 16 * rows[s] * 1e-4
