"""Attention over the paged 8-bit cache against 64 bits (run with -m gpu)."""
import numpy as np
import pytest
import torch

from oracle import cache8
from tests.cache8 import MIXED, bf16, check_attention, make, normal, starts_of, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _run(lengths, rows, heads, kv, d, window=0, sinks=0, ragged=True, seed=1, scale=None, junk=True, pad_rows=0, q_pad=0, change=None,
         lse=True):
    amd, rng = _amd(), np.random.default_rng(seed)
    c = make(rng, lengths, kv, d, junk=junk)
    if change:
        change(c)
    start = starts_of(rows)
    n = int(start[-1])
    q = bf16(normal(rng, n + pad_rows, heads, d))
    wide = torch.zeros(n + pad_rows, heads * d + q_pad, dtype=torch.bfloat16, device="cuda")
    wide[:, :heads * d] = torch.from_numpy(q).cuda().view(n + pad_rows, -1).to(torch.bfloat16)
    qg = wide[:, :heads * d].view(n + pad_rows, heads, d) if not q_pad else wide.as_strided((n + pad_rows, heads, d), (heads * d + q_pad, d, 1))
    g = to_gpu(amd, c, table_pad=2)
    out = torch.full((n + pad_rows, heads, d), 7.0, dtype=torch.bfloat16, device="cuda")
    got, got_lse = amd.attend_fp8(g, qg, torch.from_numpy(start).cuda() if ragged else None, scale, window, sinks, lse, out)
    torch.cuda.synchronize()
    assert got is out and (got[n:] == 7).all()
    by = d ** -0.5 if scale is None else scale
    want, want_lse, mass, size = cache8.attend(c, start, q[:n], by, window, sinks)
    check_attention(got[:n].float().cpu().numpy(), got_lse[:n].cpu().numpy() if lse else None, want, want_lse, mass, size, d, max(max(lengths), 1))
    return got, c


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv", [(4, 4), (8, 1), (6, 2), (1, 1), (40, 2)])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 200, 700])
def test_single_tokens(n, heads, kv, d):
    _run([n, max(1, n - 3)], [1, 1], heads, kv, d, ragged=False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,kv", [(4, 4), (8, 1), (6, 2)])
@pytest.mark.parametrize("m,n", [(2, 2), (5, 64), (8, 129), (17, 17), (33, 100), (64, 64), (65, 200), (100, 333), (260, 300)])
def test_rows_see_up_to_themselves(m, n, heads, kv, d):
    _run([n], [m], heads, kv, d, ragged=False)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 4), (7, 0), (64, 1), (65, 64), (100, 3), (130, 70), (1000, 5), (5, 1000)])
@pytest.mark.parametrize("m", [1, 9, 70, 300])
def test_windows_and_sinks(m, window, sinks):
    _run([500, max(m, 131), max(m, 64)], [m, m, m], 8, 2, 128, window, sinks)
    _run([500], [m], 2, 2, 64, window, sinks)


@pytest.mark.parametrize("heads,kv,d", [(8, 8, 64), (8, 1, 128)])
@pytest.mark.parametrize("rows", [[1, 5, 0, 2, 17], [0, 0, 40, 1, 0], [3, 64, 65, 1, 200], [1, 1, 1, 1, 500]])
def test_ragged_batches(rows, heads, kv, d):
    lengths = [max(r, n) for r, n in zip(rows, [300, 64, 128, 77, 640])]
    _run(lengths, rows, heads, kv, d, pad_rows=5, q_pad=8)
    _run(lengths, rows, heads, kv, d, window=50, sinks=2, pad_rows=1)


def test_many_sequences():
    """More than a wave's lanes of them, most with no rows."""
    rng = np.random.default_rng(4)
    rows = [int(x) for x in rng.integers(0, 3, 150)]
    _run([max(r, int(x)) for r, x in zip(rows, rng.integers(0, 200, 150))], rows, 4, 2, 64)


def test_rows_in_front_of_the_first_entry_see_nothing():
    got, _ = _run([3, 0, 5], [6, 2, 5], 4, 2, 128, pad_rows=2)
    assert (got[:3] == 0).all() and (got[6:8] == 0).all()
    _run([3, 0], [70, 90], 8, 2, 64)
    _run([3, 0, 1000], [70, 90, 70], 8, 2, 64, window=10, sinks=1)


def test_pages_that_no_row_sees_may_be_any():
    def drop(c):
        c.table[0, 1:6] = [-1, 10 ** 6, -2 ** 31, 2 ** 31 - 1, -1]
    for m in (1, 40):
        _run([500], [m], 8, 2, 128, window=50, sinks=10, change=drop)


@pytest.mark.parametrize("m", [1, 6, 150])
def test_a_page_that_is_none_makes_its_rows_nan(m):
    def drop(c):
        c.table[0, 2] = 10 ** 6
        c.table[1, 4] = -1
    got, c = _run([400, 300, 90], [m, m, min(m, 90)], 4, 2, 128, change=drop)
    assert got[:m].isnan().all() and got[2 * m - 1].isnan().all()


@pytest.mark.parametrize("heads,kv,m", [(2, 2, 7), (8, 2, 3), (8, 2, 20), (8, 1, 40), (4, 2, 150), (8, 1, 300)])
def test_rows_beside_those_that_see_such_a_page(heads, kv, m):
    """Rows of one tile of which some see the page: the others keep their results."""
    def drop(c):
        for s in range(len(c.length)):
            c.table[s, int(c.length[s] - 1) // 64] = -1
    got, _ = _run([64 * 5 + 1 + m // 2, 64 * 9 + 2], [m, min(m, 70)], heads, kv, 128, change=drop)
    assert not got[:m - m // 2 - 1].isnan().any() and got[m - 1].isnan().all()


@pytest.mark.parametrize("m", [1, 100])
def test_lengths_beyond_the_table(m):
    def grow(c):
        c.length[:] = [64 * c.table.shape[1] + 1, 2 ** 31 - 1, 200]
    got, _ = _run([200, 200, 200], [m, m, m], 4, 2, 64, change=grow)
    assert got[:2 * m].isnan().all() and not got[2 * m:].isnan().any()


@pytest.mark.parametrize("m", [1, 30, 200])
def test_a_nan_key_reaches_only_rows_that_see_it(m):
    def poison(c):
        c.k[c.table[0, 3], 1, 17] = 127                       # entry 209
        c.v[c.table[0, 3], 1, :, 17] = 0
    got, _ = _run([300], [m], 4, 2, 128, change=poison)
    first = 300 - m
    bad = got.isnan().all(2).cpu().numpy()
    assert (bad[:, 2:].all(1) == (first + np.arange(m) >= 209)).all() and not bad[:, :2].any()


def test_scores_far_apart_and_tiny():
    _run([300], [5], 4, 2, 128, scale=3.0)
    _run([300], [5], 4, 2, 64, scale=2.0 ** -40)
    def huge(c):
        c.scale[:, :, 0] = 2.0 ** 40
    _run([300], [150], 4, 2, 64, change=huge)


def test_no_sums_wanted():
    _run([300], [3], 4, 2, 128, lse=False)


def test_split_and_unsplit_rows_agree():
    """A sequence alone is cut over its pages, among many it is not: the same values up to the order of the sums."""
    amd, rng = _amd(), np.random.default_rng(9)
    c = make(rng, [2000], 8, 128)
    q = torch.from_numpy(normal(rng, 1, 64, 128)).cuda().to(torch.bfloat16)
    alone, lse = amd.attend_fp8(to_gpu(amd, c), q, want_lse=True)
    many = cache8.Cache(c.k, c.v, c.scale, np.repeat(c.table, 200, 0), np.repeat(c.length, 200))
    among, lse2 = amd.attend_fp8(to_gpu(amd, many), q.expand(200, 64, 128), want_lse=True)
    assert torch.equal(among, among[:1].expand(200, 64, 128)) and torch.equal(lse2, lse2[:1].expand(200, 64))
    assert ((alone[0].float() - among[0].float()).abs() <= 2.0 ** -7 * alone[0].float().abs() + 2.0 ** -9).all()
    assert ((lse - lse2[:1]).abs() <= 1e-5).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 5)])
@pytest.mark.parametrize("rows,lengths,heads,kv", MIXED)
def test_prompts_and_single_tokens_in_one_batch(rows, lengths, heads, kv, window, sinks, d):
    _run(lengths, rows, heads, kv, d, window, sinks, pad_rows=3)


def test_pages_and_lengths_that_are_none_in_a_mixed_batch():
    """Pages that are none and lengths beyond the table, in front of and behind sequences of the other kind."""
    def change(c):
        c.table[0, 2] = 10 ** 6
        c.table[3, 1] = -1
        c.length[2] = 64 * c.table.shape[1] + 1
        c.length[5] = 64 * c.table.shape[1] + 7
    _run([700, 300, 600, 200, 5, 90, 400], [600, 1, 300, 3, 9, 1, 41], 8, 2, 128, change=change, pad_rows=1)
