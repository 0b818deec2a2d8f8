"""Prompts beside many sequences of one row or none: parts of the prompts' tiles, as many as are planned for and beyond (run with -m gpu)."""
import numpy as np
import pytest
import torch

from oracle import cache8
from tests.cache8 import EPS, bf16, check_attention, make, normal, starts_of, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


def _rows(kind):
    """(rows, lengths) of every sequence."""
    rng = np.random.default_rng(3)
    if kind == "nobody long":
        rows = [1] * 600
    elif kind == "one long among single tokens":
        rows = [1] * 200 + [300] + [1] * 57
    elif kind == "one long among none":                      # more tiles than a row of every sequence leaves
        rows = [0] * 150 + [900] + [0] * 150
    elif kind == "as many rows as sequences":
        rows = [0] * 400 + [500] + [0] * 99
    elif kind == "several among none":
        rows = [0] * 70 + [257] + [0] * 80 + [333, 41, 700] + [0] * 200 + [5]
    elif kind == "long ones only":
        rows = [400, 500, 300]
    lengths = [r + int(x) for r, x in zip(rows, rng.integers(0, 100, len(rows)))]
    longest = int(np.argmax(rows))
    lengths[longest] += 1500
    return rows, lengths


@pytest.mark.parametrize("window,sinks", [(0, 0), (600, 3)])
@pytest.mark.parametrize("heads,kv,d", [(8, 2, 64), (16, 2, 128), (20, 1, 64)])
@pytest.mark.parametrize("kind", ["nobody long", "one long among single tokens", "one long among none", "as many rows as sequences", "several among none", "long ones only"])
def test_attention(kind, heads, kv, d, window, sinks):
    import paper_2408_11850_amd as amd
    amd.load_library()
    rng = np.random.default_rng(heads)
    rows, lengths = _rows(kind)
    c = make(rng, lengths, kv, d, junk=True)
    start, n = starts_of(rows), sum(rows)
    q = bf16(normal(rng, n + 2, heads, d))
    qg, sg, g = torch.from_numpy(q).cuda().to(torch.bfloat16), torch.from_numpy(start).cuda(), to_gpu(amd, c)
    held = torch.full((n + 2, heads, d), 7.0, dtype=torch.bfloat16, device="cuda")
    out, lse = amd.attend_fp8(g, qg, sg, window=window, sinks=sinks, want_lse=True, out=held)
    assert (out[n:] == 7).all()
    want, want_lse, mass, size = cache8.attend(c, start, q[:n], d ** -0.5, window, sinks)
    check_attention(out[:n].float().cpu().numpy(), lse[:n].cpu().numpy(), want, want_lse, mass, size, d, max(lengths))
    again, lse2 = amd.attend_fp8(g, qg, sg, window=window, sinks=sinks, want_lse=True)
    assert torch.equal(again[:n], out[:n]) and torch.equal(lse2[:n], lse[:n])


@pytest.mark.parametrize("window,sinks", [(0, 0), (600, 3)])
@pytest.mark.parametrize("heads,kv,d", [(8, 2, 64), (16, 2, 128), (20, 1, 64)])
@pytest.mark.parametrize("kind", ["nobody long", "one long among single tokens", "one long among none", "as many rows as sequences", "several among none", "long ones only"])
def test_weights(kind, heads, kv, d, window, sinks):
    """Terms off by (d + 5) steps of their exponents' magnitudes; sums of positive terms, as deep as a sequence's rows at most."""
    import paper_2408_11850_amd as amd
    amd.load_library()
    rng = np.random.default_rng(heads)
    rows, lengths = _rows(kind)
    c = make(rng, lengths, kv, d, junk=True)
    start, n = starts_of(rows), sum(rows)
    q, lse = bf16(normal(rng, n, heads, d)), (4 + normal(rng, n, heads)).astype(np.float32)
    weight = rng.random((len(rows), kv, c.table.shape[1] * 64)).astype(np.float32)
    up = lambda x: torch.from_numpy(x).cuda()
    got = amd.weigh_fp8(to_gpu(amd, c), up(q).to(torch.bfloat16), up(lse), up(weight), up(start), window=window, sinks=sinks).cpu().numpy()
    want, slack = cache8.weigh(c, start, q, lse, weight, d ** -0.5, window, sinks)
    bound = slack * (d + 5) * EPS * 1.1 + want * (max(rows) * heads // kv + 48) * EPS
    assert (np.abs(got - want) <= bound + 1e-37).all()


def test_a_captured_call_whose_long_rows_outgrow_its_parts():
    """Rows of a graph move to sequences that leave more tiles than have parts, and back."""
    import paper_2408_11850_amd as amd
    amd.load_library()
    rng, heads, kv, d, seqs, n = np.random.default_rng(4), 8, 2, 128, 200, 900
    c = make(rng, [1000] * 2, kv, d)
    c.table, c.length = np.concatenate([c.table] * (seqs // 2)), np.full(seqs, 1000, np.int32)
    g = to_gpu(amd, c)
    q = torch.from_numpy(normal(rng, n, heads, d)).cuda().to(torch.bfloat16)
    start = torch.zeros(seqs + 1, dtype=torch.int32, device="cuda")
    spread = [1] * (seqs - 1) + [n - seqs + 1]
    batches = [spread, [0] * (seqs - 1) + [n], [0] * 100 + [450] + [0] * 50 + [450] + [0] * (seqs - 152), spread[::-1], [4] * 100 + [5] * 100]
    start.copy_(torch.from_numpy(starts_of(spread)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        amd.attend_fp8(g, q, start, want_lse=True)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = amd.attend_fp8(g, q, start, want_lse=True)
    for rows in batches + batches[:1]:
        at = starts_of(rows)
        start.copy_(torch.from_numpy(at))
        graph.replay()
        torch.cuda.synchronize()
        eager = amd.attend_fp8(g, q, start, want_lse=True)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
        want, want_lse, mass, size = cache8.attend(c, at, q.float().cpu().numpy(), d ** -0.5)
        check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), want, want_lse, mass, size, d, 1000)
