"""The calls on a paged 8-bit cache one behind the other, as a decode loop uses them, captured, beside each other, and at their
largest sizes (run with -m gpu)."""
import numpy as np
import pytest
import torch

import synth
from oracle import cache8
from tests.cache8 import bf16, check_attention, codes, make, normal, same_codes, starts_of, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _pull(g, width):
    """The oracle's cache with what the GPU's holds."""
    return cache8.Cache(codes(g.k), codes(g.v), g.scale.cpu().numpy(), g.table.cpu().numpy()[:, :width], g.length.cpu().numpy())


def test_a_decode_loop_with_eviction():
    """Prompt, windows of drafts of which some are dropped, weights, and eviction to new pages when a cache is full: every step against
    its definition on what the step before it left."""
    amd, rng = _amd(), np.random.default_rng(1)
    heads, kv, d, width, window, sinks = 8, 2, 128, 5, 200, 4
    start_lengths = [130, 60]
    c = make(rng, [0, 0], kv, d, spare=40, width=width)
    pages = rng.permutation(40)
    c.table[:] = pages[:10].reshape(2, 5)
    g = to_gpu(amd, c)
    free = list(pages[10:])
    weight = torch.zeros(2, kv, width * 64, device="cuda")
    position = np.zeros(2, np.int32)
    rows, evictions = start_lengths, 0
    for step in range(24):
        start = starts_of(rows)
        n = int(start[-1])
        k, v, q = (bf16(normal(rng, n, h, d)) for h in (kv, kv, heads))
        g.length += torch.tensor(rows, dtype=torch.int32, device="cuda")
        before = _pull(g, width)
        rs, pos = torch.from_numpy(start).cuda(), torch.from_numpy(position).cuda()
        up = lambda x: torch.from_numpy(x).cuda().to(torch.bfloat16)
        qr = amd.append_fp8(g, up(k), up(v), up(q), rs, 10000.0, pos)
        before.append(start, k, v, 10000.0, position)
        now = _pull(g, width)
        assert np.array_equal(now.scale[..., 1], before.scale[..., 1]) and same_codes(now.v, before.v)
        out, lse = amd.attend_fp8(g, qr, rs, window=window, sinks=sinks, want_lse=True)
        qn = qr.float().cpu().numpy()
        want, want_lse, mass, size = cache8.attend(now, start, qn, d ** -0.5, window, sinks)
        check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), want, want_lse, mass, size, d, 320)
        was = weight.cpu().numpy()
        amd.weigh_fp8(g, qr, lse, weight, rs, window=window, sinks=sinks)
        want, _ = cache8.weigh(now, start, qn, lse.cpu().numpy(), was, d ** -0.5, window, sinks)
        assert np.allclose(weight.cpu().numpy(), want, rtol=1e-4, atol=1e-6)
        dropped = np.array([int(x) for x in rng.integers(0, 3, 2)]) if step else np.zeros(2, int)
        dropped = np.minimum(dropped, np.array(rows) - 1)
        g.length -= torch.from_numpy(dropped.astype(np.int32)).cuda()          # drafts that were not accepted
        position += np.array(rows, np.int32) - dropped.astype(np.int32)
        if int(g.length.max()) > 210:
            full = _pull(g, width)
            fresh = [free.pop() for _ in range(2 * 3)]
            table = torch.full((2, width), -1, dtype=torch.int32)
            table[:, :3] = torch.tensor(fresh, dtype=torch.int32).view(2, 3)
            to = amd.Fp8Cache(g.k, g.v, g.scale, table.cuda(), torch.zeros(2, dtype=torch.int32, device="cuda"))
            left = torch.zeros_like(weight)
            w = weight.cpu().numpy()
            kept = amd.evict_fp8(g, weight, to, 150, sinks, 32, to_weight=left)
            o = cache8.Cache(full.k, full.v, full.scale, table.numpy(), [0, 0])
            want_kept, want_left = cache8.evict(full, w, o, 150, sinks, 32)
            assert np.array_equal(kept.cpu().numpy(), want_kept) and np.array_equal(left.cpu().numpy()[..., :150], want_left)
            after = _pull(to, width)
            assert same_codes(after.k, o.k) and same_codes(after.v, o.v) and np.array_equal(after.scale, o.scale) and np.array_equal(after.length, o.length)
            free = list(g.table.cpu().numpy()[g.table.cpu().numpy() >= 0]) + free
            g, weight, evictions = to, left, evictions + 1
            # two tables more for what comes
            table[:, 3:] = torch.tensor([free.pop() for _ in range(4)], dtype=torch.int32).view(2, 2)
            g = amd.Fp8Cache(g.k, g.v, g.scale, table.cuda(), g.length)
        rows = [int(x) for x in rng.integers(1, 40 if step % 3 == 0 else 9, 2)]
    assert evictions >= 2


def test_the_attention_of_an_8_bit_forward():
    """Rows in 8 bits -> QKV -> cache and attention -> rows in 8 bits -> output projection, against the same in 64 bits from the QKV on."""
    amd, rng = _amd(), np.random.default_rng(2)
    heads, kv, d, D, m = 4, 2, 64, 256, 6
    quant = lambda n, k, seed: amd.quant_weight_fp8(synth.normal_tensor((n, k), 0.06, seed, 3, torch.float32).bfloat16().cuda())
    wqkv, wo = amd.pack_weights_fp8([quant(heads * d, D, 1), quant(kv * d, D, 2), quant(kv * d, D, 3)]), amd.pack_weights_fp8([quant(D, heads * d, 4)])
    c = make(rng, [200 - m], kv, d)
    g = to_gpu(amd, c)
    h = torch.from_numpy(normal(rng, m, D)).cuda()
    qkv = amd.gemm_fp8(*amd.add_norm_fp8(h, None, torch.ones(D, dtype=torch.bfloat16, device="cuda"), 1e-5), wqkv)
    q, k, v = (qkv[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
    g.length += m
    out, _ = amd.attend_fp8(g, amd.append_fp8(g, k, v, q, theta=10000.0))
    y = amd.gemm_fp8(*amd.quant_fp8(out.flatten(1)), wo, 0, torch.float32)
    now = _pull(g, g.table.shape[1])
    at = 200 - m + np.arange(m)
    qn = bf16(cache8.rotate(q.float().cpu().numpy().astype(np.float64), at, 10000.0))
    want, _, mass, _ = cache8.attend(now, [0, m], qn, d ** -0.5)
    # q may round to its other neighbour (2^-8 of an element): scores off by 2^-8 of |q| |k|, here below 0.05, weights by as much
    assert (np.abs(out.double().cpu().numpy() - want) <= (2.0 ** -7 + 0.1) * mass).all() and y.isfinite().all() and y.shape == (m, D)
    kr = cache8.rotate(k.float().cpu().numpy().astype(np.float64), at, 10000.0)
    got = np.stack([now.entries(0, x)[0][200 - m:] for x in range(kv)], 1)
    assert (np.abs(got - kr) <= 2.0 ** -4 * np.abs(kr) + 2.0 ** -10 * now.scale.max() + 1e-5).all()


def test_captured_steps_repeat_with_other_lengths():
    """A graph of append, attention and weights, replayed while lengths and tables grow, with eager work between the replays."""
    amd, rng = _amd(), np.random.default_rng(3)
    heads, kv, d, m = 16, 2, 128, 4
    c = make(rng, [700, 40], kv, d, width=14, spare=20)
    c.table[:] = rng.permutation(28).reshape(2, 14)
    g = to_gpu(amd, c)
    k, v, q = (torch.zeros(2 * m, h, d, dtype=torch.bfloat16, device="cuda") for h in (kv, kv, heads))
    weight = torch.zeros(2, kv, g.capacity, device="cuda")

    def run(g, weight):
        qr = amd.append_fp8(g, k, v, q, theta=10000.0)
        out, lse = amd.attend_fp8(g, qr, window=500, sinks=4, want_lse=True)
        amd.weigh_fp8(g, qr, lse, weight, window=500, sinks=4)
        return out, lse

    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        run(to_gpu(amd, c), weight.clone())
    torch.cuda.current_stream().wait_stream(st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = run(g, weight)
    g2, weight2 = to_gpu(amd, c), weight.clone()
    for rep in range(4):
        for t in (k, v, q):
            t.copy_(torch.from_numpy(normal(rng, *t.shape)))
        g.length += m + rep * 3
        g2.length += m + rep * 3
        graph.replay()
        torch.cuda.synchronize()
        eager = run(g2, weight2)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1]) and torch.equal(weight, weight2)
        assert torch.equal(g.k.view(torch.uint8), g2.k.view(torch.uint8)) and torch.equal(g.scale, g2.scale)


def test_two_graphs_and_a_second_stream():
    """Calls on different caches at once, in two captured graphs with workspaces of their own, give what they give alone."""
    amd, rng = _amd(), np.random.default_rng(4)
    caches = [to_gpu(amd, make(rng, [3000], 8, 128)) for _ in range(2)]
    q = [torch.from_numpy(normal(rng, 3, 64, 128)).cuda().to(torch.bfloat16) for _ in range(2)]
    alone = [amd.attend_fp8(c, x, want_lse=True) for c, x in zip(caches, q)]
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for c, x in zip(caches, q):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(amd.attend_fp8(c, x, want_lse=True))
        graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(5):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        for s, c, x in zip(streams, caches, q):
            with torch.cuda.stream(s):
                eager = amd.attend_fp8(c, x, want_lse=True)
        torch.cuda.synchronize()
        for a, b in zip(alone, outs):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        assert torch.equal(eager[0], alone[1][0])


def test_the_same_bits_every_time():
    amd, rng = _amd(), np.random.default_rng(5)
    c = make(rng, [2500, 900], 4, 128)
    g = to_gpu(amd, c)
    for m in (1, 6, 60):
        q = torch.from_numpy(normal(rng, 2 * m, 32, 128)).cuda().to(torch.bfloat16)
        first = None
        for _ in range(4):
            out, lse = amd.attend_fp8(g, q, want_lse=True)
            w = amd.weigh_fp8(g, q, lse, torch.zeros(2, 4, g.capacity, device="cuda"))
            first = first or (out, lse, w)
            assert all(torch.equal(a, b) for a, b in zip(first, (out, lse, w)))


@pytest.mark.parametrize("m", [1, 20, 200])
def test_more_pages_than_a_wave_lists_at_once(m):
    """20000 entries by a table that repeats 40 pages; among 300 such sequences nothing is split, alone everything is."""
    amd, rng = _amd(), np.random.default_rng(6)
    c = make(rng, [40 * 64], 1, 64, width=40)
    c.table, c.length = np.tile(c.table, (1, 8))[:, :313], np.array([20000], np.int32)
    q = bf16(normal(rng, m, 1, 64))
    want, want_lse, mass, size = cache8.attend(c, [0, m], q, 0.125)
    qg = torch.from_numpy(q).cuda().to(torch.bfloat16)
    out, lse = amd.attend_fp8(to_gpu(amd, c), qg, want_lse=True)
    check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), want, want_lse, mass, size, 64, 20000)
    many = to_gpu(amd, cache8.Cache(c.k, c.v, c.scale, np.repeat(c.table, 300, 0), np.repeat(c.length, 300)))
    out, lse = amd.attend_fp8(many, qg.repeat(300, 1, 1), want_lse=True)
    check_attention(out[-m:].float().cpu().numpy(), lse[-m:].cpu().numpy(), want, want_lse, mass, size, 64, 20000)
    assert torch.equal(out.view(300, m, 64), out[:m].view(1, m, 64).expand(300, m, 64))
    w = amd.weigh_fp8(many, qg.repeat(300, 1, 1), lse, torch.zeros(300, 1, many.capacity, device="cuda"))
    got, slack = cache8.weigh(c, [0, m], q, lse[:m].cpu().numpy(), np.zeros((1, 1, many.capacity)), 0.125)
    assert torch.equal(w, w[:1].expand_as(w)) and (np.abs(w[0].cpu().numpy() - got[0]) <= slack[0] * 70 * 2.0 ** -24 + got[0] * (m + 48) * 2.0 ** -24 + 1e-37).all()


def test_pools_beyond_4_gib():
    """Pages whose codes begin behind 2^32 bytes: append, attention, weights and eviction."""
    amd, rng = _amd(), np.random.default_rng(7)
    pages, kv, d = 70000, 8, 128
    k = torch.zeros(pages, kv, 64, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    v = torch.zeros(pages, kv, d, 64, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    scale = torch.zeros(pages, kv, 2, device="cuda")
    table = np.array([[pages - 1, 3, pages - 5]], np.int32)
    length = torch.tensor([150], dtype=torch.int32, device="cuda")
    g = amd.Fp8Cache(k, v, scale, torch.from_numpy(table).cuda(), length)
    x = [bf16(normal(rng, 150, kv, d)) for _ in range(2)]
    amd.append_fp8(g, *(torch.from_numpy(t).cuda().to(torch.bfloat16) for t in x))
    small = cache8.Cache(np.zeros((3, kv, 64, d), np.uint8), np.zeros((3, kv, d, 64), np.uint8), np.zeros((3, kv, 2), np.float32), [[0, 1, 2]], [150])
    small.append([0, 150], *x)
    ids = torch.from_numpy(table[0].astype(np.int64)).cuda()
    assert np.array_equal(k.view(torch.uint8)[ids].cpu().numpy(), small.k) and np.array_equal(v.view(torch.uint8)[ids].cpu().numpy(), small.v)
    q = bf16(normal(rng, 150, 16, d))
    for m in (1, 30, 150):
        out, lse = amd.attend_fp8(g, torch.from_numpy(q[:m]).cuda().to(torch.bfloat16), want_lse=True)
        want, want_lse, mass, size = cache8.attend(small, [0, m], q[:m], d ** -0.5)
        check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), want, want_lse, mass, size, d, 150)
    weight = torch.rand(1, kv, 192, device="cuda")
    to = amd.Fp8Cache(k, v, scale, torch.tensor([[pages - 2, pages - 3]], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda"))
    kept = amd.evict_fp8(g, weight, to, 100, 4, 10)
    o = cache8.Cache(np.zeros((2, kv, 64, d), np.uint8), np.zeros((2, kv, d, 64), np.uint8), np.zeros((2, kv, 2), np.float32), [[0, 1]], [0])
    want, _ = cache8.evict(small, weight.cpu().numpy(), o, 100, 4, 10)
    assert np.array_equal(kept.cpu().numpy(), want) and same_codes(codes(k[pages - 3:pages - 1]), o.k[::-1]) and same_codes(codes(v[pages - 3:pages - 1]), o.v[::-1])


def test_many_weights():
    """More entries than a wave of the selection keeps in registers."""
    amd, rng = _amd(), np.random.default_rng(8)
    c = make(rng, [64 * 20, 64 * 20], 2, 64, width=20)
    c.table, c.length = np.tile(c.table, (1, 20))[:, :400], np.array([25000, 17000], np.int32)
    to = make(rng, [64 * 150] * 2, 2, 64)
    for kind in (lambda w: w, lambda w: np.round(w * 3) / 3, lambda w: np.zeros_like(w)):
        w = kind(rng.random((2, 2, 400 * 64))).astype(np.float32)
        o = to_gpu(amd, to)
        kept = amd.evict_fp8(to_gpu(amd, c), torch.from_numpy(w).cuda(), o, 9001, 4, 1000)
        mine = cache8.Cache(to.k, to.v, to.scale, to.table, to.length)
        want, _ = cache8.evict(c, w, mine, 9001, 4, 1000)
        assert np.array_equal(kept.cpu().numpy(), want)
        assert np.array_equal(o.scale.cpu().numpy(), mine.scale) and same_codes(codes(o.k), mine.k) and same_codes(codes(o.v), mine.v)


def test_python_calls_refuse():
    amd, rng = _amd(), np.random.default_rng(9)
    g = to_gpu(amd, make(rng, [100, 30], 2, 64))
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    lse, w = torch.zeros(2, 4, device="cuda"), torch.zeros(2, 2, g.capacity, device="cuda")
    bad = [lambda: amd.attend_fp8(g, q.float()), lambda: amd.attend_fp8(g, q[..., :32]), lambda: amd.attend_fp8(g, q.cpu()), lambda: amd.attend_fp8(g, q.transpose(0, 1)),
           lambda: amd.attend_fp8(g, q, window=-1), lambda: amd.attend_fp8(g, q, sinks=1 << 31), lambda: amd.attend_fp8(g, q, window=1 << 32),
           lambda: amd.attend_fp8(g, q, out=q.float()), lambda: amd.attend_fp8(g, q, lse=lse[:1]), lambda: amd.attend_fp8(g, q, rows=torch.zeros(2, dtype=torch.int32, device="cuda")),
           lambda: amd.attend_fp8(g, q, rows=torch.zeros(3, dtype=torch.int64, device="cuda")),
           lambda: amd.append_fp8(g, k, k.float()), lambda: amd.append_fp8(g, k, k[:1]), lambda: amd.append_fp8(g, k[:, :1], k), lambda: amd.append_fp8(g, k, k, q.float()),
           lambda: amd.append_fp8(g, k, k, q[:1]), lambda: amd.append_fp8(g, k.half(), k.half()), lambda: amd.append_fp8(g, k, k, position=torch.zeros(3, dtype=torch.int32, device="cuda")),
           lambda: amd.weigh_fp8(g, q, lse.double(), w), lambda: amd.weigh_fp8(g, q, lse, w[..., :-1]), lambda: amd.weigh_fp8(g, q, lse, w[:, :1]), lambda: amd.weigh_fp8(g, q, lse, w, sinks=-3),
           lambda: amd.evict_fp8(g, w, g, g.capacity + 1), lambda: amd.evict_fp8(g, w, g, 1 << 33), lambda: amd.evict_fp8(g, w, g, 10, -1),
           lambda: amd.evict_fp8(g, w, to_gpu(amd, make(rng, [100], 2, 64)), 10), lambda: amd.evict_fp8(g, w, g, 64, to_weight=w[..., :20])]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(i))
    refused = [lambda: amd.attend_fp8(g, q[:1]), lambda: amd.attend_fp8(g, torch.zeros(2, 3, 64, dtype=torch.bfloat16, device="cuda")), lambda: amd.attend_fp8(g, q, scale=0.0),
               lambda: amd.attend_fp8(g, q, out=q), lambda: amd.append_fp8(g, k, k, theta=0.5), lambda: amd.weigh_fp8(g, q, lse, w, scale=float("nan")),
               lambda: amd.evict_fp8(g, w, g, 64), lambda: amd.evict_fp8(g, w, g, 0), lambda: amd.attend_fp8(g, q[:0]), lambda: amd.attend_fp8(g, q[:, :0])]
    for i, call in enumerate(refused):
        with pytest.raises(amd.SpecError):
            call()
            pytest.fail(str(i))
    parts = (g.k, g.v, g.scale, g.table, g.length)
    change = lambda i, t: tuple(t if j == i else p for j, p in enumerate(parts))
    for args in (change(0, g.k.view(torch.uint8)), change(0, g.k[:, :1]), change(1, g.k[..., :32]), change(2, g.scale[..., :1]), change(2, g.scale.double()), change(3, g.table.long()),
                 change(3, g.table[:, ::2]), change(3, g.table[:, :0]), change(4, g.length[:1]), change(4, g.length.cpu()), change(0, g.k[:-1])):
        with pytest.raises(ValueError):
            amd.Fp8Cache(*args)


def test_a_captured_batch_whose_rows_move_between_its_sequences():
    """Prompts and single tokens change places between replays: rows of all sequences are looked up when a graph runs."""
    amd, rng = _amd(), np.random.default_rng(11)
    heads, kv, d, n = 8, 2, 128, 700
    g = to_gpu(amd, make(rng, [900, 900, 900, 900], kv, d))
    q = torch.from_numpy(normal(rng, n, heads, d)).cuda().to(torch.bfloat16)
    start = torch.tensor([0, 600, 601, 641, 700], dtype=torch.int32, device="cuda")
    weight = torch.zeros(4, kv, g.capacity, device="cuda")

    def step():
        weight.zero_()
        out, lse = amd.attend_fp8(g, q, start, want_lse=True)
        return out, lse, amd.weigh_fp8(g, q, lse, weight, start)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for rows in ([600, 1, 40, 59], [1, 1, 697, 1], [0, 350, 0, 350], [40, 41, 578, 41], [600, 1, 40, 59]):
        start.copy_(torch.from_numpy(starts_of(rows)))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in held]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.isfinite(got[0]).all()
        assert ((got[2].double().sum(2) - torch.tensor(rows, device="cuda")[:, None] * 4).abs() <= 2800 * 1e-4).all()
