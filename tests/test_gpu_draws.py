"""Truncated draws against the oracle in 64 bits: the same ids kept, the same token, q to its rounding (run with -m gpu)."""
import numpy as np
import pytest
import torch

import synth
from oracle import draws, sampling
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]
NAN, INF = float("nan"), float("inf")


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _logits(n, V, seed, coarse=False):
    x = synth.normal_tensor((n, V), 2.5, seed, V, torch.float32)
    for i in range(n):
        x[i, (torch.arange(min(V, 20)) * 7919 + 13 * i) % V] += 5
    return x.bfloat16().float() if coarse else x


def _u(n, seed):
    return synth.uniform_array(n, seed, 77)


def _check(x, u, tokens, q, masked, **how):
    x, V = x.cpu().numpy(), x.shape[1]
    for i in range(x.shape[0]):
        tok, want = draws.row(x[i], float(u[i]), **how)
        if tokens is not None:
            assert int(tokens[i]) == tok, (i, how)
        if tok < 0:                                       # no distribution
            assert all(t is None or t[i].isnan().all() for t in (q, masked)), (i, how)
            continue
        w = draws.weights(x[i], **how)
        full = np.exp((x[i].astype(np.float64) - x[i].max()) * how.get("logit_scale", 1.0) / (how.get("temperature", 1.0) or 1.0))
        kept, low = w > 0, full < 1e-300                  # below that a kept weight may be 0 in one of the two
        if masked is not None:
            m = masked[i].cpu().numpy()
            assert np.array_equal(m[kept & ~low], x[i][kept & ~low]), (i, how)
            assert (m[~kept & ~low] == -np.inf).all(), (i, how)
        if q is not None:
            g = q[i].double().cpu().numpy()
            assert np.array_equal(g[~kept], np.zeros((~kept).sum())), (i, how)
            # one rounding to fp32, and a total whose every term is off by at most 2^-44 of the largest weight
            assert (np.abs(g - want)[kept] <= (2.0 ** -24 + V * 2.0 ** -44 + 1e-12) * want[kept] + 2.0 ** -149).all(), (i, how)


SETTINGS = [dict(), dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.02), dict(top_k=40, top_p=0.95),
            dict(top_k=500, top_p=0.7, min_p=0.01, temperature=0.7), dict(top_p=0.999, temperature=1.5), dict(top_p=0.0),
            dict(temperature=0.0), dict(min_p=1.0), dict(top_k=3000, logit_scale=0.5), dict(top_p=0.5, temperature=4.0)]


@pytest.mark.parametrize("V", [1, 2, 5, 63, 1000, 8191, 8192, 8193, 32000, 50257, 128256, 262147])
@pytest.mark.parametrize("how", SETTINGS, ids=str)
@pytest.mark.parametrize("coarse", [False, True])
def test_rows(V, how, coarse):
    amd = _amd()
    print(f"draws V={V} {how} coarse={coarse}", flush=True)
    n = 3 if V <= 50257 else 2
    x, u = _logits(n, V, 51, coarse), _u(n, V)
    xd = x.cuda()
    tokens, q = amd.sample_rows(xd, u.cuda(), **how)
    masked = amd.filter_rows(xd, **how)
    assert torch.equal(xd.cpu(), x)
    _check(x, u, tokens, q, masked, **how)
    assert torch.equal(masked > -INF, q > 0)
    only, none = amd.sample_rows(xd, u.cuda(), want_q=False, **how)
    assert none is None and torch.equal(only, tokens)


@pytest.mark.parametrize("V", [4, 5000, 40000, 140000])
@pytest.mark.parametrize("how", [dict(top_k=2), dict(top_p=0.5), dict(top_k=3, top_p=0.5), dict(min_p=1.0), dict()], ids=str)
def test_equal_logits(V, how):
    """Every id is a candidate, the border falls between equal ones: rising ids.  40000 of them do not fit a list."""
    amd = _amd()
    how = dict(how)
    if "top_k" in how and V > 4:
        how["top_k"] = V // 2 + 1
    x = torch.full((2, V), -1.25)
    x[1] = 3.0
    x[1, V - 1] = 3.5
    tokens, q = amd.sample_rows(x.cuda(), torch.tensor([0.0, 0.999]).cuda(), **how)
    _check(x, [0.0, 0.999], tokens, q, amd.filter_rows(x.cuda(), **how), **how)


@pytest.mark.parametrize("how", [dict(), dict(top_k=20), dict(top_p=0.8), dict(top_k=30000, top_p=0.99)], ids=str)
def test_masked_and_extreme_logits(how):
    """-inf in halves and everywhere but one place, the type's lowest value, zeros of both signs, far tails."""
    amd = _amd()
    V = 40000
    x = _logits(6, V, 52)
    x[0, :V // 2] = -INF
    x[1] = -INF
    x[1, 31000] = -7.0
    x[2] = torch.finfo(torch.float32).min
    x[2, 5] = 0.0
    x[3] = 0.0
    x[3, ::2] = -0.0
    x[4] = torch.linspace(-3e38, 3e38, V)                 # overflows on the way: no distribution
    x[5] = torch.linspace(0, -1e4, V)
    x = torch.cat([x, ((torch.arange(V, dtype=torch.float64) - V // 2) * (3.0e38 / V)).float()[None]])
    u = _u(7, 3)
    tokens, q = amd.sample_rows(x.cuda(), u.cuda(), **how)
    _check(x, u, tokens, q, amd.filter_rows(x.cuda(), **how), **how)


@pytest.mark.parametrize("V", [1000, 40000])
@pytest.mark.parametrize("how", [dict(), dict(top_k=7), dict(top_p=0.9), dict(min_p=0.5)], ids=str)
def test_rows_without_a_distribution(V, how):
    """Beside rows that have one, whose results do not change."""
    amd = _amd()
    x = _logits(6, V, 53)
    x[1] = -INF
    x[2, V // 2] = NAN
    x[3, 4] = INF
    x[4] = NAN
    u = _u(6, 4)
    tokens, q = amd.sample_rows(x.cuda(), u.cuda(), **how)
    masked = amd.filter_rows(x.cuda(), **how)
    for i in (1, 2, 3, 4):
        assert int(tokens[i]) == -1 and q[i].isnan().all() and masked[i].isnan().all()
    good = torch.tensor([0, 5])
    _check(x[good], u[good], tokens.cpu()[good], q.cpu()[good], masked.cpu()[good], **how)


def test_greedy_rows():
    amd = _amd()
    x = torch.full((5, 20000), -INF)
    x[1] = NAN
    x[1, 5] = x[1, 17000] = -2.0
    x[2, 9000] = 1.0
    x[3] = 0.0
    x[4] = _logits(1, 20000, 54)[0]
    tokens, q = amd.sample_rows(x.cuda(), None, temperature=0.0, top_k=3, top_p=0.5)
    want = [0, 5, 9000, 0, int(x[4].argmax())]
    assert tokens.tolist() == want
    assert (q.sum(1) == 1).all() and [int(r.argmax()) for r in q] == want
    masked = amd.filter_rows(x.cuda(), temperature=0.0)
    assert (masked[2] > -INF).sum() == 1 and masked[2, 9000] == 1.0


def test_uniforms_at_the_ends():
    amd = _amd()
    x = _logits(1, 9000, 55).repeat(7, 1)
    u = torch.tensor([0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, NAN, 2.0 ** -30])
    tokens, q = amd.sample_rows(x.cuda(), u.cuda(), top_k=100)
    ids = torch.nonzero(q[0] > 0)[:, 0].tolist()
    assert tokens.tolist() == [ids[0], ids[-1], ids[-1], ids[-1], ids[0], ids[0], ids[0]]


def test_strided_rows_odd_addresses_and_results_in_place():
    amd = _amd()
    n, V = 3, 10001
    big = _logits(n, V + 10, 56).cuda()
    x = big[:, 3:3 + V]
    u = _u(n, 5).cuda()
    how = dict(top_k=900, top_p=0.9)
    ref = amd.sample_rows(x.contiguous(), u, **how)
    got = amd.sample_rows(x, u, **how)
    assert torch.equal(ref[0], got[0]) and torch.equal(ref[1], got[1])
    masked = amd.filter_rows(x, **how)
    own = x.contiguous()
    assert amd.filter_rows(own, out=own, **how) is own and torch.equal(own, masked)
    import ctypes as C
    own = x.contiguous()
    work = torch.empty(amd.load_library().spec_sample_rows_workspace_bytes(n, V), dtype=torch.uint8, device="cuda")
    s = amd.Sampling(1.0, 1.0, 900, 0.9, 0.0)
    amd.check(amd.load_library().spec_sample_rows(own.data_ptr(), V, n, V, C.byref(s), None, own.data_ptr(), None, None,
                                                  work.data_ptr(), torch.cuda.current_stream().cuda_stream))
    assert torch.equal(own, ref[1])


@pytest.mark.parametrize("V", [270001, 600001, 1048576])
@pytest.mark.parametrize("how", [dict(), dict(top_k=1000), dict(top_k=5000, top_p=0.9), dict(top_p=0.95, temperature=1.3), dict(min_p=0.001)],
                         ids=str)
def test_the_longest_rows(V, how):
    """Chunks of every size; more groups than registers hold; nuclei of tens of thousands of ids."""
    amd = _amd()
    print(f"draws V={V} {how}", flush=True)
    x, u = _logits(1, V, 130), _u(1, 8)
    tokens, q = amd.sample_rows(x.cuda(), u.cuda(), **how)
    _check(x, u, tokens, q, amd.filter_rows(x.cuda(), **how), **how)


@pytest.mark.parametrize("how", [dict(top_k=7), dict(top_p=0.7), dict(min_p=0.2), dict()], ids=str)
def test_many_rows(how):
    amd = _amd()
    n, V = 3001, 67
    x, u = _logits(n, V, 131), _u(n, 9)
    tokens, q = amd.sample_rows(x.cuda(), u.cuda(), **how)
    some = torch.tensor([0, 1, 1500, 2999, 3000])
    _check(x[some], u[some], tokens.cpu()[some], q.cpu()[some], None, **how)
    one = [amd.sample_rows(x[i:i + 1].cuda(), u[i:i + 1].cuda(), **how)[0] for i in range(0, n, 500)]
    assert torch.equal(torch.cat(one), tokens[::500])


def test_every_result_of_one_call():
    """q, the truncated logits and the tokens together are what calls of their own give."""
    import ctypes as C
    amd = _amd()
    n, V = 3, 33333
    x, u = _logits(n, V, 132).cuda(), _u(n, 10).cuda()
    lib = amd.load_library()
    for how in (dict(), dict(top_k=30), dict(top_k=3000, top_p=0.6), dict(top_p=0.9, min_p=0.0001), dict(temperature=0.0)):
        q, m = torch.empty_like(x), torch.empty_like(x)
        tok = torch.empty(n, dtype=torch.int32, device="cuda")
        work = torch.empty(lib.spec_sample_rows_workspace_bytes(n, V), dtype=torch.uint8, device="cuda")
        s = amd.Sampling(how.get("temperature", 1.0), 1.0, how.get("top_k", 0), how.get("top_p", 1.0), how.get("min_p", 0.0))
        amd.check(lib.spec_sample_rows(x.data_ptr(), V, n, V, C.byref(s), u.data_ptr(), q.data_ptr(), m.data_ptr(), tok.data_ptr(),
                                       work.data_ptr(), torch.cuda.current_stream().cuda_stream))
        ref = amd.sample_rows(x, u, **how)
        assert torch.equal(tok, ref[0]) and torch.equal(q, ref[1]) and torch.equal(m, amd.filter_rows(x, **how))


def test_streams_graphs_and_repeats():
    amd = _amd()
    x, u = _logits(4, 70000, 57, True).cuda(), _u(4, 6).cuda()
    how = dict(top_k=2000, top_p=0.97, min_p=0.001)
    ref = amd.sample_rows(x, u, **how)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        a = amd.sample_rows(x, u, **how)
    b = amd.sample_rows(x, u, **how)
    torch.cuda.synchronize()
    for got in (a, b):
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tokens, q = amd.sample_rows(x, u, **how)
    for rep in range(3):
        x.copy_(_logits(4, 70000, 58 + rep, rep == 1))
        g.replay()
        torch.cuda.synchronize()
        want = amd.sample_rows(x, u, **how)
        assert torch.equal(tokens, want[0]) and torch.equal(q, want[1])
        _check(x.cpu(), u.cpu(), tokens, q, None, **how)


@pytest.mark.parametrize("how", [dict(top_k=8), dict(top_p=0.8, temperature=0.8), dict(min_p=0.1, logit_scale=1.5)], ids=str)
def test_acceptance_of_truncated_rows(how):
    """Speculative sampling with both models truncated alike: sample_rows gives the drafts and their q, filter_rows the target's
    rows for accept_rows; the outcome is the oracle's on the truncated distributions, up to decisions that fp32 can flip."""
    amd = _amd()
    V, n = 5000, 4
    temp, scale = how.get("temperature", 1.0), how.get("logit_scale", 1.0)
    accepted = 0
    for rep in range(12):
        target = _logits(n + 1, V, 60 + rep)
        draft = target[:n] + synth.normal_tensor((n, V), 0.3, 80 + rep, V, torch.float32)
        u, r = _u(n, 90 + rep), _u(n + 1, 110 + rep)
        x, q = amd.sample_rows(draft.cuda(), u.cuda(), **how)
        rows = amd.filter_rows(target.cuda(), **how)
        got = amd.accept_rows(rows, q, x.tolist(), r[:n].tolist(), temp, scale, float(r[n]))
        p = [w / w.sum() for w in (draws.weights(t, **how) for t in target.numpy())]
        qs = [draws.row(d, 0.5, **how)[1] for d in draft.numpy()]
        margin, k = 1.0, 0
        while k < n:
            margin = min(margin, sampling.accept_margin(p[k], qs[k], int(x[k]), float(r[k])))
            if not sampling.accept(p[k], qs[k], int(x[k]), float(r[k])):
                break
            k += 1
        w = sampling.residual(p[k], qs[k]) if k < n else p[k]
        w = w if w.sum() > 0 else p[k]
        margin = min(margin, sampling.sample_margin(w, float(r[n])))
        if margin > 2e-5:                                 # the acceptance's own fp32 rounding
            assert got == (k, sampling.sample(w, float(r[n]))), rep
            accepted += k
    assert accepted > 0
