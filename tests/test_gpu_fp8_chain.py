"""The 8-bit operators one behind the other, as the end of a forward uses them: norm -> gate/up -> rows to 8 bits -> down ->
residual add and norm -> LM head -> truncated draws and their acceptance (run with -m gpu)."""
import numpy as np
import pytest
import torch

import synth
from oracle import draws
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]
D, F, V, EPS = 528, 1360, 4112, 1e-5           # widths that end inside a block of 128
HOW = dict(temperature=0.8, top_k=60, top_p=0.9)


def _amd():
    import paper_2408_11850_amd as amd
    amd.load_library()
    return amd


def _normal(shape, std, seed):
    return synth.normal_tensor(shape, std, seed, 91, torch.float32)


class Tail:
    """Weights as a program keeps them: quantised and packed once."""

    def __init__(self, amd):
        self.amd = amd
        self.gains = [(1 + 0.3 * _normal((D,), 1.0, 1 + i)).bfloat16().cuda() for i in range(2)]
        quant = lambda n, k, seed: amd.quant_weight_fp8((_normal((n, k), 0.8 / k ** 0.5, seed)).bfloat16().cuda())
        self.gate, self.up, self.down, self.head = quant(F, D, 5), quant(F, D, 6), quant(D, F, 7), quant(V, D, 8)
        self.w_gateup = amd.pack_weights_fp8([self.gate, self.up], interleave=True)
        self.w_down, self.w_head = amd.pack_weights_fp8([self.down]), amd.pack_weights_fp8([self.head])

    def run(self, h, u):
        amd = self.amd
        x = amd.add_norm_fp8(h, None, self.gains[0], EPS)
        z = amd.gemm_fp8(*x, self.w_gateup, 2)
        zq = amd.quant_fp8(z)
        y = amd.gemm_fp8(*zq, self.w_down)
        x2 = amd.add_norm_fp8(h, y, self.gains[1], EPS)
        logits = amd.gemm_fp8(*x2, self.w_head, 0, torch.float32)
        tokens, q = amd.sample_rows(logits, u, **HOW)
        return x, z, zq, y, x2, logits, tokens, q


def _value(q, scale):
    """What e4m3 rows stand for, in 64 bits."""
    return q.double() * scale.double().t().repeat_interleave(128, 1)[:, :q.shape[1]]


def _weight(q, scale):
    return q.double() * scale.double().repeat_interleave(128, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]


def _norm(h, gain):
    h = h.double()
    return h / torch.sqrt(h.square().mean(dim=1, keepdim=True) + EPS) * gain.double()


def _near_rows(got, want):
    """e4m3 rows of `want`: half a step, 2^-4 of a value, or half of the smallest step 2^-9 of its block's scale; 2^-20 for fp32."""
    scale = torch.stack([want[:, b:b + 128].abs().amax(dim=1) / 448 for b in range(0, want.shape[1], 128)], 1)
    step = scale.repeat_interleave(128, 1)[:, :want.shape[1]] * 2.0 ** -10
    assert ((_value(*got) - want).abs() <= (2.0 ** -4 + 2.0 ** -20) * want.abs() + step * (1 + 2.0 ** -20)).all()


@pytest.mark.parametrize("M", [1, 5, 40])
def test_every_step_against_its_definition(M):
    """Each step is held to the definition on what the step before it gave."""
    amd = _amd()
    tail = Tail(amd)
    h0 = _normal((M, D), 2.0, 20 + M).cuda()
    h, u = h0.clone(), synth.uniform_array(M, 21, 5).cuda()
    x, z, zq, y, x2, logits, tokens, q = tail.run(h, u)
    _near_rows(x, _norm(h0, tail.gains[0]))
    xv = _value(*x)
    g, up = xv @ _weight(*tail.gate).t().contiguous(), xv @ _weight(*tail.up).t().contiguous()
    mag = xv.abs() @ torch.maximum(_weight(*tail.gate).abs(), _weight(*tail.up).abs()).t().contiguous()
    sums = 2.0 ** -10 * mag                    # from 33 rows on: 8 products at a time, each off by 2^-13 of the largest
    want = g * torch.sigmoid(g) * up
    assert ((z.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1.2 * sums * (up.abs() + g.abs() + sums) + 1e-6).all()
    _near_rows(zq, z.double())
    want = _value(*zq) @ _weight(*tail.down).t().contiguous()
    mag = _value(*zq).abs() @ _weight(*tail.down).abs().t().contiguous()
    assert ((y.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1.01 * 2.0 ** -10 * mag).all()
    assert torch.equal(h, h0 + y.float())
    _near_rows(x2, _norm(h, tail.gains[1]))
    want = _value(*x2) @ _weight(*tail.head).t().contiguous()
    mag = _value(*x2).abs() @ _weight(*tail.head).abs().t().contiguous()
    assert ((logits.double() - want).abs() <= (2 * 128 + 2 + 5 + 8) * 2.0 ** -24 * mag).all()
    for i in range(M):
        tok, p = draws.row(logits[i].cpu().numpy(), float(u[i]), **HOW)
        assert int(tokens[i]) == tok and np.array_equal(q[i].cpu().numpy() > 0, p > 0)


def test_a_captured_chain_repeats():
    amd = _amd()
    tail = Tail(amd)
    h, u = _normal((7, D), 2.0, 30).cuda(), synth.uniform_array(7, 22, 5).cuda()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        tail.run(h.clone(), u)
    torch.cuda.current_stream().wait_stream(st)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = tail.run(h, u)
    for rep in range(3):
        start = _normal((7, D), 2.0, 31 + rep).cuda()
        h.copy_(start)
        g.replay()
        torch.cuda.synchronize()
        eager = tail.run(start, u)
        assert torch.equal(h, start)
        for a, b in zip(out[-3:], eager[-3:]):
            assert torch.equal(a, b)


def test_a_window_is_accepted_by_the_model_that_drafted_it():
    """Draft and target are the same tail: every draft drawn from the truncated rows is accepted, and the bonus token lies in the
    truncated set."""
    amd = _amd()
    tail = Tail(amd)
    n = 6
    out = tail.run(_normal((n + 1, D), 2.0, 40).cuda(), synth.uniform_array(n + 1, 23, 5).cuda())
    logits, tokens, q = out[-3:]
    rows = amd.filter_rows(logits, **HOW)
    r = synth.uniform_array(n + 1, 24, 5)
    got, bonus = amd.accept_rows(rows, q[:n].contiguous(), tokens[:n].tolist(), (r[:n] * 0.999).tolist(), HOW["temperature"], 1.0,
                                 float(r[n]))
    assert got == n and q[n, bonus] > 0
