"""The attention of an 8-bit forward, every step against 64 bits on what the step before it gave (run with -m gpu)."""
import numpy as np
import pytest
import torch

import synth
from oracle import cache8
from tests.cache8 import check_attention, codes, make, normal, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


@pytest.mark.parametrize("m,heads,kv,d", [(6, 4, 2, 64), (1, 8, 2, 128), (40, 8, 1, 64)])
def test_every_step_from_qkv_to_the_output_projection(m, heads, kv, d):
    import paper_2408_11850_amd as amd
    amd.load_library()
    rng, D, n = np.random.default_rng(2), 256, 200
    quant = lambda rows, k, seed: amd.quant_weight_fp8(synth.normal_tensor((rows, k), 0.06, seed, 3, torch.float32).bfloat16().cuda())
    wo = quant(D, heads * d, 4)
    wqkv = amd.pack_weights_fp8([quant(heads * d, D, 1), quant(kv * d, D, 2), quant(kv * d, D, 3)])
    c = make(rng, [n - m], kv, d)
    c.table = np.pad(c.table, ((0, 0), (0, 1)))
    free = [p for p in range(c.k.shape[0]) if p not in c.table[0, :-(-(n - m) // 64)]]
    c.table[0, -(-(n - m) // 64):-(-n // 64)] = free[:-(-n // 64) - -(-(n - m) // 64)]
    g = to_gpu(amd, c)
    h = torch.from_numpy(normal(rng, m, D)).cuda()
    qkv = amd.gemm_fp8(*amd.add_norm_fp8(h, None, torch.ones(D, dtype=torch.bfloat16, device="cuda"), 1e-5), wqkv)
    q, k, v = (qkv[:, a * d:b * d].unflatten(1, (b - a, d)) for a, b in ((0, heads), (heads, heads + kv), (heads + kv, heads + 2 * kv)))
    g.length += m
    qr = amd.append_fp8(g, k, v, q, theta=10000.0)
    out, lse = amd.attend_fp8(g, qr, want_lse=True)
    x, xs = amd.quant_fp8(out.flatten(1))
    y = amd.gemm_fp8(x, xs, amd.pack_weights_fp8([wo]), 0, torch.float32)
    now = cache8.Cache(codes(g.k), codes(g.v), g.scale.cpu().numpy(), g.table.cpu().numpy(), g.length.cpu().numpy())
    # q: rotated in fp32, rounded to bf16; keys and values: half a step of their codes (2^-4 of a value, 2^-10 of the scale)
    at = n - m + np.arange(m)
    wide = lambda t: t.double().cpu().numpy()
    want = cache8.rotate(wide(q), at, 10000.0)
    size = np.abs(wide(q))
    size = np.concatenate([size[..., :d // 2] + size[..., d // 2:]] * 2, -1)
    assert (np.abs(wide(qr) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * size).all()
    for head in range(kv):
        for got, rows, which in zip(now.entries(0, head), (cache8.rotate(wide(k), at, 10000.0), wide(v)), (0, 1)):
            step = now.scale[now.table[0, at // 64], head, which][:, None]
            assert (np.abs(got[n - m:] - rows[:, head]) <= (2.0 ** -4 + 2.0 ** -20) * np.abs(rows[:, head]) + 2.0 ** -10 * step + 2.0 ** -20).all()
    # the attention of the q that the append gave
    want, want_lse, mass, size = cache8.attend(now, [0, m], qr.float().cpu().numpy(), d ** -0.5)
    check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), want, want_lse, mass, size, d, n)
    # its rows in 8 bits (a block's scale by its largest value over 448), and their product with the weights: fp32 sums of blocks of 128,
    # from 33 rows on 8 products at a time, each off by less than 2^-13 of the largest
    K = heads * d
    value = wide(x) * wide(xs).T.repeat(128, 1)[:, :K]
    flat = wide(out).reshape(m, K)
    assert (np.abs(value - flat) <= (2.0 ** -4 + 2.0 ** -20) * np.abs(flat) + wide(xs).T.repeat(128, 1)[:, :K] * 2.0 ** -10 * 1.01).all()
    w = wide(wo[0]) * wide(wo[1]).repeat(128, 0)[:D].repeat(128, 1)[:, :K]
    magnitude = np.abs(value) @ np.abs(w).T
    bound = ((128 * 2 + 2 + -(-K // 128) + 8) * 2.0 ** -24 + (2.0 ** -10 if m > 32 else 0)) * magnitude
    assert (np.abs(wide(y) - value @ w.T) <= bound).all()
