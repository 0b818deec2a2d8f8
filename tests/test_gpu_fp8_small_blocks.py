"""Codes of blocks near the least scale, bit by bit those of IEEE divisions (run with -m gpu): there the residual of a division needs
bits below the smallest fp32 value."""
import numpy as np
import pytest
import torch

import synth
from tests.test_gpu_fp8_codes import _codes
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]

# largest magnitude of a block and a value beside it whose quotient lies next to a border between two codes
PAIRS = """0x1.bffb12p-98 0x1.fffa6p-117  0x1.5002f6p-96 0x1.e0043cp-113  0x1.bf8768p-100 0x1.ff763p-119  0x1.bfe03ep-98 0x1.ffdbb6p-117
0x1.bfd686p-100 0x1.ffd09cp-119  0x1.500e6ap-100 0x1.500e6ap-116  0x1.bfa7e6p-99 0x1.ff9b52p-118  0x1.bfeca2p-97 0x1.ffe9ep-116
0x1.c00dfcp-99 0x1.800bfcp-116  0x1.bfad6p-99 0x1.ffa194p-118  0x1.bfeacp-97 0x1.ffe7b8p-116  0x1.c002a4p-96 0x1.800242p-113
0x1.bfffc6p-95 0x1.ffffcp-114  0x1.bffc1ap-96 0x1.7ffca8p-113  0x1.bfff5p-97 0x1.ffff38p-116  0x1.4ffc5p-98 0x1.dffabep-115
0x1.bfffa2p-94 0x1.7fffaep-111"""


def _borders():
    """All the values half way between two neighbouring codes."""
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    return (codes[1:] + codes[:-1]) / 2


def _blocks(n, seed):
    """Blocks whose largest magnitudes spread over 2^-100 .. 2^-80, their other values next to the borders."""
    r = synth.uniform_array(2 * n, seed, 1).double().view(2, n)
    top = torch.exp2(-100 + 20 * r[0]).float()
    near = ((top / 448).double()[:, None] * _borders()[None]).float()
    step = torch.from_numpy(np.spacing(near.numpy()))
    x = torch.cat([top[:, None], near + step * (torch.arange(n)[:, None] % 5 - 2), -near[:, -1:]], 1)
    return x[:, torch.randperm(128, generator=torch.Generator().manual_seed(seed))].contiguous()


def _check(x):
    import paper_2408_11850_amd as amd
    q, scale = amd.quant_fp8(x.cuda())
    want_q, want_s = _codes(x.view(x.shape[0], -1, 128))
    assert torch.equal(scale.cpu(), want_s[..., 0].t())
    assert torch.equal(q.cpu().view(torch.uint8), want_q.reshape(x.shape))


def test_values_next_to_borders():
    p = [float.fromhex(v) for v in PAIRS.split()]
    x = torch.full((len(p) // 2, 128), 2.0 ** -130)
    x[:, 5], x[:, 77] = torch.tensor(p[::2]), torch.tensor(p[1::2])
    x[:, 78] = -x[:, 77]
    _check(x)
    _check(torch.cat([x, torch.ones_like(x), x.flip(0)], 1))           # beside blocks of an ordinary size


@pytest.mark.parametrize("seed", [161, 162])
def test_small_blocks(seed):
    _check(_blocks(200000, seed))


def test_the_least_scale():
    """Every 64th value from 2^-121 to 2^-100, and zeros."""
    lo, hi = (int(np.float32(v).view(np.int32)) for v in (2.0 ** -121, 2.0 ** -100))
    x = torch.arange(lo, hi, 64, dtype=torch.int32).view(torch.float32).reshape(-1, 128)
    _check(torch.cat([x, torch.zeros(3, 128)]))


def test_small_weights():
    import paper_2408_11850_amd as amd
    w = (synth.normal_tensor((256, 256), 1.0, 163, 1, torch.float32) * 2.0 ** -101).bfloat16()
    q, scale = amd.quant_weight_fp8(w.cuda())
    want_q, want_s = _codes(w.float().view(2, 128, 2, 128).transpose(1, 2).reshape(2, 2, 128 * 128))
    assert torch.equal(scale.cpu(), want_s[..., 0])
    want_q = want_q.view(2, 2, 128, 128).transpose(1, 2).reshape(256, 256)
    assert torch.equal(q.cpu().view(torch.uint8), want_q)
