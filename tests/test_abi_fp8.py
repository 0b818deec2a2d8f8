"""Refusals of the 8-bit operand calls: found on the host, before anything is launched (no GPU is needed)."""
import ctypes as C
import os

import pytest
import torch


@pytest.fixture(scope="module")
def amd():
    import paper_2408_11850_amd as amd
    if not os.path.exists(amd.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    amd.load_library()
    return amd


P = 4096          # an address that is aligned to everything and never read


def _norm(lib, **change):
    a = dict(h=P, ht=0, ldh=256, delta=P, dt=0, ldd=256, gain=P, eps=1e-5, M=2, d=256, q=P, s=P)
    a.update(change)
    return lib.spec_add_norm_quant(a["h"], a["ht"], a["ldh"], a["delta"], a["dt"], a["ldd"], a["gain"], a["eps"], a["M"], a["d"],
                                 a["q"], a["s"], None)


@pytest.mark.parametrize("change", [
    dict(h=None), dict(gain=None), dict(q=None), dict(s=None), dict(ht=2), dict(dt=-1), dict(M=0), dict(M=-1), dict(d=0),
    dict(d=8), dict(d=250), dict(d=32784, ldh=40000, ldd=40000), dict(ldh=255), dict(ldh=0), dict(ldd=128), dict(ldd=-256),
    dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(h=P + 2), dict(ht=1, h=P + 1),
    dict(delta=P + 2), dict(gain=P + 1), dict(q=P + 4), dict(s=P + 2)], ids=str)
def test_add_norm_refuses(amd, change):
    assert _norm(amd.load_library(), **change) == amd.SPEC_E_INVAL


@pytest.mark.parametrize("change", [dict(x=None), dict(q=None), dict(s=None), dict(t=5), dict(M=0), dict(K=24), dict(K=40000, ld=40000),
                                    dict(ld=100), dict(ld=-1), dict(x=P + 1), dict(t=0, x=P + 2), dict(q=P + 4)], ids=str)
def test_quant_refuses(amd, change):
    a = dict(x=P, t=1, ld=256, M=2, K=256, q=P, s=P)
    a.update(change)
    assert amd.load_library().spec_quant_rows(a["x"], a["t"], a["ld"], a["M"], a["K"], a["q"], a["s"], None) == amd.SPEC_E_INVAL


def test_weight_calls_refuse(amd):
    lib, bad = amd.load_library(), amd.SPEC_E_INVAL
    assert lib.spec_quant_weight(None, 32, 64, P, P, None) == bad
    assert lib.spec_quant_weight(P, 24, 64, P, P, None) == bad
    assert lib.spec_quant_weight(P, 32, 72, P, P, None) == bad
    assert lib.spec_quant_weight(P + 1, 32, 64, P, P, None) == bad
    assert lib.spec_pack_quant(P, P, P, None, 32, 64, 0, 1, None) == bad
    assert lib.spec_pack_quant(P, P, P, P, 32, 64, -1, 1, None) == bad
    assert lib.spec_pack_quant(P, P, P, P, 32, 64, 0, 0, None) == bad
    assert lib.spec_pack_quant(P + 8, P, P, P, 32, 64, 0, 1, None) == bad
    assert lib.spec_pack_quant(P, P, P, P, 32, 8, 0, 1, None) == bad
    assert lib.spec_packed_quant_bytes(32, 144) == 2 * 2 * 2048        # 2 panels x ceil(144 / 128) blocks x 2 KiB
    assert lib.spec_packed_quant_bytes(40, 144) == 0


@pytest.mark.parametrize("change", [
    dict(x=None), dict(xs=None), dict(w=None), dict(ws=None), dict(out=None), dict(epi=1), dict(epi=3), dict(epi=-1), dict(t=2),
    dict(epi=2, t=0), dict(M=0), dict(N=0), dict(N=24), dict(epi=2, t=1, N=48), dict(K=0), dict(K=72), dict(K=2 << 20),
    dict(N=2 << 20), dict(M=1 << 28, K=256), dict(x=P + 8), dict(w=P + 8), dict(out=P + 8), dict(t=1, out=P + 4), dict(xs=P + 2)],
    ids=str)
def test_gemm_refuses(amd, change):
    a = dict(out=P, t=0, x=P, xs=P, w=P, ws=P, M=2, N=64, K=128, epi=0)
    a.update(change)
    assert amd.load_library().spec_gemm_quant(a["out"], a["t"], a["x"], a["xs"], a["w"], a["ws"], a["M"], a["N"], a["K"], a["epi"],
                                              None) == amd.SPEC_E_INVAL


def test_python_calls_refuse_host_tensors_and_wrong_types(amd):
    h, gain = torch.zeros(2, 256), torch.ones(256, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        amd.add_norm_fp8(h, None, gain, 1e-5)
    with pytest.raises(ValueError):
        amd.quant_fp8(h)
    with pytest.raises(ValueError):
        amd.quant_weight_fp8(h.bfloat16())
    with pytest.raises(ValueError):
        amd.pack_weights_fp8([])
    with pytest.raises(ValueError):
        amd.pack_weights_fp8([(h.to(torch.float8_e4m3fn), torch.ones(1, 2))])


@pytest.mark.parametrize("M,d", [(1 << 26, 16), (1 << 26, 512), (1 << 25, 528), (1 << 22, 8192), (1 << 20, 32768), (2 ** 31 - 1, 32768)])
def test_rows_beyond_a_launch(amd, M, d):
    assert _norm(amd.load_library(), M=M, d=d, ldh=d, ldd=d) == amd.SPEC_E_INVAL
    assert amd.load_library().spec_quant_rows(P, 1, d, M, d, P, P, None) == amd.SPEC_E_INVAL
