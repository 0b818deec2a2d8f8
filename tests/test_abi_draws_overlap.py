"""Truncated draws: results and workspaces that overlap each other or what is read are refused on the host (no GPU is needed for
these; that neighbours and rows between rows are taken needs one)."""
import ctypes as C
import os

import pytest
import torch

import synth
from tests.util import gpu_available

N, V, LD = 3, 100, 250
ROW, ALL = 4 * V, 4 * V * N


@pytest.fixture(scope="module")
def amd():
    import paper_2408_11850_amd as amd
    if not os.path.exists(amd.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    amd.load_library()
    return amd


# addresses far from each other that are never read
AT = dict(logits=1 << 20, u=2 << 20, q=3 << 20, masked=4 << 20, tok=5 << 20, work=1 << 24)


def _call(lib, amd, a, temperature=1.0):
    s = amd.Sampling(temperature, 1.0, 0, 1.0, 0.0)
    return lib.spec_sample_rows(a["logits"], a.get("ld", LD), N, V, C.byref(s), a["u"], a["q"], a["masked"], a["tok"], a["work"], None)


@pytest.mark.parametrize("change", [
    dict(q=AT["logits"] + 4), dict(q=AT["logits"] - 4), dict(masked=AT["logits"] + ROW - 4), dict(q=AT["logits"] - ALL + 4),
    dict(masked=AT["logits"] + 4 * (LD - 1)), dict(q=AT["logits"] + 4 * (2 * LD + V - 1)), dict(masked=AT["logits"] + 4 * LD),
    dict(tok=AT["logits"]), dict(tok=AT["logits"] + 4 * (LD - 2)), dict(work=AT["logits"]), dict(work=AT["logits"] - 16),
    dict(q=AT["u"]), dict(tok=AT["u"]), dict(work=AT["u"] - 32), dict(q=AT["masked"] + 4), dict(masked=AT["q"] + ALL - 4),
    dict(tok=AT["q"] + 8), dict(work=AT["q"]), dict(work=AT["masked"] + 16), dict(work=AT["tok"]),
    dict(logits=AT["q"], ld=V, masked=AT["q"] + 4), dict(logits=AT["q"], ld=V, tok=AT["q"]),
    dict(logits=AT["masked"], ld=V, u=AT["masked"] + 4)], ids=str)
def test_refuses(amd, change):
    lib = amd.load_library()
    a = {**AT, **change}
    if a["logits"] == a["q"]:
        a["masked"] = change.get("masked")
    assert _call(lib, amd, a) == amd.SPEC_E_INVAL
    assert b"overlap" in lib.spec_last_error()


@pytest.mark.gpu
@pytest.mark.skipif(not gpu_available(), reason="needs a GPU")
def test_neighbours_and_gaps(amd):
    """One allocation for everything: results between the rows of the logits, and right behind each other."""
    lib = amd.load_library()
    x = synth.normal_tensor((N, V), 2.0, 150, 1, torch.float32).cuda()
    u = torch.tensor([0.1, 0.5, 0.9], device="cuda")
    tokens, q = amd.sample_rows(x, u, top_p=0.9)
    ld = 2000
    big = torch.full((8 * ld,), -1.0, device="cuda")
    rows = big.as_strided((N, V), (ld, 1), 8)
    rows.copy_(x)
    base = big.data_ptr()
    work = torch.empty(lib.spec_sample_rows_workspace_bytes(N, V), dtype=torch.uint8, device="cuda")
    at = lambda i: base + 4 * i
    a = dict(logits=at(8), ld=ld, u=u.data_ptr(), q=at(8 + V), masked=at(8 + V + N * V), tok=at(8 + V + 2 * N * V), work=work.data_ptr())
    s = amd.Sampling(1.0, 1.0, 0, 0.9, 0.0)
    amd.check(lib.spec_sample_rows(a["logits"], ld, N, V, C.byref(s), a["u"], a["q"], a["masked"], a["tok"], a["work"],
                                   torch.cuda.current_stream().cuda_stream))
    assert torch.equal(rows, x) and torch.equal(big[8 + V:8 + V + N * V].view(N, V), q)
    assert torch.equal(big[8 + V + N * V:8 + V + 2 * N * V].view(N, V), amd.filter_rows(x, top_p=0.9))
    assert torch.equal(big.view(torch.int32)[8 + V + 2 * N * V:][:N], tokens)
    assert (big[8 + V + 2 * N * V + N:8 + ld] == -1).all() and (big[:8] == -1).all()
    own = torch.cat([x.flatten(), torch.zeros(7, device="cuda")])
    with pytest.raises(amd.SpecError):
        amd.filter_rows(own[:N * V].view(N, V), out=own[7:].view(N, V))
    assert torch.equal(own[:N * V].view(N, V), x)


@pytest.mark.parametrize("ld", [1 << 40, 1 << 61, 1 << 62, (1 << 63) - 1])
def test_far_rows(amd, ld):
    """Strides whose bytes do not fit 64 bits: the first row is looked at all the same."""
    lib = amd.load_library()
    for change in (dict(q=AT["logits"] + ROW - 4), dict(work=AT["logits"]), dict(masked=AT["logits"] - 4)):
        assert _call(lib, amd, {**AT, **change, "ld": ld}) == amd.SPEC_E_INVAL
        assert b"overlap" in lib.spec_last_error()
