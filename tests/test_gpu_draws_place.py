"""Truncated draws in place and with whatever a workspace holds, over every way a row can take (run with -m gpu)."""
import ctypes as C

import pytest
import torch

import synth
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]
WAYS = [dict(), dict(temperature=0.0), dict(min_p=0.01), dict(top_k=40), dict(top_k=900, top_p=0.9, min_p=0.001), dict(top_k=4000),
        dict(top_p=0.9), dict(top_p=0.999, temperature=2.0)]


def _call(amd, x, u, q, masked, tok, how, fill):
    lib, (n, V) = amd.load_library(), x.shape
    work = torch.full((lib.spec_sample_rows_workspace_bytes(n, V),), fill, dtype=torch.uint8, device="cuda")
    s = amd.Sampling(how.get("temperature", 1.0), 1.0, how.get("top_k", 0), how.get("top_p", 1.0), how.get("min_p", 0.0))
    ptr = [t.data_ptr() if t is not None else None for t in (u, q, masked, tok, work)]
    amd.check(lib.spec_sample_rows(x.data_ptr(), V, n, V, C.byref(s), *ptr, torch.cuda.current_stream().cuda_stream))


@pytest.mark.parametrize("V", [7, 5000, 70001])
@pytest.mark.parametrize("how", WAYS, ids=str)
def test_in_place_and_workspace(V, how):
    import paper_2408_11850_amd as amd
    print(f"in place V={V} {how}", flush=True)
    n = 3
    x = (3 * synth.normal_tensor((n, V), 1.0, 71, V, torch.float32)).cuda()
    x[1, V // 2] = -float("inf")
    u = torch.tensor([0.1, 0.5, 0.97], device="cuda")
    q, masked, tok = torch.empty_like(x), torch.empty_like(x), torch.empty(n, dtype=torch.int32, device="cuda")
    _call(amd, x, u, q, masked, tok, how, 0)
    want = amd.sample_rows(x, u, **how)
    assert torch.equal(tok, want[0]) and torch.equal(q, want[1])
    for fill in (0x00, 0x7f, 0xff):
        for which in ("q", "masked", "both", "none"):
            own, other, t = x.clone(), torch.full_like(x, float("nan")), torch.full_like(tok, -7)
            if which == "q":
                _call(amd, own, u, own, None, t, how, fill)
                assert torch.equal(own, q)
            elif which == "masked":
                _call(amd, own, u, None, own, t, how, fill)
                assert torch.equal(own, masked)
            elif which == "both":
                _call(amd, own, u, own, other, t, how, fill)
                assert torch.equal(own, q) and torch.equal(other, masked)
            else:
                _call(amd, own, u, None, None, t, how, fill)
                assert torch.equal(own, x)
            assert torch.equal(t, tok)
