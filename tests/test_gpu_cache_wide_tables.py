"""The same batch under tables of other widths (run with -m gpu)."""
import numpy as np
import pytest
import torch

from oracle import cache8
from tests.cache8 import EPS, bf16, check_attention, make, normal, starts_of, to_gpu
from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


@pytest.mark.parametrize("width", [40, 1000, 1 << 17])
@pytest.mark.parametrize("window,sinks", [(1000, 0), (100, 70), (1, 0)])
@pytest.mark.parametrize("lengths,rows,heads,kv,d", [([1500], [1100], 16, 1, 64), ([2500], [600], 8, 2, 128), ([2100, 300, 700], [700, 1, 90], 8, 1, 128)])
def test_weights_and_attention_under_a_window(lengths, rows, heads, kv, d, window, sinks, width):
    """Sums of slices stand by the pages that are seen: as many as the window and the rows allow, whatever the table's width."""
    import paper_2408_11850_amd as amd
    amd.load_library()
    rng = np.random.default_rng(sum(rows))
    c = make(rng, lengths, kv, d, width=40)
    start, n = starts_of(rows), sum(rows)
    q = bf16(normal(rng, n, heads, d))
    qg, sg = torch.from_numpy(q).cuda().to(torch.bfloat16), torch.from_numpy(start).cuda()
    want, want_lse, mass, size = cache8.attend(c, start, q, d ** -0.5, window, sinks)
    wide = to_gpu(amd, c)
    table = torch.full((len(lengths), width), -1, dtype=torch.int32, device="cuda")
    table[:, :40] = wide.table
    g = amd.Fp8Cache(wide.k, wide.v, wide.scale, table, wide.length)
    out, lse = amd.attend_fp8(g, qg, sg, window=window, sinks=sinks, want_lse=True)
    check_attention(out.float().cpu().numpy(), lse.cpu().numpy(), want, want_lse, mass, size, d, max(lengths))
    weight = rng.random((len(lengths), kv, 40 * 64)).astype(np.float32)
    w = torch.full((len(lengths), kv, g.capacity), 7.0, device="cuda")
    w[..., :40 * 64] = torch.from_numpy(weight).cuda()
    amd.weigh_fp8(g, qg, lse, w, sg, window=window, sinks=sinks)
    want, slack = cache8.weigh(c, start, q, lse.cpu().numpy(), weight, d ** -0.5, window, sinks)
    bound = slack * (d + 5) * EPS * 1.1 + want * (max(rows) * heads // kv + 48) * EPS
    assert (np.abs(w[..., :40 * 64].cpu().numpy() - want) <= bound + 1e-37).all() and (w[..., 40 * 64:] == 7).all()
