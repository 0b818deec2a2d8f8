"""8-bit operands: sizes whose low 32 bits alone would be sizes too are refused (run with -m gpu)."""
import pytest
import torch

from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]
WIDE = (1 << 32) + 128


@pytest.fixture(autouse=True)
def give_back():
    """The large tensors do not stay in the allocator's cache."""
    yield
    torch.cuda.empty_cache()


def test_columns_of_rows():
    import paper_2408_11850_amd as amd
    x = torch.empty((1, WIDE), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        amd.quant_fp8(x)
    with pytest.raises(ValueError):
        amd.add_norm_fp8(x, None, x[0], 1e-5)


def test_sizes_of_weights():
    import paper_2408_11850_amd as amd
    for shape in ((0, WIDE), (WIDE, 0)):                            # no element, refused for the size
        with pytest.raises(ValueError):
            amd.quant_weight_fp8(torch.empty(shape, dtype=torch.bfloat16, device="cuda"))
    q = torch.empty((WIDE, 16), dtype=torch.float8_e4m3fn, device="cuda")
    with pytest.raises(ValueError, match="2\\^31"):
        amd.pack_weights_fp8([(q, torch.empty((WIDE // 128, 1), device="cuda"))])
