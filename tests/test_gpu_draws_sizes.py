"""Truncated draws: sizes whose low 32 bits alone would be sizes too are refused (run with -m gpu)."""
import pytest
import torch

from tests.util import gpu_available

pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not gpu_available(), reason="needs a GPU")]


@pytest.fixture(autouse=True)
def give_back():
    """The large tensors do not stay in the allocator's cache."""
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [(1 << 32) + 1, 1 << 31])
def test_rows(n):
    import paper_2408_11850_amd as amd
    x = torch.zeros((1, 1), device="cuda").expand(n, 1)          # one element; refused before anything of n rows is made
    with pytest.raises(ValueError):
        amd.sample_rows(x, None, temperature=0.0)


def test_ids():
    import paper_2408_11850_amd as amd
    x = torch.empty((1, (1 << 32) + 5), device="cuda")
    with pytest.raises(ValueError):
        amd.sample_rows(x, None, temperature=0.0)
    with pytest.raises(ValueError):
        amd.filter_rows(x, out=x)
