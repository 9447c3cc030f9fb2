"""Clipping of as many tensors as fill launches exactly, with empty ones before, between and behind."""
import pytest

from test_gpu_clip import check, tensors

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


@pytest.mark.parametrize("sizes", [[1] * 1000 + [0], [700] * 2000 + [0, 0], [0] * 3 + [600] * 1000 + [0], [0] * 1000 + [600] * 1000,
                                   [600] * 999 + [0] * 5 + [700, 0, 0], [600] * 1000 + [0] * 1001 + [5]])
@pytest.mark.parametrize("apart", [False, True])
def test_empty_tensors_around_full_launches(mf, sizes, apart):
    check(mf, tensors(sizes, "fb"), 0.5, apart=apart)
