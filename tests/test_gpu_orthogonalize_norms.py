"""Orthogonalisation of matrices whose norms are at the ends of the range."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


@pytest.mark.parametrize("dtype,value", [("float32", 2.0 ** 50), ("bfloat16", 2.0 ** 50), ("float32", 3e38), ("float32", 1e-44)])
def test_sums_of_many_squares_stay_in_range(mf, dtype, value):
    """2^28 equal values (whose squares add up to 2^128 at the first), divided by their norm: 2^-14 each, to the norm's fp32 sums (2^28 terms by
    threads, warps and blocks: chains of at most some thousand additions, 2^-12 of the sum at worst)."""
    import torch
    g = torch.full((1, 1 << 14, 1 << 14), value, dtype=getattr(torch, dtype), device="cuda")
    out = mf.orthogonalize(g, steps=0, eps=0.0).float()
    assert (out * 2.0 ** 14 - 1).abs().max() <= 2.0 ** -12 + (2.0 ** -8 if dtype == "bfloat16" else 0)
