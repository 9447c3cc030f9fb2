"""Clipping of values whose squares' sum is no float32, although their norm is."""
import pytest


pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


@pytest.mark.parametrize("value", [1.12e15, 2.0 ** 41, 2.0 ** 39])
def test_many_large_values(mf, value):
    """Hundreds of millions of values whose squares' sum passes 2^128, although the norm is an ordinary float32.  Equal
    values v: the norm is v sqrt(n).  Off by the square's rounding, sums of 2^5 a thread, then chunks (up to 2^9 of a
    block), lanes, warps and blocks: fewer than 1200 roundings in a row, halved by the root; the results are rounded to
    bf16 (half a step: 2^-8)."""
    import torch
    if torch.cuda.mem_get_info()[0] < 6 << 30:
        pytest.skip("less than 6 GB free")
    n = 1 << 29
    x = torch.full((n,), value, device="cuda", dtype=torch.bfloat16)
    v = float(x[0])
    norm = float(mf.clip_gradients([x], 1.0))
    want = v * n ** 0.5
    assert abs(norm / want - 1) <= 600 * 2.0 ** -24
    assert abs(float(x[0]) * n ** 0.5 - 1) <= 2.0 ** -8 + 1e-4 and bool((x == x[0]).all())
