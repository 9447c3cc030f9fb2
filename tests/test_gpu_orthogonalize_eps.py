"""Orthogonalisation of matrices whose norms are far below eps."""
import numpy as np
import pytest

import _ops_ref as R

pytestmark = pytest.mark.gpu
MUON = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


def _relative(mf, g, eps, dtype, steps=5):
    got = mf.orthogonalize(g, steps=steps, eps=eps).double().cpu().numpy()
    off = []
    for y, x in zip(got, g.double().cpu().numpy()):
        want = R.orthogonalize(x, steps, MUON, eps)[-1]
        off.append(np.linalg.norm(y - want) / np.linalg.norm(want))
    return max(off)


# All steps in one block, tiles of one SM, pairs of SMs (16 x 512 x 512).
@pytest.mark.parametrize("shape", [(3, 48, 30), (3, 64, 64), (2, 256, 256), (2, 300, 200), (16, 512, 512)])
@pytest.mark.parametrize("dtype,eps,least", [("float32", 1e-7, -30), ("float32", 1.0, -20), ("bfloat16", 1e-7, -30)])
def test_norms_far_below_eps(mf, shape, dtype, eps, least):
    """X = g / (|g| + eps) is then small, and the steps scale it up by a at a time: as precise as for any other norm.  fp32:
    operands of 22 bits, so each step leaves about 2^-22 of X a product and 2^-23 an fp16 pair: below 1e-5 in five steps.
    bf16: the result's rounding, 2^-9 at most and 2^-9 / sqrt(3) as a root mean square, and as much again for 11-bit operands."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    g = torch.randn(shape, device="cuda", generator=gen)
    g /= torch.linalg.matrix_norm(g, keepdim=True)
    most = 1e-5 if dtype == "float32" else 4e-3
    for e in range(0, least - 1, -3):
        off = _relative(mf, (g * 10.0 ** e).to(getattr(torch, dtype)), eps, dtype)
        assert off <= most, (e, off)


def test_norms_of_a_batch_side_by_side(mf):
    """Each matrix has a scale of its own, and one far above eps gives the bits that it gives alone."""
    import torch
    for shape in ((5, 40, 60), (5, 200, 300)):
        g = torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
        g[1] *= 1e-12
        g[3] *= 1e-20
        assert _relative(mf, g, 1e-7, "float32") <= 1e-5
        out = mf.orthogonalize(g)
        for i in range(5):
            assert mf.orthogonalize(g[i:i + 1]).equal(out[i:i + 1])
