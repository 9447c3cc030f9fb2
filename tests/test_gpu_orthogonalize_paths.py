"""Orthogonalisation on every path, held to limits that operands or sums with fewer bits would not pass."""
import numpy as np
import pytest

import _orth_limits as L
import _ops_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


def _draw(shape, dtype, kind="normal", seed=0):
    import torch
    r = np.random.default_rng([seed, *shape])
    b, m, n = shape
    v = r.standard_normal(shape)
    if kind == "falling":
        k = min(m, n)
        v = np.stack([r.standard_normal((m, k)) / np.arange(1, k + 1) @ r.standard_normal((k, n)) for _ in range(b)])
    return torch.tensor(0.01 * v).to({"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]).cuda()


def _check(mf, g, dtype, steps=5, some=None, coeffs=L.MUON):
    got = mf.orthogonalize(g, steps=steps, coeffs=coeffs)
    for i in range(g.shape[0]) if some is None else some:
        exact, most = L.limit(g[i].double().cpu().numpy(), dtype, steps, coeffs)
        off = L.off(got[i].double().cpu().numpy(), exact)
        assert off <= most, (i, off, most)
    assert got.equal(mf.orthogonalize(g, steps=steps, coeffs=coeffs))  # equal calls, equal bits
    assert mf.check_operators() == mf.MF_OK
    return got


# All steps in one block; tiles of 128 x 64 and 128 x 128 on one SM, with the depth split over clusters of 2 and 4 and without;
# 256 x 256 on pairs of SMs, in one round and in several; each result written as it is and transposed.
SIZES = [(2, 64, 64), (3, 64, 12), (1, 128, 500), (2, 129, 600), (2, 600, 129), (40, 520, 40), (3, 517, 1031), (5, 300, 700), (5, 700, 300),
         (16, 512, 512), (6, 1024, 520), (1, 1200, 2048), (1, 1600, 1700), (1, 1700, 1600), (3, 1700, 1600)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", SIZES)
def test_five_steps(mf, size, dtype):
    _check(mf, _draw(size, dtype), dtype, some=sorted({0, size[0] // 2, size[0] - 1}))
    if size[1] * size[2] <= 600_000:
        _check(mf, _draw(size, dtype, "falling"), dtype, some=[size[0] - 1])


@pytest.mark.parametrize("size", [(3, 64, 64), (2, 129, 600), (3, 517, 1031), (16, 512, 512), (1, 1700, 1600)])
@pytest.mark.parametrize("steps", [1, 2])
def test_few_steps(mf, size, steps):
    for dtype in ("f32", "bf16"):
        _check(mf, _draw(size, dtype), dtype, steps, some=[0, size[0] - 1])


def test_pairs_on_strided_views(mf):
    """Transposed, shifted and strided inputs and outputs of the pairs' path: the same bits, nothing beside the result written."""
    import torch
    g = _draw((16, 512, 520), "bf16")
    want = mf.orthogonalize(g)
    assert mf.orthogonalize(g.mT).mT.equal(want)
    wide = torch.full((16, 512, 533), float("nan"), dtype=g.dtype, device="cuda")
    wide[..., 5:525] = g
    out = torch.full((16, 512, 527), 3.0, dtype=g.dtype, device="cuda")
    mf.orthogonalize(wide[..., 5:525], out=out[..., 3:523])
    assert out[..., 3:523].equal(want) and (out[..., :3] == 3).all() and (out[..., 523:] == 3).all()


def test_zeros_and_nan_on_pairs(mf):
    for dtype in ("f32", "bf16"):
        g = _draw((16, 512, 512), dtype)
        want = mf.orthogonalize(g)
        bad = g.clone()
        bad[3] = 0
        bad[7, 300, 400] = float("nan")
        bad[8, 1, 511] = float("inf")
        got = mf.orthogonalize(bad)
        assert not got[3].any() and got[7].isnan().all() and got[8].isnan().all()
        keep = [i for i in range(16) if i not in (3, 7, 8)]
        assert got[keep].equal(want[keep])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_batch_in_parts(mf, dtype):
    """More matrices than a call works on at a time (16384): each part gives the bits that it gives by itself.  (Rows whose
    norm lies in one value: what that one rounds to decides the error, so no limit that averages over values holds.)"""
    g = _draw((16500, 1, 520), dtype)
    g[:, 0, 0] = 0.5
    got = mf.orthogonalize(g)
    assert got[:16384].equal(mf.orthogonalize(g[:16384])) and got[16384:].equal(mf.orthogonalize(g[16384:]))
    for i in (0, 16383, 16384, 16385, 16499):
        xs = R.orthogonalize(g[i].double().cpu().numpy(), 5, L.MUON, 1e-7)
        assert np.linalg.norm(got[i].double().cpu().numpy() - xs[-1]) <= R.orth_bound(xs, L.MUON, dtype)


@pytest.mark.parametrize("size", [(1, 4, 16384), (1, 16384, 4), (1, 200, 16384)])
def test_long_sums_of_one_sign_lose_no_more(mf, size):
    """One step of X X^T X on positive values, so that every addition to a sum of 16384 products truncates the same way.  Sums
    that leave every 256 of depth take 48 additions of up to 2^-24 of a part, half of it on average, 64 additions in
    registers round by up to 2^-25 (1.9e-6 if all went one way), and five 22-bit operands leave 2^-23 each: 4e-6 with the
    short sum of the other product.  In one accumulator 3072 truncations would leave 5e-5 and more."""
    import torch
    g = torch.rand(size, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) + 0.5
    exact = R.orthogonalize(g[0].double().cpu().numpy(), 1, (0.0, 1.0, 0.0), 1e-7)[-1]
    assert L.off(mf.orthogonalize(g, steps=1, coeffs=(0.0, 1.0, 0.0))[0].double().cpu().numpy(), exact) <= 4e-6
