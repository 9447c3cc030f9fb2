"""Newton-Schulz orthogonalisation on the GPU against the 64-bit reference."""
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


def _dt(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def _draw(batch, rows, cols, dtype, seed=0, kind="normal"):
    """[batch][rows][cols] on the GPU: full rank, or with singular values that fall off as 1 / i."""
    import torch
    g = torch.Generator().manual_seed(seed + rows * 7 + cols)
    if kind == "normal":
        v = torch.randn(batch, rows, cols, generator=g, dtype=torch.float64)
    else:
        k = min(rows, cols)
        v = torch.randn(batch, rows, k, generator=g, dtype=torch.float64) / torch.arange(1, k + 1) @ torch.randn(
            batch, k, cols, generator=g, dtype=torch.float64)
    return (0.01 * v).to(_dt(dtype)).cuda()


def _check(got, g, dtype, steps=5, coeffs=MUON, eps=1e-7):
    got, g = got.double().cpu().numpy(), g.double().cpu().numpy()
    for y, x in zip(got, g):
        xs = R.orthogonalize(x, steps, coeffs, eps)
        off, most = np.linalg.norm(y - xs[-1]), R.orth_bound(xs, coeffs, dtype)
        assert off <= most, (off, most, np.linalg.norm(xs[-1]))


SIZES = [(1, 1, 1), (2, 1, 7), (2, 9, 1), (3, 2, 2), (5, 64, 64), (7, 64, 12), (4, 12, 64), (2, 65, 63), (3, 128, 128), (2, 128, 20),
         (2, 100, 257), (2, 129, 130), (3, 256, 256), (1, 300, 1000), (1, 1031, 517), (1, 8, 5000), (1, 700, 640)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("size", SIZES)
def test_against_64_bits(mf, size, dtype):
    for kind in ("normal", "falling"):
        g = _draw(*size, dtype, kind=kind)
        keep = g.clone()
        out = mf.orthogonalize(g)
        _check(out, g, dtype)
        assert g.equal(keep) and out.equal(mf.orthogonalize(g))
    assert mf.check_operators() == mf.MF_OK


@pytest.mark.parametrize("steps", [0, 1, 2, 3, 7])
@pytest.mark.parametrize("coeffs", [MUON, (1.5, -0.5, 0.0), (1.875, -1.25, 0.375)])
def test_steps_and_coefficients(mf, steps, coeffs):
    for size, dtype in (((3, 40, 70), "f32"), ((2, 200, 130), "bf16"), ((1, 300, 400), "f16")):
        g = _draw(*size, dtype)
        _check(mf.orthogonalize(g, steps=steps, coeffs=coeffs), g, dtype, steps, coeffs)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [(40, 24), (24, 40), (300, 200)])
def test_layouts(mf, size, dtype):
    """Strided rows, strided batches, transposed views and a given output."""
    import torch
    b, (m, n) = 3, size
    g = _draw(b, m, n, dtype)
    want = mf.orthogonalize(g)
    _check(want, g, dtype)
    wide = torch.full((b, m, n + 13), float("nan"), dtype=g.dtype, device="cuda")
    wide[..., 5:5 + n] = g
    assert mf.orthogonalize(wide[..., 5:5 + n]).equal(want)
    apart = torch.full((2 * b, m, n), float("nan"), dtype=g.dtype, device="cuda")
    apart[::2] = g
    assert mf.orthogonalize(apart[::2]).equal(want)
    out = torch.full((b, m, n + 7), 3.0, dtype=g.dtype, device="cuda")
    assert mf.orthogonalize(g, out=out[..., 3:3 + n]).data_ptr() == out[..., 3:3 + n].data_ptr()
    assert out[..., 3:3 + n].equal(want) and (out[..., :3] == 3).all() and (out[..., 3 + n:] == 3).all()
    flip = mf.orthogonalize(g.mT)
    assert flip.shape == g.mT.shape and flip.mT.equal(want)
    _check(mf.orthogonalize(g.mT.contiguous()), g.mT, dtype)
    assert mf.orthogonalize(g.view(1, b, m, n)).equal(want.view(1, b, m, n)) and mf.orthogonalize(g[1]).equal(want[1])


def test_long_sums(mf):
    """Sums of 200,000 products: rounding to fp16 leaves at most 2^-10 / sqrt(12) = 2.8e-4 of each value (root mean
    square); what the sums add has to stay well below (here 2e-5)."""
    for size in ((1, 3, 200_000), (1, 200_000, 5)):
        g = _draw(*size, "f16")
        xs = R.orthogonalize(g[0].double().cpu().numpy(), 5, MUON, 1e-7)
        off = np.linalg.norm(mf.orthogonalize(g)[0].double().cpu().numpy() - xs[-1]) / np.linalg.norm(xs[-1])
        assert off <= 3e-4, off


def test_special_matrices(mf):
    """Zeros give zeros, NaN and infinities stay in their own matrix, scales do not matter."""
    import torch
    for size in ((5, 48, 30), (5, 260, 300)):
        g = _draw(*size, "f32")
        want = mf.orthogonalize(g)
        bad = g.clone()
        bad[1] = 0
        bad[2, 3, 4] = float("nan")
        bad[3, 5, 6] = float("inf")
        got = mf.orthogonalize(bad)
        assert got[0].equal(want[0]) and got[4].equal(want[4])
        assert not got[1].any() and got[2].isnan().all() and got[3].isnan().all()
        assert not mf.orthogonalize(bad, eps=0.0)[1].any()
        # powers of two change nothing but the exponents, up to the ends of the range
        for e in (-100, -40, 40, 110):
            assert mf.orthogonalize(g * 2.0 ** e, eps=0.0).equal(mf.orthogonalize(g, eps=0.0))
        one = torch.zeros(1, *size[1:], device="cuda")
        one[0, 2, 3] = 1e30  # rank one: every other direction stays zero
        _check(mf.orthogonalize(one), one, "f32")


@pytest.mark.parametrize("shape", [(0, 4, 5), (3, 0, 5), (3, 4, 0)])
def test_empty(mf, shape):
    import torch
    assert mf.orthogonalize(torch.zeros(shape, device="cuda")).shape == shape


def test_many_matrices(mf):
    """More matrices than a launch has blocks for, small ones: the first, the last, some between."""
    g = _draw(1, 6, 5, "f32").expand(70_000, 6, 5).contiguous()
    g[1::3] *= 2
    out = mf.orthogonalize(g)
    _check(out[:1], g[:1], "f32")
    assert out.equal(out[:1].expand_as(out)) or (out - out[:1]).abs().max() < 1e-5
    g2 = _draw(70_000, 3, 4, "bf16")
    out = mf.orthogonalize(g2)
    pick = [0, 1, 32_767, 32_768, 65_535, 65_536, 69_999]
    _check(out[pick], g2[pick], "bf16")


def test_on_other_streams(mf):
    import torch
    gs = [_draw(2, 300, 280, "bf16"), _draw(9, 64, 64, "f32")]
    want = [mf.orthogonalize(g) for g in gs]
    torch.cuda.synchronize()
    outs = []
    streams = [torch.cuda.Stream() for _ in range(3)]
    for k in range(9):
        with torch.cuda.stream(streams[k % 3]):
            outs.append([mf.orthogonalize(g) for g in gs])
    torch.cuda.synchronize()
    assert all(a.equal(b) for o in outs for a, b in zip(o, want))
    assert mf.check_operators() == mf.MF_OK


def test_in_a_graph(mf):
    import torch
    g = _draw(1, 200, 300, "bf16")
    want = mf.orthogonalize(g)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        mf.orthogonalize(g)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = mf.orthogonalize(g)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert got.equal(want)


def test_refusals(mf):
    import torch
    g = torch.zeros(2, 6, 8, device="cuda")
    bad = [lambda: mf.orthogonalize(g[0, 0]), lambda: mf.orthogonalize(g.double()), lambda: mf.orthogonalize(g[..., ::2]),
           lambda: mf.orthogonalize(g, steps=-1), lambda: mf.orthogonalize(g, steps=40), lambda: mf.orthogonalize(g, coeffs=(9.0, 0, 0)),
           lambda: mf.orthogonalize(g, coeffs=(float("nan"), 0, 0)), lambda: mf.orthogonalize(g, eps=-1.0),
           lambda: mf.orthogonalize(g, out=g[:1]), lambda: mf.orthogonalize(g, out=g.half()),
           lambda: mf.orthogonalize(torch.zeros(4, 6, 3, 8, device="cuda").transpose(1, 2)[:, :2]),
           lambda: mf.orthogonalize(g, out=torch.zeros(2, 8, 6, device="cuda").mT)]
    for call in bad:
        with pytest.raises(mf.MFError) as e:
            call()
        assert e.value.status == mf.MF_EINVAL
