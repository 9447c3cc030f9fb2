"""The gated linear recurrence and its gradient on the GPU against the 64-bit reference."""
import numpy as np
import pytest

import _ops_ref as R

pytestmark = pytest.mark.gpu


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


def _marks(kind, b, t, r):
    if kind == "none":
        return None
    if kind == "missing":  # every step of every row
        return np.zeros((b, t), np.uint8)
    if kind == "firsts":
        return np.full((b, t), R.FIRST, np.uint8)
    m = r.choice(np.array([0, 1, 2], np.uint8), (b, t), p=[0.2, 0.75, 0.05])
    if b > 1:
        m[1] = R.MISSING  # a row with no sample at all
    return m


def _draw(shape, dtype, marks, seed, zshift=0.0):
    """Inputs on the GPU and what they hold as float64; missing places hold NaN."""
    import torch
    r = np.random.default_rng(seed)
    b, t, d = shape
    m = _marks(marks, b, t, r)
    gpu = {}
    for k, v in (("x", r.standard_normal(shape)), ("z", 2 * r.standard_normal(shape) + zshift + 3 * r.random(d)),
                 ("dh", r.standard_normal(shape))):
        gpu[k] = torch.tensor(v).to(_dt(dtype)).cuda()
    if m is not None:
        gap = torch.tensor(m == R.MISSING).cuda()[..., None]
        gpu["x"].masked_fill_(gap, float("nan"))
        gpu["z"].masked_fill_(gap, float("inf"))
    for k in ("h0", "dlast"):
        gpu[k] = torch.tensor(r.standard_normal((b, d)), dtype=torch.float32).cuda()
    gpu["marks"] = None if m is None else torch.tensor(m).cuda()
    host = {k: None if v is None else v.double().cpu().numpy() for k, v in gpu.items() if k != "marks"}
    return gpu, host, m


def _near(got, want, bound, dtype):
    """|got - want| within the bound and the rounding to the type (and to its smallest numbers)."""
    got = got.double().cpu().numpy()
    u = R.TYPE_U[dtype] if dtype != "f32" else 0.0
    tiny = 2.0 ** -24 if dtype == "f16" else 2.0 ** -125
    off = np.abs(got - want) - (bound + u * (np.abs(want) + bound) + tiny)
    assert np.isfinite(got).all() and (off.size == 0 or off.max() <= 0), float(off.max())


def _check(mf, shape, dtype, marks, seed=1, h0=True, dlast=True, zshift=0.0):
    gpu, host, m = _draw(shape, dtype, marks, seed, zshift)
    h0g, h0h = (gpu["h0"], host["h0"]) if h0 else (None, None)
    dlg, dlh = (gpu["dlast"], host["dlast"]) if dlast else (None, None)
    h, last, saved = mf.recurrence(gpu["x"], gpu["z"], h0g, gpu["marks"], save=True)
    dx, dz, dh0 = mf.recurrence_backward(gpu["dh"], gpu["x"], gpu["z"], saved, dlg, gpu["marks"])
    wh, wlast = R.recurrence(host["x"], host["z"], h0h, m)
    wx, wz, w0 = R.recurrence_grad(host["x"], host["z"], h0h, m, host["dh"], dlh)
    eh, ex, ez, e0 = R.recurrence_bounds(host["x"], host["z"], h0h, m, host["dh"], dlh)
    _near(h, wh, eh, dtype)
    _near(last, wlast, eh[:, -1] if shape[1] else 0.0, "f32")
    _near(dx, wx, ex, dtype)
    _near(dz, wz, ez, dtype)
    _near(dh0, w0, e0, "f32")
    if m is not None:
        gone = (m == R.MISSING)
        assert not dx.float().cpu().numpy()[gone].any()
        assert not dz.float().cpu().numpy()[gone].any()
    h2, last2 = mf.recurrence(gpu["x"], gpu["z"], h0g, gpu["marks"])
    assert h2.equal(h) and last2.equal(last)  # the same bits, with or without what the gradient needs
    assert mf.check_operators() == mf.MF_OK


SHAPES = [(1, 1, 1), (16, 1, 8), (2, 3, 5), (1, 16, 8), (3, 17, 33), (2, 129, 64), (4, 1000, 7), (1, 4097, 130), (64, 300, 48),
          (5, 70, 1000), (2, 9000, 3), (3, 2047, 250)]


@pytest.mark.parametrize("marks", ["none", "mixed"])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_64_bits(mf, shape, dtype, marks):
    _check(mf, shape, dtype, marks, seed=sum(shape))


@pytest.mark.parametrize("marks", ["missing", "firsts"])
@pytest.mark.parametrize("shape", [(2, 1, 4), (2, 100, 40), (1, 3000, 8)])
def test_uniform_marks(mf, shape, marks):
    _check(mf, shape, "f32", marks)
    _check(mf, shape, "bf16", marks)


@pytest.mark.parametrize("h0,dlast", [(False, True), (True, False), (False, False)])
def test_without_states(mf, h0, dlast):
    _check(mf, (3, 70, 24), "f32", "mixed", h0=h0, dlast=dlast)
    _check(mf, (1, 5000, 16), "bf16", "none", h0=h0, dlast=dlast)


def test_long_memories(mf):
    _check(mf, (2, 6000, 10), "f32", "none", zshift=6.0)


@pytest.mark.parametrize("shape", [(0, 5, 4), (3, 0, 4), (3, 5, 0)])
def test_empty(mf, shape):
    import torch
    x = torch.zeros(shape, device="cuda")
    h0 = torch.randn(shape[0], shape[2], device="cuda")
    h, last, saved = mf.recurrence(x, x, h0, save=True)
    assert h.shape == shape and (shape[1] and not last.numel() or last.equal(h0))
    dx, dz, dh0 = mf.recurrence_backward(x, x, x, saved, h0)
    assert dx.shape == dz.shape == shape and (shape[1] and not dh0.numel() or dh0.equal(h0))
    assert mf.recurrence(x, x)[1].abs().sum() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["time_major", "slice", "odd_offset", "broadcast_z", "batch_stride"])
def test_strides(mf, dtype, how):
    """The same values in other layouts give the same bits."""
    import torch
    b, t, d = 3, 333, 40
    gpu, _, _ = _draw((b, t, d), dtype, "mixed", 9)
    if how == "broadcast_z":
        gpu["z"] = gpu["z"][:1, :1].nan_to_num(posinf=0.5).expand(b, t, d)
    want = mf.recurrence(gpu["x"], gpu["z"].contiguous(), gpu["h0"], gpu["marks"], save=True)
    wgrad = mf.recurrence_backward(gpu["dh"], gpu["x"], gpu["z"].contiguous(), want[2], gpu["dlast"], gpu["marks"])

    def other(v):
        if how == "time_major":
            return v.transpose(0, 1).contiguous().transpose(0, 1)
        if how == "slice":
            big = torch.full((b, t, d + 24), float("nan"), dtype=v.dtype, device="cuda")
            big[..., 8:8 + d] = v
            return big[..., 8:8 + d]
        if how == "odd_offset":
            big = torch.full((b, t, d + 3), float("nan"), dtype=v.dtype, device="cuda")
            big[..., 1:1 + d] = v
            return big[..., 1:1 + d]
        if how == "batch_stride":
            big = torch.full((b, t + 2, d), float("nan"), dtype=v.dtype, device="cuda")
            big[:, 1:-1] = v
            return big[:, 1:-1]
        return v
    marks = gpu["marks"]
    if how == "time_major":
        marks = marks.t().contiguous().t()
    if how == "odd_offset":
        marks = torch.cat((marks, marks), 1)[:, :t]
    x, dh, z = other(gpu["x"]), other(gpu["dh"]), gpu["z"] if how == "broadcast_z" else other(gpu["z"])
    got = mf.recurrence(x, z, gpu["h0"], marks, save=True)
    ggrad = mf.recurrence_backward(dh, x, z, got[2], gpu["dlast"], marks)
    for p, q in zip((*want, *wgrad), (*got, *ggrad)):
        assert p.equal(q)


@pytest.mark.parametrize("shape", [(1, 50, 8), (1, 40000, 8)])
def test_infinities_and_nan_stay_where_they_are(mf, shape):
    """A NaN reaches what follows it in its own channel, up to the next trace, and nothing else."""
    import torch
    b, t, d = shape
    x = torch.randn(shape, device="cuda")
    z = torch.full(shape, 1.0, device="cuda")
    marks = torch.ones(b, t, dtype=torch.uint8, device="cuda")
    cut = 3 * t // 5
    marks[:, cut] = mf.MARK_FIRST
    clean = mf.recurrence(x, z, None, marks, save=True)
    dh = torch.randn(shape, device="cuda")
    gclean = mf.recurrence_backward(dh, x, z, clean[2], None, marks)
    bad = x.clone()
    bad[0, 5, 2], bad[0, 7, 4] = float("nan"), float("inf")
    h, last, saved = mf.recurrence(bad, z, None, marks, save=True)
    assert last.equal(clean[1]) and h[:, cut:].equal(clean[0][:, cut:]) and h[:, :5].equal(clean[0][:, :5])
    keep = [c for c in range(d) if c not in (2, 4)]
    assert h[..., keep].equal(clean[0][..., keep])
    assert h[0, 5:cut, 2].isnan().all() and (h[0, 7:cut, 4] == float("inf")).all()
    dx, dz, dh0 = mf.recurrence_backward(dh, bad, z, saved, None, marks)
    assert dx.equal(gclean[0]) and dh0.equal(gclean[2])
    assert dz[..., keep].equal(gclean[1][..., keep]) and dz[:, cut:].equal(gclean[1][:, cut:])
    # and a NaN gradient reaches what lies before it, back to the start of its trace
    bad = dh.clone()
    bad[0, t - 3, 1] = float("nan")
    dx, dz, dh0 = mf.recurrence_backward(bad, x, z, clean[2], None, marks)
    keep = [c for c in range(d) if c != 1]
    assert dx[0, cut:t - 2, 1].isnan().all() and dx[:, :cut].equal(gclean[0][:, :cut]) and dh0.equal(gclean[2])
    assert dx[..., keep].equal(gclean[0][..., keep])


def test_extreme_gates(mf):
    """Gates at the ends of the range: kept whole, replaced whole, no NaN."""
    import torch
    big = torch.finfo(torch.float32).max
    z = torch.tensor([-float("inf"), -big, -200.0, -100.0, 100.0, 200.0, big, float("inf")], device="cuda").view(1, 1, 8)
    x = torch.full((1, 40, 8), 2.0, device="cuda")
    h0 = torch.full((1, 8), 5.0, device="cuda")
    h, last, saved = mf.recurrence(x, z.expand(1, 40, 8), h0, save=True)
    assert (h[..., :4] == 2).all() and (h[..., 4:] == 5).all()
    dx, dz, dh0 = mf.recurrence_backward(torch.ones_like(x), x, z.expand(1, 40, 8), saved)
    assert (dx[..., :4] == 1).all() and dz.isfinite().all() and dx.isfinite().all()
    assert (dh0[..., 4:] == 40).all() and (dh0[..., :4].abs() < 1e-30).all()


def test_the_gradient_is_that_of_differences(mf):
    """Along random directions: the GPU's gradient against central differences of the 64-bit definition."""
    gpu, host, m = _draw((2, 400, 6), "f32", "mixed", 21)
    h, last, saved = mf.recurrence(gpu["x"], gpu["z"], gpu["h0"], gpu["marks"], save=True)
    grads = [g.double().cpu().numpy() for g in
             mf.recurrence_backward(gpu["dh"], gpu["x"], gpu["z"], saved, gpu["dlast"], gpu["marks"])]
    r = np.random.default_rng(5)
    args = [np.where((m == 0)[..., None], 0.0, host["x"]), np.where((m == 0)[..., None], 0.0, host["z"]), host["h0"]]

    def loss(a):
        h, s = R.recurrence(*a, m)
        return (h * host["dh"]).sum() + (s * host["dlast"]).sum()
    _, ex, ez, e0 = R.recurrence_bounds(args[0], args[1], args[2], m, host["dh"], host["dlast"])
    for k in range(3):
        v = r.standard_normal(args[k].shape)
        eps = 1e-5
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + eps * v, args[k] - eps * v
        # truncation eps^2 |v|^3 times a third derivative of order 1 at 4800 places, rounding 1e-13 / eps
        tol = (np.abs(v) * (ex, ez, e0)[k]).sum() + 1e-6 + 1e-8
        assert abs((loss(up) - loss(down)) / (2 * eps) - (grads[k] * v).sum()) < tol


def test_on_another_stream_and_repeated(mf):
    import torch
    gpu, _, _ = _draw((2, 9000, 24), "bf16", "mixed", 4)
    torch.cuda.synchronize()
    want = mf.recurrence(gpu["x"], gpu["z"], gpu["h0"], gpu["marks"], save=True)
    wg = mf.recurrence_backward(gpu["dh"], gpu["x"], gpu["z"], want[2], gpu["dlast"], gpu["marks"])
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(3)], []
    for k in range(6):
        with torch.cuda.stream(streams[k % 3]):
            f = mf.recurrence(gpu["x"], gpu["z"], gpu["h0"], gpu["marks"], save=True)
            outs.append((*f, *mf.recurrence_backward(gpu["dh"], gpu["x"], gpu["z"], f[2], gpu["dlast"], gpu["marks"])))
    torch.cuda.synchronize()
    for o in outs:
        assert all(p.equal(q) for p, q in zip(o, (*want, *wg)))
    assert mf.check_operators() == mf.MF_OK


def test_in_a_graph(mf):
    import torch
    gpu, _, _ = _draw((1, 20000, 24), "f32", "none", 6)
    want = mf.recurrence(gpu["x"], gpu["z"], gpu["h0"])
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        mf.recurrence(gpu["x"], gpu["z"], gpu["h0"])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = mf.recurrence(gpu["x"], gpu["z"], gpu["h0"])
    for _ in range(3):
        got[0].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert got[0].equal(want[0]) and got[1].equal(want[1])


def test_offsets_past_32_bits(mf):
    """2.2e9 elements a tensor; gates of about 1/2, so that a state holds its last 64 samples."""
    import torch
    t, d = 1_075_000, 2048
    x = torch.empty(1, t, d, dtype=torch.bfloat16, device="cuda").normal_()
    z = torch.empty(1, t, d, dtype=torch.bfloat16, device="cuda").normal_(std=0.1)
    h, last, saved = mf.recurrence(x, z, save=True)
    for lo in (0, 1_048_576 - 100, t - 300):
        cut = [v[:, lo:lo + 300].double().cpu().numpy() for v in (x, z)]
        want, _ = R.recurrence(*cut, None, None)
        skip = 0 if lo == 0 else 100  # (the state before the cut decays below 2^-60)
        _near(h[:, lo + skip:lo + 300], want[:, skip:], 1e-5, "bf16")
    dx, dz, _ = mf.recurrence_backward(h, x, z, saved)
    lo = t - 300
    cut = [v[:, lo:].double().cpu().numpy() for v in (x, z, h)]
    before, _ = R.recurrence(*[v[:, lo - 100:lo].double().cpu().numpy() for v in (x, z)], None, None)
    wx, wz, _ = R.recurrence_grad(cut[0], cut[1], before[:, -1], None, cut[2], None)
    _near(dx[:, lo:], wx, 1e-5, "bf16")
    _near(dz[:, lo:], wz, 1e-5, "bf16")
    del h, dx, dz, x, z, saved
    torch.cuda.empty_cache()


def test_refusals(mf):
    import torch
    x = torch.zeros(2, 6, 4, device="cuda")
    s = torch.zeros(2, 4, device="cuda")
    bad = [lambda: mf.recurrence(x[0], x[0]), lambda: mf.recurrence(x.double(), x.double()), lambda: mf.recurrence(x, x.half()),
           lambda: mf.recurrence(x, x[:, :5]), lambda: mf.recurrence(x.transpose(1, 2), x.transpose(1, 2)),
           lambda: mf.recurrence(x, x.cpu()), lambda: mf.recurrence(x, x, s.half()), lambda: mf.recurrence(x, x, s[:1]),
           lambda: mf.recurrence(x, x, s, torch.ones(2, 6, device="cuda")),
           lambda: mf.recurrence(x, x, s, torch.ones(2, 5, dtype=torch.uint8, device="cuda")),
           lambda: mf.recurrence_backward(x, x, x, s), lambda: mf.recurrence_backward(x, x, x, None),
           lambda: mf.recurrence_backward(x[:1], x, x, mf.recurrence(x, x, save=True)[2])]
    for call in bad:
        with pytest.raises(mf.MFError) as e:
            call()
        assert e.value.status == mf.MF_EINVAL
