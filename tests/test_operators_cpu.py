"""The training operators without a GPU: their formulas against differences, and what the C ABI refuses."""
import ctypes as C

import numpy as np
import pytest

import _ops_ref as R


@pytest.fixture(scope="module")
def mf():
    from paper_2609_02109_gb300 import build
    build.build()
    from paper_2609_02109_gb300 import mf as mod
    return mod


@pytest.mark.parametrize("with_marks", [False, True])
def test_the_recurrence_gradient_is_that_of_differences(with_marks):
    r = np.random.default_rng(3)
    b, t, d = 2, 23, 3
    x, z, dh = (r.standard_normal((b, t, d)) for _ in range(3))
    h0, dlast = r.standard_normal((b, d)), r.standard_normal((b, d))
    marks = r.integers(0, 3, (b, t)).astype(np.uint8) if with_marks else None
    loss = lambda x, z, h0: (lambda h, s: (h * dh).sum() + (s * dlast).sum())(*R.recurrence(x, z, h0, marks))  # noqa: E731
    got = R.recurrence_grad(x, z, h0, marks, dh, dlast)
    eps = 1e-5  # central differences: about eps^2 = 1e-10 of truncation, 1e-16 / eps = 1e-11 of rounding, sums of 100
    for k, grad in enumerate(got):
        args = [x, z, h0]
        for _ in range(12):
            at = tuple(r.integers(0, n) for n in args[k].shape)
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[k][at] += eps
            down[k][at] -= eps
            assert abs((loss(*up) - loss(*down)) / (2 * eps) - grad[at]) < 1e-7


def test_five_steps_bring_singular_values_near_one():
    r = np.random.default_rng(4)
    g = r.standard_normal((24, 40))
    x = R.orthogonalize(g, 5, (3.4445, -4.7750, 2.0315), 1e-7)[-1]
    s = np.linalg.svd(x, compute_uv=False)
    assert s.max() < 1.25 and s.min() > 0.3
    u, sv, vt = np.linalg.svd(g / (np.linalg.norm(g) + 1e-7), full_matrices=False)
    for _ in range(5):
        sv = 3.4445 * sv - 4.7750 * sv ** 3 + 2.0315 * sv ** 5
    assert np.abs(u @ np.diag(sv) @ vt - x).max() < 1e-9
    assert np.abs(R.orthogonalize(g.T, 5, (3.4445, -4.7750, 2.0315), 1e-7)[-1] - x.T).max() < 1e-12


# -- what the C ABI refuses, before anything runs ---------------------------------------------
P = 0x10000  # an address that is never read


def _recur(mf, cls, **over):
    b, t, d = over.get("batch", 2), over.get("time", 5), over.get("dim", 4)
    seq = lambda: mf._Seq(P, 5 * 4, 4)  # noqa: E731
    kw = dict(type=0, batch=b, time=t, dim=d, x=seq(), z=seq(), d_marks=None, marks_stride_batch=0, marks_stride_time=0,
              d_status=None)
    kw.update(dict(d_h0=None, h=seq(), d_last=None, d_saved=None) if cls is mf._Recurrence else
              dict(d_saved=P, dh=seq(), d_dlast=None, dx=seq(), dz=seq(), d_dh0=None))
    kw.update(over)
    return cls(**kw)


RECUR_BAD = [dict(type=3), dict(type=-1), dict(batch=-1), dict(time=-1), dict(dim=-4), dict(time=1 << 31),
             dict(batch=1 << 30, dim=1 << 30), dict(x=(None, 20, 4)), dict(z=(None, 20, 4)), dict(x=(P + 2, 20, 4)),
             dict(x=(P, -20, 4)), dict(z=(P, 20, 1 << 62)), dict(d_marks=P, marks_stride_time=-1)]


@pytest.mark.parametrize("over", RECUR_BAD + [dict(h=(None, 20, 4)), dict(h=(P, 0, 4)), dict(h=(P, 20, 3)), dict(h=(P, 12, 4)),
                                              dict(d_h0=P + 1), dict(d_saved=P + 2), dict(d_status=P + 1)])
def test_forward_refuses(mf, over):
    over = {k: mf._Seq(*v) if isinstance(v, tuple) else v for k, v in over.items()}
    p = _recur(mf, mf._Recurrence, **over)
    assert mf.lib().mf_recurrence_forward(C.byref(p), None, 0, None) == mf.MF_EINVAL
    assert mf.lib().mf_last_error().startswith(b"mf_recurrence_forward: ")


@pytest.mark.parametrize("over", RECUR_BAD + [dict(dh=(None, 20, 4)), dict(dx=(P, 0, 4)), dict(dz=(P, 20, 2)), dict(dx=(P + 1, 20, 4)),
                                              dict(d_saved=None), dict(d_dlast=P + 1), dict(d_dh0=P + 3)])
def test_backward_refuses(mf, over):
    over = {k: mf._Seq(*v) if isinstance(v, tuple) else v for k, v in over.items()}
    p = _recur(mf, mf._RecurrenceGrad, **over)
    assert mf.lib().mf_recurrence_backward(C.byref(p), None, 0, None) == mf.MF_EINVAL
    assert mf.lib().mf_last_error().startswith(b"mf_recurrence_backward: ")


def _orth(mf, **over):
    kw = dict(type=0, batch=2, rows=4, cols=6, d_g=P, g_stride_batch=24, g_stride_row=6, d_out=2 * P, out_stride_batch=24,
              out_stride_row=6, steps=5, a=3.4445, b=-4.775, c=2.0315, eps=1e-7, d_status=None)
    kw.update(over)
    return mf._Orthogonalize(**kw)


@pytest.mark.parametrize("over", [
    dict(type=5), dict(batch=-1), dict(rows=-2), dict(cols=(1 << 20) + 1), dict(steps=-1), dict(steps=33), dict(a=float("nan")),
    dict(b=float("inf")), dict(eps=-1.0), dict(eps=float("nan")), dict(a=9.0), dict(c=50.0), dict(d_g=None), dict(d_out=None),
    dict(d_g=P + 2), dict(type=1, d_out=P + 1), dict(g_stride_row=-6), dict(out_stride_row=5), dict(out_stride_batch=23),
    dict(out_stride_batch=0), dict(d_status=P + 2)])
def test_orthogonalize_refuses(mf, over):
    p = _orth(mf, **over)
    n = C.c_uint64()
    st = mf.lib().mf_orthogonalize_workspace(C.byref(p), C.byref(n))
    assert st in (mf.MF_OK, mf.MF_EINVAL)
    assert mf.lib().mf_orthogonalize(C.byref(p), P, 1 << 40, None) == mf.MF_EINVAL
    assert mf.lib().mf_last_error().startswith(b"mf_orthogonalize: ")


def test_null_arguments(mf):
    lib = mf.lib()
    assert lib.mf_recurrence_forward(None, None, 0, None) == mf.MF_EINVAL
    assert lib.mf_recurrence_backward(None, None, 0, None) == mf.MF_EINVAL
    assert lib.mf_orthogonalize(None, None, 0, None) == mf.MF_EINVAL
    assert lib.mf_orthogonalize_workspace(None, None) == mf.MF_EINVAL


def test_empty_sizes_are_not_errors(mf):
    lib = mf.lib()
    for over in (dict(batch=0), dict(dim=0)):
        p = _recur(mf, mf._Recurrence, **over)
        assert lib.mf_recurrence_forward(C.byref(p), None, 0, None) == mf.MF_OK
        p = _recur(mf, mf._RecurrenceGrad, **over)
        assert lib.mf_recurrence_backward(C.byref(p), None, 0, None) == mf.MF_OK
    for over in (dict(batch=0), dict(rows=0), dict(cols=0)):
        p = _orth(mf, **over)
        n = C.c_uint64(7)
        assert lib.mf_orthogonalize_workspace(C.byref(p), C.byref(n)) == mf.MF_OK and n.value == 0
        assert lib.mf_orthogonalize(C.byref(p), None, 0, None) == mf.MF_OK


def test_the_binding_refuses_what_is_not_on_a_gpu(mf):
    import torch
    x = torch.zeros(1, 2, 3)
    for call in (lambda: mf.recurrence(x, x), lambda: mf.orthogonalize(x), lambda: mf.recurrence_backward(x, x, x, x[0, 0])):
        with pytest.raises(mf.MFError) as e:
            call()
        assert e.value.status == mf.MF_EINVAL
