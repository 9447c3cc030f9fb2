"""Gradients of missing samples are zeros, whatever the rest of a trace holds."""
import numpy as np
import pytest

from test_gpu_linear_attention import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(8, 8), (16, 24), (48, 40), (64, 128), (128, 128)])
@pytest.mark.parametrize("where", ["dlast", "q", "do", "v"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_zeros_beside_what_is_not_finite(mf, kind, dk, dv, where, value):
    import torch
    t = 300
    c = Case(kind, 2, t, 2, dk, dv, state=True)
    c.decay.fill_(-0.01)
    c.marks = torch.ones(2, t, dtype=torch.uint8, device="cuda")
    gone = [0, 3, 31, 32, 100, 127, 128, 250, 299]
    c.marks[:, gone] = 0
    c.k[:, gone] = float("nan")
    c.v[:, gone] = float("inf")
    if where == "dlast":
        c.dlast[1, :, dk // 2, dv // 3] = value
    else:
        getattr(c, where)[1, 260, 1, 5] = value
    o, last, saved = mf.linear_attention(c.q, c.k, c.v, c.decay, c.state, c.marks, c.scale, save=True)
    dq, dkey, dvalue, dstate = mf.linear_attention_backward(c.do, c.q, c.k, c.v, c.decay, saved, c.dlast, c.marks, c.scale)
    for name, x in (("dk", dkey), ("dv", dvalue)):
        assert not x[:, gone].any(), name
        live = np.setdiff1d(np.arange(t), gone)
        assert bool(torch.isfinite(x[0]).all()) and bool(x[0][live].any())
    if where != "v":
        assert torch.isfinite(o[0]).all() and not torch.isfinite(dkey[1, :260]).all()
