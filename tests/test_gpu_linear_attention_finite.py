"""Linear attention beside values that are not finite: the rest keeps its bounds."""
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


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(16, 24), (64, 128), (128, 128)])
@pytest.mark.parametrize("where", ["q", "k", "v", "do"])
def test_finite_results_beside_a_value_that_is_not(mf, kind, dk, dv, where):
    """What does not depend on a NaN keeps its bounds: compared with the exact results of the inputs without it."""
    import _attend_ref as A
    import torch
    t, at = 400, 150
    c = Case(kind, 1, t, 2, dk, dv)
    c.decay.fill_(-0.01)
    c.marks = torch.ones(1, t, dtype=torch.uint8, device="cuda")
    c.marks[0, 200] = 2
    host, d = c.host(), lambda x: x.double().cpu().numpy()
    want = (*A.attend(*host)[:2], *A.attend_grad(d(c.do), d(c.dlast), *host))
    bounds = (*A.attend_bounds(kind, None, None, *host), *A.attend_bounds(kind, d(c.do), d(c.dlast), *host))
    getattr(c, where)[0, at, 1, 5] = float("nan")
    o, last, saved = mf.linear_attention(c.q, c.k, c.v, c.decay, c.state, c.marks, c.scale, save=True)
    got = (o, last, *mf.linear_attention_backward(c.do, c.q, c.k, c.v, c.decay, saved, c.dlast, c.marks, c.scale))
    for name, x, exact, bound in zip(("o", "last", "dq", "dk", "dv", "dstate"), map(d, got), want, bounds):
        finite = np.isfinite(x)
        assert finite[0, :, 0].all() if x.ndim == 4 and name not in ("last", "dstate") else finite[0, 0].all(), name
        assert (np.abs(x - exact)[finite] <= bound[finite]).all(), name
        assert finite.mean() > 0.4, name
