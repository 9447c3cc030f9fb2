"""Linear attention on columns of very different sizes: each result is off relative to its own terms (tests/_attend_ref.py
gives bounds value by value), whatever stands beside it."""
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


def columns(d, most, seed):
    """Nine powers of two from 1 to 2^-most, mixed over the columns."""
    import torch
    e = np.random.default_rng(seed).permutation(d) % 9
    return torch.tensor(2.0 ** (-most / 8.0 * e).round(), dtype=torch.float32).cuda()


@pytest.mark.parametrize("kind,most", [("f32", 48), ("bf16", 48), ("f16", 16)])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128), (64, 128), (128, 72), (24, 24)])
@pytest.mark.parametrize("which", ["q", "k", "v", "do", "all"])
def test_columns_of_different_sizes(mf, kind, dk, dv, which, most):
    """Columns of one step 2^most apart: a column of o depends on that column of v alone, a row of the state on that
    column of k."""
    c = Case(kind, 2, 300, 2, dk, dv, marks="some")
    for i, name in enumerate(("q", "k", "v", "do")):
        if which in (name, "all"):
            x = getattr(c, name)
            x.mul_(columns(x.shape[3], most, i).to(x.dtype))
    if which != "q":
        c.state = None
        c.dlast = None
    c.check(mf)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 128)])
@pytest.mark.parametrize("decay", [-0.5, -0.3])
def test_keys_that_were_used_once(mf, kind, dk, dv, decay):
    """Keys with one column each: a row of the state holds what its key saw last, 2^-40 to 2^-90 of the others by now."""
    import torch
    c = Case(kind, 1, 125, 2, dk, dv, state=False)
    c.decay.fill_(decay)
    one = torch.zeros(125, dk, device="cuda")
    one[torch.arange(125), torch.arange(125) % dk if dk < 125 else torch.arange(125)] = 1
    c.k.mul_(one[None, :, None].to(c.k.dtype))
    c.check(mf)
    # and queries that ask for one row each
    c.q.mul_(one.flip(0)[None, :, None].to(c.q.dtype))
    c.check(mf)
