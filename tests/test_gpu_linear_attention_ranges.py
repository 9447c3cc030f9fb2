"""Linear attention on values near the ends of float32, whose products are ordinary."""
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


@pytest.mark.parametrize("kind,dk,dv,t", [("f32", 16, 16, 200), ("f32", 40, 72, 100), ("bf16", 24, 20, 200), ("bf16", 32, 8, 70),
                                          ("bf16", 128, 128, 12)])
@pytest.mark.parametrize("large,small", [("v", "k"), ("k", "v"), ("q", "k"), ("k", "q"), ("do", "v"), ("q", "do")])
@pytest.mark.parametrize("decay", [-0.86, -0.05, 0.05])
def test_products_of_large_and_small_values(mf, kind, dk, dv, t, large, small, decay):
    """1e33 and 1e-20: products that are ordinary, of factors near the type's ends."""
    c = Case(kind, 1, t, 2, dk, dv, state=False, marks="some")
    c.decay.fill_(decay)
    for name, by in ((large, 1e33), (small, 1e-20)):
        getattr(c, name).mul_(by)
    for name in {"q", "k", "v", "do"} - {large, small}:
        getattr(c, name).mul_(1e-6)
    c.check(mf)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(16, 16), (64, 64)])
@pytest.mark.parametrize("size", [1e36, 1e-30])
def test_a_large_or_small_state_that_decays(mf, kind, dk, dv, size):
    c = Case(kind, 1, 60, 2, dk, dv, marks="some")
    c.decay.fill_(-0.8)
    c.state.mul_(size)
    c.q.mul_(0.0 if kind == "f16" else 1e-3)
    c.do.mul_(0.0 if kind == "f16" else 1e-3)
    c.check(mf)


@pytest.mark.parametrize("kind,dk,dv", [("f32", 16, 16), ("f32", 64, 40), ("f32", 128, 24), ("bf16", 8, 32), ("bf16", 128, 128)])
@pytest.mark.parametrize("which", ["q", "k", "v", "do"])
@pytest.mark.parametrize("decay", [-0.8, -0.1, 0.0])
def test_a_few_large_values_on_the_way(mf, kind, dk, dv, which, decay):
    """Steps of 1e30 among ordinary ones: what follows them, and in reverse what comes before, while they decay."""
    c = Case(kind, 2, 300, 2, dk, dv, marks="some")
    c.decay.fill_(decay)
    x = getattr(c, which)
    x[:, [40, 41, 47, 150]] *= 1e30
    c.check(mf)


@pytest.mark.parametrize("kind,dk,dv", [("f32", 16, 16), ("bf16", 32, 32), ("f16", 16, 8), ("bf16", 64, 128)])
@pytest.mark.parametrize("scale", [-3000.0, 1e30, -1e-30, 0.0])
def test_scales(mf, kind, dk, dv, scale):
    c = Case(kind, 2, 200, 2, dk, dv, marks="some", scale=scale, state=False)
    if kind == "f16" and abs(scale) > 1:
        scale = c.scale = 40.0 if scale > 0 else -40.0
    c.check(mf)
