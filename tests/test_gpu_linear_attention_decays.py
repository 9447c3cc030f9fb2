"""Linear attention with every kind of decay, on every way that steps pass."""
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
@pytest.mark.parametrize("dk,dv,t", [(16, 16, 5), (16, 16, 60), (64, 64, 60), (128, 128, 20), (128, 128, 60), (72, 128, 200)])
@pytest.mark.parametrize("decay", [0.0, -float("inf"), -40.0, -3.0, -1e-7, 0.01, 0.3, 0.5, 0.7, 1.0, 5.0])
def test_decays_on_every_way(mf, kind, dk, dv, t, decay):
    """Memories that grow among them, where the results stay in the type's range."""
    grown = max(decay, 0.0) * (t + 2)
    if grown > (6.0 if kind == "f16" else 75.0):
        t = max(2, int((6.0 if kind == "f16" else 75.0) / decay) - 2)
    c = Case(kind, 1, t, 2, dk, dv, marks="some", scale=0.7 if kind != "f16" else 2.0 ** -7)
    c.decay.fill_(decay)
    if decay > 0.1:
        for name in ("q", "k", "v", "do"):
            x = getattr(c, name)
            x[:, ::3] = 0   # (nothing times what has grown is nothing)
        c.state[:, :, ::2] = 0
        c.dlast[:, :, 1::2] = 0
    c.check(mf)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv,decay", [(16, 16, 0.1), (64, 64, 0.1), (64, 64, 2.0), (16, 16, 2.0), (128, 128, 100.0)])
def test_nothing_times_what_has_grown_is_nothing(mf, kind, dk, dv, decay):
    """Zeros over segments whose factor is no float32: no NaN, and a late sample's results."""
    import torch
    c = Case(kind, 1, 5000 if dk == 16 else 1500, 2, dk, dv, state=True)
    c.decay.fill_(decay)
    c.k.zero_()
    c.state.zero_()
    c.do.zero_()
    c.dlast.zero_()
    c.k[:, -1] = 1
    if decay < 88:  # (else the state's gradient is no float32)
        c.do[:, 0] = 1
    c.check(mf)
    assert torch.isfinite(mf.linear_attention(c.q, c.k, c.v, c.decay, c.state)[0]).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dk,dv", [(16, 16), (64, 128), (128, 128), (40, 72)])
@pytest.mark.parametrize("layout", ["bthd", "padded", "bhtd"])
def test_heads_of_every_kind_in_one_call(mf, kind, dk, dv, layout):
    """Heads that grow beside heads that decay, by rows of every width, over segments of several chunks."""
    import torch
    for b, t in ((2, 140), (1, 150)):
        c = Case(kind, b, t, 5, dk, dv, marks="some", layout=layout)
        c.decay = torch.tensor([-float("inf"), 0.5, -0.1, 0.36, 0.0], device="cuda")
        c.check(mf)
