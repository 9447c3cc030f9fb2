"""Linear attention with one operand at a time on rows that allow no wide loads, beside others that do: equal bits."""
import pytest

from test_gpu_linear_attention_paths import laid_out, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dk,dv", [(64, 128), (128, 64), (40, 104), (104, 40), (64, 64), (128, 128)])
@pytest.mark.parametrize("b,t,h", [(2, 300, 2), (1, 2000, 1)])
def test_one_operand_at_a_time(mf, kind, dk, dv, b, t, h):
    """Odd offsets and strides, even ones of two, and rows of four: of q, k, v and do in turn."""
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]
    g = torch.Generator(device="cuda").manual_seed(dk + 5 * dv)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    args = [normal(b, t, h, d).to(dt) for d in (dk, dk, dv, dv)]
    decay, state = -torch.rand(h, device="cuda", generator=g) / 10, normal(b, h, dk, dv)
    marks = (torch.rand(b, t, device="cuda", generator=g) > 0.1).to(torch.uint8)
    marks[:, t // 2] = 2
    want = run(mf, *args, decay, state, marks)
    for i in range(4):
        for pad, at in ((3, 1), (2, 2), (12, 4)):
            moved = list(args)
            moved[i] = laid_out(args[i], pad, at)
            got = run(mf, *moved, decay, state, marks)
            assert all(x.equal(y) for x, y in zip(got, want)), (i, pad, at)
    assert mf.check_operators() == mf.MF_OK


def test_a_gradient_that_comes_as_a_narrow_view(mf):
    """What is joined behind a column of another tensor gets its gradient as a view at an odd offset."""
    import torch
    from paper_2609_02109_gb300 import train
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(2, 150, 3, d, device="cuda", generator=g).bfloat16().requires_grad_() for d in (64, 64, 128))
    decay = torch.tensor([-0.1, -0.01, -0.5], device="cuda")
    weight = torch.randn(2, 150, 3, 129, device="cuda", generator=g).bfloat16()
    o, _ = train.linear_attention(q, k, v, decay)
    joined = torch.cat((torch.ones_like(o[..., :1]), o), -1)
    got = torch.autograd.grad((joined * weight).sum(), (q, k, v))
    o, _ = train.linear_attention(q, k, v, decay)
    want = torch.autograd.grad(o, (q, k, v), weight[..., 1:].contiguous())
    assert all(x.equal(y) for x, y in zip(got, want)) and mf.check_operators() == mf.MF_OK
