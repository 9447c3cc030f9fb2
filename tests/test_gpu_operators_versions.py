"""Tensors that operators write in place say so: a gradient that still needs them raises instead of being wrong."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


def test_a_step_changes_its_state(mf):
    import torch
    from paper_2609_02109_gb300 import train
    q, k, v = (torch.randn(2, 20, 2, 8, device="cuda").requires_grad_() for _ in range(3))
    decay = torch.tensor([-0.1, -0.2], device="cuda")
    _, last = train.linear_attention(q, k, v, decay)
    loss = (last * last).sum()   # (needs the state that it was)
    one = [x.detach()[:, 0].contiguous() for x in (q, k, v)]
    mf.linear_attention_step(*one, decay, last.detach())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


@pytest.mark.parametrize("sizes", [[5, 7], [700000, 0, 3]])
def test_clipping_changes_what_it_writes(mf, sizes):
    import torch
    for apart in (False, True):
        grads, out = ([torch.randn(n, device="cuda") for n in sizes] for _ in range(2))
        before = [[x._version for x in s] for s in (grads, out)]
        mf.clip_gradients(grads, 0.5, out=out if apart else None)
        assert [x._version == n for x, n in zip(grads, before[0])] == [apart] * len(sizes)
        assert [x._version == n for x, n in zip(out, before[1])] == [not apart] * len(sizes)


def test_orthogonalize_changes_its_out(mf):
    import torch
    g, out = torch.randn(6, 4, device="cuda"), torch.empty(6, 4, device="cuda")
    for x, y in ((g, out), (g.mT, out.mT)):
        before = out._version, g._version
        mf.orthogonalize(x, out=y)
        assert out._version > before[0] and g._version == before[1]


def test_in_inference_mode(mf):
    import torch
    with torch.inference_mode():
        state = torch.zeros(2, 2, 8, 8, device="cuda")
        x = torch.ones(2, 2, 8, device="cuda")
        o = mf.linear_attention_step(x, x, x, torch.zeros(2, device="cuda"), state)
        assert bool((state == 1).all()) and bool((o == 8).all())
        mf.clip_gradients([state], 1.0)
