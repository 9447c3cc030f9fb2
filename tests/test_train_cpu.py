"""The training example's autograd without a GPU: the library's two calls replaced by the 64-bit reference."""
import numpy as np
import pytest

import _ops_ref as R


@pytest.fixture
def train(monkeypatch):
    import torch
    from paper_2609_02109_gb300 import build
    build.build()
    from paper_2609_02109_gb300 import train as mod

    def num(t):
        return None if t is None else t.detach().numpy()

    def forward(x, z, h0=None, marks=None, save=False):
        h, last = R.recurrence(num(x), num(z), num(h0), num(marks))
        return tuple(map(torch.tensor, (h, last))) + ((torch.zeros(1),) if save else ())

    def backward(dh, x, z, saved, dlast=None, marks=None):
        return tuple(map(torch.tensor, R.recurrence_grad(num(x), num(z), None, num(marks), num(dh), num(dlast))))
    monkeypatch.setattr(mod.mf, "recurrence", forward)
    monkeypatch.setattr(mod.mf, "recurrence_backward", backward)
    return mod


def _inputs():
    import torch
    r = np.random.default_rng(1)
    return [torch.tensor(r.standard_normal((2, 6, 3)), requires_grad=True) for _ in range(2)]


def test_first_order(train):
    import torch
    x, z = _inputs()
    h, last = train.recurrence(x, z)
    dx, dz = torch.autograd.grad((h ** 2).sum() + last.sum(), (x, z))
    want = R.recurrence_grad(x.detach().numpy(), z.detach().numpy(), None, None, 2 * h.detach().numpy(), np.ones((2, 3)))
    assert np.allclose(dx, want[0], atol=1e-14) and np.allclose(dz, want[1], atol=1e-14)


def test_a_second_derivative_is_refused(train):
    """The gradient has no gradient of its own: a loss that holds it raises, rather than losing its part."""
    import torch
    x, z = _inputs()
    h, _ = train.recurrence(x, z)
    dx, dz = torch.autograd.grad((h ** 2).sum(), (x, z), create_graph=True)
    with pytest.raises(RuntimeError, match="twice"):
        ((h ** 2).sum() + (dx ** 2).sum()).backward()


def test_the_optimiser_leaves_parameters_without_a_gradient(train, monkeypatch):
    import torch
    monkeypatch.setattr(train.mf, "orthogonalize", lambda u, steps: u)
    w = [torch.ones(2, 3, 4, requires_grad=True) for _ in range(2)]
    opt = train.Muon(w, lr=0.5, beta=0.0)
    w[0].grad = torch.ones(2, 3, 4)
    opt.step()
    assert (w[0] == 0.5).all() and (w[1] == 1).all() and not opt.buffers[1].any()
