"""The training example: its autograd, its optimiser and a whole fit."""
import os
import subprocess
import sys

import numpy as np
import pytest

import _ops_ref as R
from paper_2609_02109_gb300 import workload as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def train():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import train as t
    return t


def test_autograd_of_a_broadcast_gate(train):
    """A gate a channel, broadcast over a trace: its gradient is the sum of the formula's over batch and time."""
    import torch
    r = np.random.default_rng(2)
    b, t, d = 3, 500, 4
    x, w = r.standard_normal((b, t, d)), r.standard_normal((b, t, d))
    gate, wl = 2 * r.standard_normal(d), r.standard_normal((b, d))
    dev = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")  # noqa: E731
    xg, gg, h0 = dev(x).requires_grad_(), dev(gate).requires_grad_(), torch.zeros(b, d, device="cuda", requires_grad=True)
    h, last = train.recurrence(xg, gg.expand(b, t, d), h0)
    ((h * dev(w)).sum() + (last * dev(wl)).sum()).backward()
    x, z, w, wl = (v.detach().double().cpu().numpy() for v in (xg, gg.expand(b, t, d), dev(w), dev(wl)))
    dx, dz, dh0 = R.recurrence_grad(x, z, np.zeros((b, d)), None, w, wl)
    _, ex, ez, e0 = R.recurrence_bounds(x, z, np.zeros((b, d)), None, w, wl)
    assert (np.abs(xg.grad.double().cpu().numpy() - dx) <= ex).all() and (np.abs(h0.grad.double().cpu().numpy() - dh0) <= e0).all()
    # the sum of b t terms in fp32 adds at most log2(b t) + a few roundings of the terms' sizes
    off = np.abs(gg.grad.double().cpu().numpy() - dz.sum((0, 1)))
    assert (off <= ez.sum((0, 1)) + 32 * R.U * np.abs(dz).sum((0, 1))).all()


def test_one_step_of_the_optimiser(train):
    import torch
    g = torch.Generator().manual_seed(3)
    w = torch.randn(3, 40, 24, generator=g).cuda().requires_grad_()
    before = w.detach().double().cpu().numpy()
    grads = [torch.randn(3, 40, 24, generator=g).cuda() for _ in range(2)]
    opt = train.Muon([w], lr=0.1, beta=0.9)
    m = np.zeros_like(before)
    for grad in grads:
        w.grad = grad
        opt.step()
        gd = grad.double().cpu().numpy()
        m = 0.9 * m + gd
        u = gd + 0.9 * m
        for k in range(3):
            xs = R.orthogonalize(u[k], 5, (3.4445, -4.7750, 2.0315), 1e-7)
            before[k] -= 0.1 * (40 / 24) ** 0.5 * xs[-1]
            # the update's bound (its input in fp32 adds 2^-22 of roundings, which the bound's first term covers twice over)
            assert np.linalg.norm(w[k].detach().double().cpu().numpy() - before[k]) <= 0.26 * R.orth_bound(
                xs, (3.4445, -4.7750, 2.0315), "f32") + 4 * R.U * np.linalg.norm(before[k])
            before[k] = w[k].detach().double().cpu().numpy()


FIT = """
import numpy as np
from paper_2609_02109_gb300 import mf, train, workload as W
prob = W.make_problem([6, 5, 4], 8, 64, 64, 3, 60.0)
got = train.fit(prob, train.synthetic_trace(prob, 2, 2048, seed=5), steps=80)
assert np.isfinite(got["loss"]).all() and got["loss"][-1] < 0.1 * got["loss"][0], got["loss"]
with mf.Context(dict(prob, weights=got["weights"])) as ctx:
    assert ctx.search(4)["count"] <= 120
assert mf.check_operators() == mf.MF_OK
"""


def test_a_fit_learns(train):
    """Loss down by a factor of ten, and the fitted weights score in the library.  (In a process of its own: the
    example's matrix products load libraries that keep device memory.)"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIT], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
