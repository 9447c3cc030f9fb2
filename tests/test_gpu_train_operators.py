"""The training operators in a training step: their gradients together, and fits that use them."""
import os
import subprocess
import sys

import numpy as np
import pytest

from _ops_ref import U

pytestmark = pytest.mark.gpu


ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def train():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import train as t
    return t


def in_a_process_of_its_own(script):
    """(Matrix products load libraries that keep device memory.)"""
    path = os.pathsep.join([ROOT, os.path.join(ROOT, "tests")])
    r = subprocess.run([sys.executable, "-c", script], cwd=ROOT, capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, PYTHONPATH=path))
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("check", ["check_a_step_of_all_of_them", "check_single_steps_of_a_memory"])
def test_in_a_process_of_its_own(train, check):
    in_a_process_of_its_own(f"import test_gpu_train_operators as t; from paper_2609_02109_gb300 import train; t.{check}(train)")


def _steps_in_64_bits(q, k, v, decay, state, marks, scale):
    """The definition in torch operations on float64 tensors, which differentiates it by itself."""
    import torch
    keep = torch.exp(decay)[None, :, None, None]
    outs = []
    for i in range(q.shape[1]):
        m = marks[:, i, None, None, None]
        new = k[:, i, :, :, None] * v[:, i, :, None, :]
        state = torch.where(m == 0, state, torch.where(m == 2, new, keep * state + new))
        outs.append(scale * (q[:, i, :, None] @ state)[:, :, 0])
    return torch.stack(outs, 1), state


def check_a_step_of_all_of_them(train):
    """Options looked up, mixed with a trace's memory, a loss, its gradients and their clipping, against the same step in
    64-bit torch operations.  Each gradient is a sum of products in fp32 along chains of at most 200 roundings of U =
    2^-24 each, of sizes that the 64-bit step on absolute values bounds; the norms compared here are those of whole
    gradients, whose errors stay below 200 U of that step's."""
    import torch
    from paper_2609_02109_gb300 import mf
    b, t, h, d, rows = 2, 90, 3, 8, 11
    g = torch.Generator().manual_seed(4)
    normal = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    table, mix, state = normal(rows, d), normal(d, 3 * h * d) / d ** 0.5, normal(b, h, d, d)
    ids = torch.randint(-1, rows, (b, t), generator=g)
    marks = torch.randint(0, 20, (b, t), generator=g).clamp(max=2).to(torch.uint8)
    marks = torch.where(marks == 2, torch.where(torch.rand(b, t, generator=g) < 0.05, 2, 1), marks).to(torch.uint8)
    decay = torch.log1p(-1 / torch.tensor([2.0, 10.0, 100.0], dtype=torch.float64)).float()
    target = normal(b, t, h, d)

    def step(exact, absolute=False):
        kind = torch.float64 if exact else torch.float32
        size = (lambda x: x.abs()) if absolute else (lambda x: x)
        leaves = [size(x).to(kind).cuda().requires_grad_() for x in (table.float(), mix.float(), state.float())]
        tab, w, s0 = leaves
        i, m, dec = ids.cuda(), marks.cuda(), decay.cuda()
        if exact:
            x = torch.where((i >= 0)[..., None], 1.5 * tab[i.clamp(min=0)], 0.0)
        else:
            x = train.embedding(tab, i, 1.5)
        q, k, v = ((x @ p).unflatten(-1, (h, d)) for p in w.split(h * d, 1))
        if exact:
            o, last = _steps_in_64_bits(q, k, v, dec.double(), s0, m, d ** -0.5)
        else:
            o, last = train.linear_attention(q, k, v, dec, s0, m, d ** -0.5)
        weight = size(target.float()).to(kind).cuda()
        ((o * weight).sum() + last.square().sum() / 2).backward()
        return [p.grad for p in leaves]

    got, want, sizes = step(False), step(True), step(True, absolute=True)
    for x, y, z in zip(got, want, sizes):
        assert float((x.double() - y).norm()) <= 200 * U * float(z.norm())
    norm = float(torch.stack([y.square().sum() for y in want]).sum().sqrt())
    before = [x.clone() for x in got]
    told = float(mf.clip_gradients(got, 0.25 * norm))
    slack = 200 * U * float(torch.stack([z.square().sum() for z in sizes]).sum().sqrt())
    assert abs(told - norm) <= slack + 70 * U * norm
    for x, y in zip(got, before):
        assert torch.allclose(x, y * (0.25 * norm / (told + 1e-6)), rtol=1e-6, atol=0)


def test_a_broadcast_head_gets_the_sum_of_its_gradients(train):
    """Keys and values of one head, read by all: their gradients are summed over the heads, as those of copies are."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, k, v, do = normal(2, 40, 4, 6), normal(2, 40, 1, 6), normal(2, 40, 1, 6), normal(2, 40, 4, 6)
    decay = torch.tensor([-0.5, -0.1, -0.01, 0.0], device="cuda")
    grads = []
    for copies in (False, True):
        leaf_k, leaf_v = k.clone().requires_grad_(), v.clone().requires_grad_()
        wide = [x.expand(2, 40, 4, 6) for x in (leaf_k, leaf_v)]
        o, _ = train.linear_attention(q, *([x.contiguous() for x in wide] if copies else wide), decay)
        (o * do).sum().backward()
        grads.append((leaf_k.grad, leaf_v.grad))
    for x, y in zip(*grads):
        assert x.equal(y)


def test_what_has_no_gradient_raises(train):
    import torch
    q = torch.randn(1, 5, 2, 4, device="cuda", requires_grad=True)
    with pytest.raises(ValueError):
        train.linear_attention(q, q, q, torch.zeros(2, device="cuda", requires_grad=True))
    table = torch.randn(3, 4, device="cuda", requires_grad=True)
    for out, leaf in ((train.linear_attention(q, q, q, torch.zeros(2, device="cuda"))[0], q),
                      (train.embedding(table, torch.tensor([0, 2], device="cuda")), table)):
        grad, = torch.autograd.grad(out.square().sum(), [leaf], create_graph=True)
        with pytest.raises(RuntimeError):
            grad.sum().backward()


def check_single_steps_of_a_memory(train):
    """A trace taken sample by sample gives what the whole trace gives: sums of 16 and 64 products and of 16 x 30 in each,
    in fp32, 200 roundings of U at most, of values that stay below 100."""
    import torch
    memory = train.TraceMemory(seed=3)
    g = torch.Generator(device="cuda").manual_seed(6)
    with torch.no_grad():
        memory.wo.copy_(torch.randn(memory.wo.shape, device="cuda", generator=g) / 8)
    seen = torch.randn(3, 30, 4, device="cuda", generator=g)
    marks = (torch.rand(3, 30, device="cuda", generator=g) > 0.2).to(torch.uint8)
    marks[1, 20] = 2
    seen[marks == 0] = float("nan")
    with torch.no_grad():
        want, last = memory(seen, marks)
    state = torch.zeros(3, 4, 16, 16, device="cuda")
    got = torch.stack([memory.step(seen[:, i], marks[:, i], state) for i in range(30)], 1)
    assert float((got - want).abs().max()) < 200 * U * 100 and float((state - last).abs().max()) < 200 * U * 100


FIT = """
import numpy as np, torch
from paper_2609_02109_gb300 import mf, train, workload as W
prob = W.make_problem([6, 5, 4], 8, 64, 64, 3, 60.0)
trace = train.synthetic_trace(prob, 2, 1024, seed=5)
got = train.fit(prob, trace, steps=6, features=True, heads=2, clip=0.5)
assert np.isfinite(got["loss"]).all() and np.isfinite(got["norms"]).all() and got["norms"].shape == (6,)
assert got["local_feats"].shape == prob["local_feats"].shape and (got["local_feats"] != prob["local_feats"]).any()
memory, state = got["attention"]
assert state.shape == (2, 2, 16, 16) and all(torch.isfinite(p).all() and torch.isfinite(p.grad).all() for p in memory.parameters())
assert memory.wo.detach().abs().max() > 0
with mf.Context(dict(prob, weights=got["weights"], local_feats=got["local_feats"])) as ctx:
    assert ctx.search(4)["count"] <= 120
assert set(train.fit(prob, trace, steps=0, clip=1.0)) == {"weights", "memory", "state", "loss", "norms"}
assert mf.check_operators() == mf.MF_OK
"""


def test_a_fit_with_all_of_them_runs(train):
    in_a_process_of_its_own(FIT)
