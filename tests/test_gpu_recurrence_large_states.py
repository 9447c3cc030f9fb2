"""States near the end of fp32's range, and what is left of them once the gates have closed."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


# One block a chain, clusters, published maps; within a segment of 16 steps, across segments, and across tiles.
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(1, 50, 8), (160, 700, 128), (40, 1500, 128), (1, 40000, 64)])
@pytest.mark.parametrize("at", [3, 40])
def test_a_closed_gate_lets_nothing_through(mf, shape, dtype, at):
    """h0 = 3e38, a closed gate (f = 0) with x = 2 at one step, then open ones (f = 1): 2 from there on.  Factors of maps that
    underflow are held at 2^-149, so of a state s at most 2^-149 s = 4.2e-7 is left, and the sum is rounded once or twice (2^-23
    each at 2); in bf16 nothing of that shows."""
    import torch
    t, dt = shape[1], getattr(torch, dtype)
    x = torch.full(shape, 2.0, device="cuda", dtype=dt)
    z = torch.full(shape, float("inf"), device="cuda", dtype=dt)
    z[:, at] = -float("inf")
    h0 = torch.full((shape[0], shape[2]), 3e38, device="cuda")
    h, last, saved = mf.recurrence(x, z, h0, save=True)
    off = 2.0 ** -149 * 3e38 + 2 * 2.0 ** -23
    assert (h[:, :at].float() == h0.to(dt).float()[:, None]).all()
    assert (h[:, at:].float() - 2).abs().max() <= off and (last - 2).abs().max() <= off
    # and backward: 3e38 behind the last step, 1 at step 1: what passes step `at` is the rest
    dh = torch.zeros_like(x)
    dh[:, 1] = 1
    _, _, dh0 = mf.recurrence_backward(dh, x, z, saved, h0)
    assert (dh0 - 1).abs().max() <= off


def test_a_large_state_decays_as_its_gates_say(mf):
    """Gates of 1/2: after t steps 2^-t of 3e38 is left, beside x = 1."""
    import torch
    t = 3000
    x = torch.ones(1, t, 64, device="cuda")
    h, last = mf.recurrence(x, torch.zeros_like(x), torch.full((1, 64), 3e38, device="cuda"))
    left = 3e38 * torch.exp2(-torch.arange(1, t + 1, device="cuda", dtype=torch.float64))
    # a step's gate is off by 6 2^-24 of it at most and the step rounds once, so after n steps the rest is off by 8 n 2^-24 of
    # itself; the mean of x, half of whose error is left at each step, by 16 2^-24
    n = torch.arange(1, t + 1, device="cuda", dtype=torch.float64)
    off = 8 * 2.0 ** -24 * n * left + 16 * 2.0 ** -24 + 2.0 ** -149 * 3e38
    assert ((h[0].double() - (1 + left)[:, None]).abs() <= off[:, None]).all()
