"""What a fit returns beside the weights: the state that its own gates make of the traces."""
import pytest

from paper_2609_02109_gb300 import workload as W

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("steps", [0, 3])
def test_the_state_goes_with_the_memories(steps):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf, train
    prob = W.make_problem([6, 5, 4], 8, 64, 64, 3, 60.0)
    trace = train.synthetic_trace(prob, 2, 512, seed=5)
    got = train.fit(prob, trace, steps=steps, lr=0.3)  # (gates move by 1.5 a step)
    assert got["loss"].shape == (steps,)
    z = torch.log(got["memory"] - 1)  # (the gates, to a few roundings of 2^-24)
    _, last = mf.recurrence(trace["seen"], z.expand(trace["seen"].shape), None, trace["marks"])
    assert (got["state"] - last).abs().max() <= 1e-4
