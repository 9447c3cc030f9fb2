"""What a fit returns beside the weights: the state that its own gates make of the traces."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

FIT = """
import sys, torch
from paper_2609_02109_gb300 import mf, train, workload as W
steps = int(sys.argv[1])
prob = W.make_problem([6, 5, 4], 8, 64, 64, 3, 60.0)
trace = train.synthetic_trace(prob, 2, 512, seed=5)
got = train.fit(prob, trace, steps=steps, lr=0.3)  # (gates move by 1.5 a step)
assert got["loss"].shape == (steps,)
z = torch.log(got["memory"] - 1)  # (the gates, to a few roundings of 2^-24)
_, last = mf.recurrence(trace["seen"], z.expand(trace["seen"].shape), None, trace["marks"])
assert (got["state"] - last).abs().max() <= 1e-4
"""


@pytest.mark.parametrize("steps", [0, 3])
def test_the_state_goes_with_the_memories(steps):
    """(In a process of its own: the example's matrix products load libraries that keep device memory.)"""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIT, str(steps)], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
