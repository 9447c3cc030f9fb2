"""The status word of the operators' bounded waits, made by whatever call comes first."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# The first call of the process is a captured one, after the allocator has handed out and taken back words that are not zero.
CAPTURED_FIRST = """
import torch
from paper_2609_02109_gb300 import mf
x = torch.randn(1, 40000, 64, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    torch.full((1 << 18,), -1, dtype=torch.int32, device="cuda")
    got = mf.recurrence(x, x)
assert mf.check_operators() == mf.MF_OK, "before a replay"
graph.replay()
torch.cuda.synchronize()
want = mf.recurrence(x, x)
assert all(p.equal(q) for p, q in zip(got, want))
assert mf.check_operators() == mf.MF_OK
mf.debug_operators_wait_test(2)
mf.recurrence(x, x)
mf.debug_operators_wait_test(0)
graph.replay()  # clears nothing
assert mf.check_operators() == mf.MF_ETIMEOUT
assert mf.check_operators() == mf.MF_OK
"""

# First calls from many threads on streams of their own: one word, and no flag lost.
MANY_FIRST = """
import threading, torch
from paper_2609_02109_gb300 import mf
x = torch.randn(1, 40000, 64, device="cuda")
torch.cuda.synchronize()
words, gate = [], threading.Barrier(8)
def first():
    with torch.cuda.stream(torch.cuda.Stream()):
        gate.wait()
        mf.debug_operators_wait_test(2)
        mf.recurrence(x, x)
        words.append(mf._status_word(x.device))
threads = [threading.Thread(target=first) for _ in range(8)]
[t.start() for t in threads]
[t.join() for t in threads]
assert len(words) == 8 and len(set(words)) == 1
assert mf.check_operators() == mf.MF_ETIMEOUT
"""


@pytest.mark.parametrize("script", [CAPTURED_FIRST, MANY_FIRST], ids=["captured_first", "many_first"])
def test_in_a_process_of_its_own(script):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    r = subprocess.run([sys.executable, "-c", script], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
