"""Linear attention called from several threads."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


def test_two_threads_at_once_say_what_failed(mf):
    """Two types of attention on streams of their own, 20 calls a thread; what a thread raises is kept."""
    import threading
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    cases = []
    for dt in (torch.bfloat16, torch.float16, torch.float32):
        q, k, v = (torch.randn(1, 3000, 2, 128, device="cuda", generator=g).to(dt) for _ in range(3))
        decay = torch.tensor([-0.1, -0.01], device="cuda")
        cases.append((q, k, v, decay, mf.linear_attention(q, k, v, decay)))
    torch.cuda.synchronize()
    equal, raised = [], []

    def work(case):
        q, k, v, decay, want = case
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got = mf.linear_attention(q, k, v, decay)
                    torch.cuda.current_stream().synchronize()
                    equal.append(all(x.equal(y) for x, y in zip(got, want)))
        except Exception as e:
            raised.append(e)

    threads = [threading.Thread(target=work, args=(c,)) for c in cases for _ in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not raised and equal == [True] * 120 and mf.check_operators() == mf.MF_OK
