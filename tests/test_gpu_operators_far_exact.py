"""Linear attention at offsets beyond 2^31 values against the 64-bit steps."""
import numpy as np
import pytest

import _attend_ref as A

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("less than 80 GB free")
    from paper_2609_02109_gb300 import mf as m
    yield m
    torch.cuda.empty_cache()


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [128, 32])
def test_the_end_of_a_long_trace(mf, kind, dim):
    """Heads that forget half a sample's part in every step: 200 steps before the compared ones leave 2^-200 of what was,
    which is nothing beside a bound.  On the tensor cores and step by step, with the gradients of the trace's end."""
    import torch
    h, tail = 8192 // dim, 260
    t = (1 << 31) // 8192 + 700   # (time x heads x dim passes 2^31)
    g = torch.Generator(device="cuda").manual_seed(5)
    dt = torch.bfloat16 if kind == "bf16" else torch.float16
    q, k, v, do = (torch.randn(1, t, h, dim, device="cuda", generator=g, dtype=dt) for _ in range(4))
    decay = torch.full((h,), -0.7, device="cuda")
    o, last, saved = mf.linear_attention(q, k, v, decay, scale=0.3, save=True)
    dq, dk, dv, _ = mf.linear_attention_backward(do, q, k, v, decay, saved, scale=0.3)
    at = [0, h // 2, h - 1]
    d = lambda x: x[:, -tail:, at].double().cpu().numpy()  # noqa: E731
    host = (d(q), d(k), d(v), np.full(3, float(decay[0])), None, None, float(np.float32(0.3)))
    want, bounds = A.attend(*host), A.attend_bounds(kind, None, None, *host)
    assert (np.abs(d(o) - want[0])[:, 200:] <= bounds[0][:, 200:]).all()
    assert (np.abs(last[:, at].double().cpu().numpy() - want[1]) <= bounds[1]).all()
    want, bounds = A.attend_grad(d(do), None, *host), A.attend_bounds(kind, d(do), None, *host)
    for x, exact, bound in zip((dq, dk, dv), want, bounds):
        assert (np.abs(d(x) - exact)[:, 200:] <= bound[:, 200:]).all()
    assert mf.check_operators() == mf.MF_OK
