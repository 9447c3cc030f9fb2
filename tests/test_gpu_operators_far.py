"""The training operators on tensors of more than 2^31 values: offsets beyond 32 bits."""
import pytest

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


def test_an_embedding_of_many_tokens(mf):
    """720 million tokens of three values (single values: odd rows).  A row's gradient of ones is its tokens' number:
    exact in a unit's sum (below 2^24); joined in fp32 by at most 1024 sums a share and eight shares, 2^-24 each, then
    rounded to bf16 (half a step: 2^-8)."""
    import torch
    n, rows = 720_000_000, 5
    table = torch.arange(15, device="cuda", dtype=torch.float32).view(rows, 3).bfloat16()
    g = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.randint(0, rows, (n,), device="cuda", generator=g, dtype=torch.int32)
    out = mf.embedding(table, ids)
    for at in (0, 715_827_882, n - 1000):  # (715,827,882 x 3 passes 2^31)
        assert out[at:at + 1000].equal(table[ids[at:at + 1000].long()])
    assert int((out[:, 1] != table[:, 1][ids]).sum()) == 0
    out.fill_(1)
    grad = mf.embedding_backward(out, ids, rows)
    count = torch.stack([(ids == r).sum() for r in range(rows)]).double()
    assert bool(((grad.double() - count[:, None]).abs() <= (2.0 ** -8 + 1040 * 2.0 ** -24) * count[:, None]).all())
    assert mf.check_operators() == mf.MF_OK


def test_clipping_a_large_tensor(mf):
    import torch
    n = (1 << 31) + 5000
    x = torch.full((n,), 0.5, device="cuda", dtype=torch.bfloat16)
    x[-1] = 3.0
    norm = mf.clip_gradients([x], 0.25 * 0.5 * n ** 0.5)
    # (sums of up to 2^31 equal squares by chunks of 2^14, each a sum of 2^5 a thread: fewer than 400 roundings in a row)
    assert abs(float(norm) / (0.5 * n ** 0.5) - 1) < 400 * 2.0 ** -24
    assert float(x[-1]) == 0.75 and bool((x[:-1] == 0.125).all())


def test_attention_over_a_long_trace(mf):
    """A trace in two parts, the second from the first one's state, is the trace: both are rounded to bf16 (2^-8 of a
    result) from sums that are 2^-11 of their terms' sizes off, about 8 times a result's for sums of random signs."""
    import torch
    t, h, d, cut = 300_000, 64, 128, 262_000
    g = torch.Generator(device="cuda").manual_seed(3)
    q, k, v = (torch.randn(1, t, h, d, device="cuda", generator=g, dtype=torch.bfloat16) for _ in range(3))
    decay = -torch.logspace(-3, 0, h, device="cuda")
    o, last = mf.linear_attention(q, k, v, decay, scale=d ** -0.5)
    _, state = mf.linear_attention(q[:, :cut], k[:, :cut], v[:, :cut], decay, scale=d ** -0.5)
    tail, end = mf.linear_attention(q[:, cut:], k[:, cut:], v[:, cut:], decay, state, scale=d ** -0.5)
    assert float((end - last).norm() / last.norm()) < 1e-5
    for lo in (cut, t - 2000):
        x, y = o[:, lo:lo + 2000].float(), tail[:, lo - cut:lo - cut + 2000].float()
        assert float((x - y).norm() / x.norm()) < 2 * (2.0 ** -8 + 8 * 2.0 ** -11)
    assert mf.check_operators() == mf.MF_OK
