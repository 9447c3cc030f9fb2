"""The operators' bounded waits made to run out on the GPU, without a fault or a hang: a block waits on a flag that
nothing sets, those that wait for it give up in turn, the call's status word says so, and the next call is right."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    yield m
    m.debug_operators_wait_test(0)


def _gives_up(mf, call):
    """One call whose waits run out, then the same call as before: equal bits."""
    want = call()
    assert mf.check_operators() == mf.MF_OK
    mf.debug_operators_wait_test(2)
    try:
        call()
    finally:
        mf.debug_operators_wait_test(0)
    assert mf.check_operators() == mf.MF_ETIMEOUT
    assert mf.check_operators() == mf.MF_OK  # (the check clears the flag)
    assert all(p.equal(q) for p, q in zip(call(), want))
    assert mf.check_operators() == mf.MF_OK


# One block a chain, clusters, and blocks that publish their maps in memory (one round, and several); rows that come by
# tensor copies, by words, and straight from memory.
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(160, 700, 128), (40, 1500, 128), (40, 1500, 100), (1, 40000, 64), (1, 100000, 512),
                                   (2, 30000, 33), (40, 1500, 65)])
def test_recurrence(mf, shape, dtype):
    import torch
    g = torch.Generator(device="cuda").manual_seed(sum(shape))
    x, z, dh = (torch.randn(shape, device="cuda", generator=g).to(getattr(torch, dtype)) for _ in range(3))
    _gives_up(mf, lambda: mf.recurrence(x, z, save=True))
    saved = mf.recurrence(x, z, save=True)[2]
    _gives_up(mf, lambda: mf.recurrence_backward(dh, x, z, saved))


def test_a_call_without_waits_is_as_ever(mf):
    import torch
    x = torch.randn(3, 20, 8, device="cuda")
    want = mf.recurrence(x, x)
    mf.debug_operators_wait_test(2)
    try:
        got = mf.recurrence(x, x)
    finally:
        mf.debug_operators_wait_test(0)
    assert mf.check_operators() == mf.MF_OK and all(p.equal(q) for p, q in zip(got, want))


# All steps in one block; tiles of one SM, with the depth split over a cluster and without; pairs of SMs; one part and two.
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shape", [(5, 64, 64), (700, 20, 12), (2, 256, 256), (1, 300, 700), (40, 200, 260), (16, 512, 512)])
def test_orthogonalize(mf, shape, dtype):
    import torch
    g = torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(sum(shape))).to(getattr(torch, dtype))
    for steps in (1, 3):
        _gives_up(mf, lambda: (mf.orthogonalize(g, steps=steps),))
