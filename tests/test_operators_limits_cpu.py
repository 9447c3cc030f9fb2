"""Sizes of the training operators at their limits, without a GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def mf():
    from paper_2609_02109_gb300 import build
    build.build()
    from paper_2609_02109_gb300 import mf as mod
    return mod


@pytest.mark.parametrize("type_,dim", [(0, 33), (1, 65), (2, 65)])
def test_more_sequences_than_a_launch_holds_are_refused(mf, type_, dim):
    """A sequence's channels make a block for every 32 words: two here, so 2^30 sequences are 2^31 blocks."""
    lib = mf.lib()
    got = [C.c_uint64() for _ in range(3)]
    assert lib.mf_recurrence_sizes(type_, (1 << 30) - 1, 1, dim, *map(C.byref, got)) == mf.MF_OK
    assert lib.mf_recurrence_sizes(type_, 1 << 30, 1, dim, *map(C.byref, got)) == mf.MF_EINVAL
    assert b"too many" in lib.mf_last_error()


def _bytes(mf, batch, rows, cols, steps):
    p = mf._Orthogonalize(type=0, batch=batch, rows=rows, cols=cols, steps=steps, a=3.4445, b=-4.775, c=2.0315, eps=1e-7)
    n = C.c_uint64()
    assert mf.lib().mf_orthogonalize_workspace(C.byref(p), C.byref(n)) == mf.MF_OK
    return n.value


def test_scratch_is_what_the_steps_need(mf):
    """Operands are two fp16 parts of X, X^T and, on the smaller side, A and B: none for steps = 0, one X for steps = 1."""
    for batch, m, n in ((1, 4096, 4096), (3, 1000, 3000), (40, 700, 300)):
        lo, hi = min(m, n), max(m, n)
        x, a = 8 * batch * lo * hi, 8 * batch * lo * lo  # X and X^T; A and B
        small = 1 << 20  # sums, scales and roundings to whole blocks
        assert _bytes(mf, batch, m, n, 0) <= small
        assert x + a <= _bytes(mf, batch, m, n, 1) <= 1.02 * (x + a) + small
        assert 2 * x + a <= _bytes(mf, batch, m, n, 2) <= 1.02 * (2 * x + a) + small
        assert _bytes(mf, batch, m, n, 5) >= _bytes(mf, batch, m, n, 2)
