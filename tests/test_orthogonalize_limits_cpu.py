"""The limits of the orthogonalisation's GPU tests tell the promised arithmetic from one with fewer bits."""
import numpy as np
import pytest

import _orth_limits as L


def _draw(rows, cols, type_, kind):
    r = np.random.default_rng(rows * 7 + cols)
    v = r.standard_normal((rows, cols))
    if kind == "falling":
        k = min(rows, cols)
        v = r.standard_normal((rows, k)) / np.arange(1, k + 1) @ r.standard_normal((k, cols))
    return L.round_to(0.01 * v, type_)


@pytest.mark.parametrize("kind", ["normal", "falling"])
@pytest.mark.parametrize("size", [(64, 64), (64, 12), (128, 500), (256, 256), (300, 700), (640, 520)])
def test_operands_with_fewer_bits_fail(size, kind):
    # fp32: two parts of 11 bits pass, one does not
    g = _draw(*size, "f32", kind)
    exact, most = L.limit(g, "f32")
    assert L.off(L.emulated(g, "f32", lambda k: 2), exact) <= most
    assert L.off(L.emulated(g, "f32", lambda k: 1), exact) > 10 * most
    # (nor do two in all steps but the last two)
    assert L.off(L.emulated(g, "f32", lambda k: 2 if k < 3 else 1), exact) > 10 * most
    # bf16: 11 bits in the last two steps pass, 8 bits in every step do not
    g = _draw(*size, "bf16", kind)
    exact, most = L.limit(g, "bf16")
    assert L.off(L.emulated(g, "bf16", lambda k: 2 if k < 3 else 1), exact) <= most
    assert L.off(L.emulated(g, "bf16", lambda k: 1, bits=8), exact) > most
    # f16: as fp32
    g = _draw(*size, "f16", kind)
    exact, most = L.limit(g, "f16")
    assert L.off(L.emulated(g, "f16", lambda k: 2), exact) <= most
    assert L.off(L.emulated(g, "f16", lambda k: 1), exact) > most
