"""How far an orthogonalised matrix may be off: limits near what the arithmetic that include/mf.h promises leaves, so that
operands with fewer bits do not pass (test_orthogonalize_limits_cpu.py holds them to that)."""
import numpy as np

import _ops_ref as R

MUON = (3.4445, -4.7750, 2.0315)


def round_to(x, type_):
    """x in 64 bits, rounded to the type's significant bits (24, 8, 11), to nearest."""
    m, e = np.frexp(x)
    bits = {"f32": 24, "bf16": 8, "f16": 11}[type_]
    return np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)


def in_fp32(g, steps, coeffs, eps):
    """The formulas in fp32 arithmetic."""
    a, b, c = (np.float32(v) for v in coeffs)
    x = g.astype(np.float32)
    tall = x.shape[0] > x.shape[1]
    x = np.ascontiguousarray(x.T) if tall else x
    x = x / (np.sqrt((x * x).sum(dtype=np.float32)) + np.float32(eps))
    for _ in range(steps):
        s = x @ x.T
        x = a * x + (b * s + c * (s @ s)) @ x
    return (x.T if tall else x).astype(np.float64)


def off(y, exact):
    return np.linalg.norm(y - exact) / np.linalg.norm(exact)


def limit(g, type_, steps=5, coeffs=MUON, eps=1e-7):
    """(exact, limit of the relative error in the Frobenius norm) of one matrix g (64 bits, values of the type).

    fp32 results: fp32 arithmetic rounds to 24 bits, two fp16 parts hold 22, and both errors grow alike from step to step, so
    at most four times what fp32 arithmetic leaves.  f16 results: that and a quarter more than the rounding of the
    exact result to the type.  bf16 results: 11-bit operands in the last two steps leave 1.1e-3 beside the rounding's 1.66e-3
    (the emulation below), root mean squares, 1.2 times the rounding together; a tenth more for the sums, which truncate."""
    exact = R.orthogonalize(g, steps, coeffs, eps)[-1]
    most = 4 * off(in_fp32(g, steps, coeffs, eps), exact) + 2.0 ** -23
    if type_ != "f32":
        most += (1.35 if type_ == "bf16" else 1.25) * off(round_to(exact, type_), exact)
    return exact, most


def emulated(g, type_, parts_of, steps=5, coeffs=MUON, eps=1e-7, bits=11):
    """The kernels' scheme with sums in 64 bits: step k's operands in parts_of(k) parts of `bits` bits."""
    a, b, c = coeffs
    x = g / (np.linalg.norm(g) + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x

    def cut(v):
        m, e = np.frexp(v)
        return np.ldexp(np.rint(np.ldexp(m, bits)), e - bits)

    def split(v, parts):
        hi = cut(v)
        return (hi, cut(v - hi) if parts > 1 else 0.0 * v)

    def product(p, q):
        return p[0] @ q[0] + p[0] @ q[1] + p[1] @ q[0]
    for k in range(steps):
        n = parts_of(k)
        xs = split(x, n)
        s = split(product(xs, (xs[0].T, xs[1].T)), n)
        bb = split(b * (s[0] + s[1]) + c * product(s, s), n)
        x = a * (xs[0] + xs[1]) + product(bb, xs)
    x = x.T if tall else x
    return round_to(x, type_)
