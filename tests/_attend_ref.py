"""64-bit references of linear attention, the embedding's gradient and clipping, step by step from their definitions, and
the bounds that the GPU tests hold the kernels to (derived beside each)."""
import numpy as np

from _ops_ref import FIRST, MISSING, SAMPLE, TYPE_U, U


def attend(q, k, v, log_decay, state, marks, scale):
    """(o, last, states after each step); q, k [B][T][H][dk], v [B][T][H][dv], float64."""
    b, t, h, dk = q.shape
    s = np.zeros((b, h, dk, v.shape[3])) if state is None else state.astype(np.float64).copy()
    f = np.exp(log_decay)[None, :, None, None]
    o, states = np.empty((b, t, h, v.shape[3])), np.empty((b, t, *s.shape[1:]))
    for i in range(t):
        m = (np.full(b, SAMPLE) if marks is None else marks[:, i])[:, None, None, None]
        with np.errstate(invalid="ignore", over="ignore"):
            new = k[:, i, :, :, None] * v[:, i, :, None, :]
            s = np.where(m == MISSING, s, np.where(m == FIRST, new, f * s + new))
            o[:, i] = scale * np.einsum("bhk,bhkv->bhv", q[:, i], s)
        states[:, i] = s
    return o, s, states


def attend_grad(do, dlast, q, k, v, log_decay, state, marks, scale):
    b, t, h, dk = q.shape
    _, _, states = attend(q, k, v, log_decay, state, marks, scale)
    f = np.exp(log_decay)[None, :, None, None]
    g = np.zeros((b, h, dk, v.shape[3])) if dlast is None else dlast.astype(np.float64).copy()
    dq, dk_, dv = np.empty_like(q), np.zeros_like(k), np.zeros_like(v)
    for i in range(t - 1, -1, -1):
        m = np.full(b, SAMPLE) if marks is None else marks[:, i]
        live, m4 = (m != MISSING)[:, None, None], m[:, None, None, None]
        g = g + scale * q[:, i, :, :, None] * do[:, i, :, None, :]
        dq[:, i] = scale * np.einsum("bhkv,bhv->bhk", states[:, i], do[:, i])
        with np.errstate(invalid="ignore"):
            dk_[:, i] = np.where(live, np.einsum("bhkv,bhv->bhk", g, np.where(live, v[:, i], 0)), 0)
            dv[:, i] = np.where(live, np.einsum("bhkv,bhk->bhv", g, np.where(live, k[:, i], 0)), 0)
        g = np.where(m4 == FIRST, 0, np.where(m4 == MISSING, g, f * g))
    return dq, dk_, dv, g


def without_missing(k, v, marks):
    if marks is None:
        return k, v
    gone = (marks == MISSING)[:, :, None, None]
    return np.where(gone, 0, k), np.where(gone, 0, v)


def relative(kind, t, dk, dv):
    """What a result is off before its rounding, relative to the sum of its terms' sizes.  Each term is a product of two
    or three inputs, a weight and the scale: 6 roundings of U = 2^-24.  Its weight f^n comes in one factor for each chunk
    that the term passes (chunks of 32 or more: t / 32 + 2 factors, 4 U each: two of exp2, two of its argument, whose
    size x leaves x 2^-x < 0.6 of itself in the weight), and the state that carries it is rounded once a chunk.  The
    sums: dk or dv terms a product, up to 128 terms of a chunk, one a chunk; tensor cores truncate (2 U a term instead
    of U).  16-bit types on the tensor cores: the weighted products of x and y of a chunk as one part of 11 bits for bf16
    results (2^-11; the values of bf16's type stay as they are), two parts of 11 bits else (2^-21), the state as two
    parts of 8 (2^-15) or 11 bits, the weighted y in two of 11."""
    fp32 = U * (6 + 6 * (t / 32 + 2) + 2 * (dk + dv + 128))
    return fp32 + {"f32": 0.0, "bf16": 2.0 ** -11 + 2.0 ** -15, "f16": 2.0 ** -20}[kind]


def state_relative(kind, t, dk, dv):
    """The same for a state, which fp32 holds: no product of a chunk nor a state passes fewer bits."""
    return U * (6 + 6 * (t / 32 + 2) + 2 * (dk + dv + 128)) + (0.0 if kind == "f32" else 2.0 ** -20)


def attend_bounds(kind, do, dlast, q, k, v, log_decay, state, marks, scale):
    """Bounds of (o, last) or, with do, of (dq, dk, dv, dstate): the relative ones times the results of the inputs'
    sizes, and half a step of the results' type (2^-24, 2^-8, 2^-11 of them; below the normal range of fp16 half of
    2^-24)."""
    t, dk, dv = q.shape[1], q.shape[3], v.shape[3]
    k, v = without_missing(k, v, marks)
    a = [None if x is None else np.abs(x.astype(np.float64)) for x in (q, k, v, state, do, dlast)]
    rel, state_rel = relative(kind, t, dk, dv), state_relative(kind, t, dk, dv)
    tiny = 2.0 ** -25 if kind == "f16" else 1e-45

    def rounded(x, size):
        return rel * size + TYPE_U[kind] * (np.abs(x) + rel * size) + tiny

    if do is None:
        o, last, _ = attend(q, k, v, log_decay, state, marks, scale)
        so, slast, _ = attend(a[0], a[1], a[2], log_decay, a[3], marks, abs(scale))
        return rounded(o, so), state_rel * slast + 1e-45
    got = attend_grad(do, dlast, q, k, v, log_decay, state, marks, scale)
    size = attend_grad(a[4], a[5], a[0], a[1], a[2], log_decay, a[3], marks, abs(scale))
    return (*(rounded(x, s) for x, s in zip(got[:3], size[:3])), state_rel * size[3] + 1e-45)


def embedding_grad(dout, ids, rows, scale):
    """(gradient, bound): the sum of n terms in fp32 is off by at most n U of the terms' sizes, the scale one rounding
    more, then half a step of the type."""
    total, size = np.zeros((rows, dout.shape[1])), np.zeros((rows, dout.shape[1]))
    live = ids >= 0
    np.add.at(total, ids[live], dout[live])
    np.add.at(size, ids[live], np.abs(dout[live]))
    count = np.bincount(ids[live], minlength=rows)[:, None]
    return scale * total, abs(scale) * size * U * (count + 1)
