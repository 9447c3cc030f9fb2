"""64-bit references of the training operators, step by step from their definitions, and the error bounds
that the GPU tests hold the kernels to (derived beside each)."""
import numpy as np

U = 2.0 ** -24  # rounding to fp32
TYPE_U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # half a unit in the last of 24, 8 and 11 bits
MISSING, SAMPLE, FIRST = 0, 1, 2


def gates(z):
    with np.errstate(over="ignore"):
        f = 1.0 / (1.0 + np.exp(-z))
        g = 1.0 / (1.0 + np.exp(z))
    return f, g


def marks_or_samples(marks, b, t):
    return np.full((b, t), SAMPLE, np.uint8) if marks is None else marks


def recurrence(x, z, h0, marks):
    """(h, last) in 64 bits; x, z [B][T][D] float64."""
    b, t, d = x.shape
    m = marks_or_samples(marks, b, t)
    f, g = gates(z)
    s = np.zeros((b, d)) if h0 is None else h0.astype(np.float64).copy()
    h = np.empty((b, t, d))
    for i in range(t):
        with np.errstate(invalid="ignore"):
            new = f[:, i] * s + g[:, i] * x[:, i]
            first = g[:, i] * x[:, i]
        k = m[:, i, None]
        s = np.where(k == MISSING, s, np.where(k == FIRST, first, new))
        h[:, i] = s
    return h, s


def recurrence_grad(x, z, h0, marks, dh, dlast):
    b, t, d = x.shape
    m = marks_or_samples(marks, b, t)
    f, g = gates(z)
    h, _ = recurrence(x, z, h0, marks)
    s0 = np.zeros((b, d)) if h0 is None else h0.astype(np.float64)
    back = np.zeros((b, d)) if dlast is None else dlast.astype(np.float64).copy()
    dx, dz = np.zeros_like(x), np.zeros_like(x)
    for i in range(t - 1, -1, -1):
        lam = dh[:, i] + back
        k = m[:, i, None]
        before = np.where(k == FIRST, 0.0, h[:, i - 1] if i else s0)
        live = k != MISSING
        with np.errstate(invalid="ignore"):
            dx[:, i] = np.where(live, g[:, i] * lam, 0.0)
            dz[:, i] = np.where(live, lam * (before - x[:, i]) * f[:, i] * g[:, i], 0.0)
            back = np.where(k == FIRST, 0.0, np.where(live, f[:, i] * lam, lam))
    return dx, dz, back


def recurrence_bounds(x, z, h0, marks, dh=None, dlast=None):
    """Bounds on |h - exact| before the final rounding, and on the gradients'.

    A step in fp32 has |error of f| <= U/2 + 3 U (1 - f), relative error of 1 - f <= 4 U and two more
    roundings, so its own error is at most (2 + 8 (1 - f)) U H, where |h|, |x| <= H (h is a mean of x and
    h0).  It decays with f: E_t = f E_{t-1} + (2 + 8 (1 - f)) U H.  Sums in another order (a sequence
    worked on in pieces, whose factors are multiplied up) at most double each term's count of roundings;
    one more factor of two covers the second-order terms.  Gradients: the same count for l with its own
    magnitudes L_t = |dh_t| + f L_{t+1}, and the product rule for dz."""
    b, t, d = x.shape
    m = marks_or_samples(marks, b, t)
    live = (m != MISSING)[..., None]
    xs = np.where(live, x, 0.0)
    f, g = gates(np.where(live, z, 0.0))
    H = np.maximum(np.abs(xs).max((0, 1), initial=0.0), 0.0 if h0 is None else np.abs(h0).max(0, initial=0.0))
    E, e = np.empty_like(x), np.zeros((b, d))
    for i in range(t):
        k = m[:, i, None]
        own = (2 + 8 * g[:, i]) * U * H
        e = np.where(k == MISSING, e, np.where(k == FIRST, 8 * U * H * g[:, i], f[:, i] * e + own))
        E[:, i] = e
    E *= 4
    if dh is None:
        return E
    s0 = np.zeros((b, d)) if h0 is None else h0.astype(np.float64)
    h, _ = recurrence(x, z, h0, marks)
    L = np.zeros((b, d)) if dlast is None else np.abs(dlast.astype(np.float64))
    e = np.zeros((b, d))
    bx, bz = np.zeros_like(x), np.zeros_like(x)
    for i in range(t - 1, -1, -1):
        k = m[:, i, None]
        L = np.abs(dh[:, i]) + L
        e = e + 2 * U * L
        before = np.where(k == FIRST, 0.0, h[:, i - 1] if i else s0)
        eb = np.where(k == FIRST, 0.0, E[:, i - 1] if i else 0.0)
        gap = np.abs(before - xs[:, i])
        fg = f[:, i] * g[:, i]
        lv = live[:, i]
        bx[:, i] = np.where(lv, g[:, i] * (4 * e + 8 * U * L), 0.0)
        bz[:, i] = np.where(lv, fg * (4 * e * gap + L * (eb + 2 * U * (np.abs(before) + np.abs(xs[:, i])))
                                      + 16 * U * L * gap) + 8 * U * U * L * (np.abs(before) + np.abs(xs[:, i])), 0.0)
        e = np.where(k == FIRST, 0.0, np.where(lv, f[:, i] * e + 4 * U * L * f[:, i], e))
        L = np.where(k == FIRST, 0.0, np.where(lv, f[:, i] * L, L))
    return E, bx, bz, 4 * e + 4 * U * L


def orthogonalize(g, steps, coeffs, eps):
    """([X after k steps for k = 0..steps] in 64 bits) of one matrix."""
    a, b, c = coeffs
    x = g / (np.sqrt((g * g).sum()) + eps) if g.any() else g * 0.0
    out = [x]
    for _ in range(steps):
        s = x @ x.T if x.shape[0] <= x.shape[1] else x.T @ x
        p = b * s + c * (s @ s)
        x = a * x + (p @ x if x.shape[0] <= x.shape[1] else x @ p)
        out.append(x)
    return out


def orth_bound(xs, coeffs, type_):
    """Bound on the Frobenius norm of the error of the last of `xs` (iterates in 64 bits).

    Step k works on operands rounded by u_k (2^-11 for one fp16 part; 2^-21 for two, with the low parts'
    product left out) and sums of n products, whose fp32 accumulation adds at most n / 16 truncations of
    2^-24 of the sum: its own error is at most (|a| + 3 |b| + 5 |c|) (u_k + 2^-24 (2 + n / 16)) |X_k|_F
    (each factor X or A enters once per product; |A|_2 <= 1.5).  A later step lets an error grow by at most the polynomial's largest slope
    on [0, 1.25].  At the end the result is rounded to its type."""
    a, b, c = (abs(v) for v in coeffs)
    s = np.linspace(0.0, 1.25, 2001)
    slope = np.abs(coeffs[0] + 3 * coeffs[1] * s ** 2 + 5 * coeffs[2] * s ** 4).max()
    n, steps = max(xs[0].shape), len(xs) - 1
    total = 2.0 ** -22 * np.linalg.norm(xs[0]) * slope ** steps
    for k in range(steps):
        u = 2.0 ** -11 if type_ == "bf16" and k >= steps - 2 else 2.0 ** -21
        total += (a + 3 * b + 5 * c) * (u + 2.0 ** -24 * (2 + n / 16)) * np.linalg.norm(xs[k]) * slope ** (steps - 1 - k)
    return total + TYPE_U[type_] * np.linalg.norm(xs[-1]) + 1e-38
