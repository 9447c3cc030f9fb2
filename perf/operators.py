"""Performance cases of the operators that train a predictor and its monitor state.

Two operators: `recur`, the gated linear recurrence over a monitor's trace (forward alone as a
scheduler serves it, or forward and backward as a training step runs it), and `orth`, the
orthogonalisation of an update by Newton-Schulz products, on batches of matrices.  `run` computes
them in elementary torch operations in 32 bits, or, where `own` is true, by the library's calls.

Sizes: 12 -> 64 -> 64 -> 2 and 20 -> 128 -> 128 -> 2 predictors of 5 to 8 models, 256 as the widest
hidden layer, 8 features and 16 servers are this repository's own; the others are generic.
"""
import math

import torch

own = False

STEPS, COEFFS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _recur(batch, time, dim, dtype, train, marks):
    return {"op": "recur", "batch": batch, "time": time, "dim": dim, "dtype": dtype, "train": train, "marks": marks}


def _orth(batch, rows, cols, dtype):
    return {"op": "orth", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype}


def listed():
    return [
        # one new sample of 16 servers' 8 features: a scheduler's decision tick, latency alone
        dict(_recur(16, 1, 8, "f32", False, False), name="tick"),
        # a day of samples a second of 8 servers, some missing: the state rebuilt when a scheduler starts
        dict(_recur(8, 86400, 8, "f32", False, True), name="day_of_samples"),
        # a training step on short packed traces with an odd length and width
        dict(_recur(16, 2047, 250, "bf16", True, True), name="train_packed_odd"),
        # a training step of a wide layer on many long sequences
        dict(_recur(8, 8192, 2048, "bf16", True, False), name="train_wide"),
        # a training step on one very long trace: few channels, so the work splits along time
        dict(_recur(1, 200003, 512, "f32", True, True), name="train_one_long"),
        # forward over a long context of one wide layer, as a prompt is read
        dict(_recur(1, 65536, 4096, "f16", False, False), name="prefill"),
        # the hidden layers of the five predictors of the 78,732-configuration space
        dict(_orth(5, 64, 64, "f32"), name="orth_five_hidden"),
        # first layers of six models in 5 seeds x 5 folds: many tall, narrow matrices
        dict(_orth(150, 64, 12, "f32"), name="orth_folds"),
        # the widest hidden layers, 16 models
        dict(_orth(16, 256, 256, "bf16"), name="orth_widest_hidden"),
        # odd, wide, a few matrices
        dict(_orth(3, 517, 1031, "bf16"), name="orth_odd"),
        # a tall matrix of a larger network, exact products
        dict(_orth(1, 4096, 1024, "f32"), name="orth_tall"),
        # a square matrix of a larger network: bound by the tensor cores
        dict(_orth(1, 4096, 4096, "bf16"), name="orth_large"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if rng.random() < 0.5:
        while True:
            batch, time, dim = _log(rng, 1, 64), _log(rng, 1, 262144), _log(rng, 1, 4096)
            if batch * time * dim <= 100_000_000:
                return _recur(batch, time, dim, dtype, rng.random() < 0.6, rng.random() < 0.5)
    while True:
        batch, rows, cols = _log(rng, 1, 200), _log(rng, 2, 4096), _log(rng, 2, 4096)
        case = _orth(batch, rows, cols, dtype)
        if batch * rows * cols <= 16_000_000 and work(case)["flops"] <= 6e11:
            return case


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    if case["op"] == "orth":
        # the gradient of a layer: outputs' errors times inputs, over samples whose directions fall off as 1 / i
        b, m, n = case["batch"], case["rows"], case["cols"]
        k = min(m, n)
        fall = 1.0 / torch.arange(1, k + 1, device="cuda", dtype=torch.float32)
        grad = (normal(b, m, k) * fall) @ normal(b, k, n) / math.sqrt(k)
        return {"case": case, "g": (1e-3 * grad).to(dt)}
    b, t, d = case["batch"], case["time"], case["dim"]
    s = {"case": case, "x": normal(b, t, d).to(dt), "marks": None}
    # memories from a few samples to about a thousand
    s["z"] = (normal(b, t, d) + 5.0 * torch.rand(d, device="cuda", generator=g)).to(dt)
    s["h0"] = normal(b, d)
    if case["marks"]:
        # one sample in 20 missing (the monitor leaves NaN there), a new trace about every 5,000
        u = torch.rand(b, t, device="cuda", generator=g)
        s["marks"] = torch.where(u < 0.05, 0, torch.where(u > 0.9998, 2, 1)).to(torch.uint8)
        s["x"].masked_fill_((s["marks"] == 0)[..., None], float("nan"))
    if case["train"]:
        s["dh"] = normal(b, t, d).to(dt)
        s["dlast"] = normal(b, d)
    return s


def _scan(a, b):
    """Every h_t = a_t h_{t-1} + b_t along axis 1 (h before the first is 0), by doubling: log2(T) sums, as T in a
    row would take T of them."""
    step, t = 1, a.shape[1]
    while step < t:
        b = torch.cat((b[:, :step], b[:, step:] + a[:, step:] * b[:, :-step]), 1)
        a = torch.cat((a[:, :step], a[:, step:] * a[:, :-step]), 1)
        step *= 2
    return b


def _plain_recur(s):
    x, f = s["x"].float(), torch.sigmoid(s["z"].float())
    keep = 1 - f
    prev_of = f
    if s["marks"] is not None:
        m = s["marks"][..., None]
        x = torch.where(m == 0, 0.0, x)
        keep = torch.where(m == 0, 0.0, keep)
        prev_of = torch.where(m == 0, 1.0, torch.where(m == 2, 0.0, f))
    b = keep * x
    b[:, 0] += prev_of[:, 0] * s["h0"]
    h = _scan(prev_of, b)
    out = {"h": h.to(s["x"].dtype), "last": h[:, -1].clone()}
    if not s["case"]["train"]:
        return out
    before = torch.cat((s["h0"][:, None], h[:, :-1]), 1)
    if s["marks"] is not None:
        before = torch.where(m == 2, 0.0, before)
    g = s["dh"].to(torch.float32, copy=True)  # (a copy for 32-bit inputs too: the state stays as it was)
    g[:, -1] += s["dlast"]
    behind = torch.cat((prev_of[:, 1:], torch.zeros_like(prev_of[:, :1])), 1)
    lam = _scan(behind.flip(1), g.flip(1)).flip(1)
    out["dx"] = (keep * lam).to(s["x"].dtype)
    out["dz"] = (lam * (before - x) * f * keep).to(s["x"].dtype)
    out["dh0"] = prev_of[:, 0] * lam[:, 0]
    return out


def _plain_orth(g):
    a, b, c = COEFFS
    x = g.float()
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.mT
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for _ in range(STEPS):
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    return (x.mT if tall else x).contiguous().to(g.dtype)


def run(state):
    if not own:
        return _plain_orth(state["g"]) if state["case"]["op"] == "orth" else _plain_recur(state)
    from paper_2609_02109_gb300 import mf

    if state["case"]["op"] == "orth":
        return mf.orthogonalize(state["g"], steps=STEPS, coeffs=COEFFS, eps=EPS)
    if not state["case"]["train"]:
        h, last = mf.recurrence(state["x"], state["z"], state["h0"], state["marks"])
        return {"h": h, "last": last}
    h, last, saved = mf.recurrence(state["x"], state["z"], state["h0"], state["marks"], save=True)
    dx, dz, dh0 = mf.recurrence_backward(state["dh"], state["x"], state["z"], saved, state["dlast"], state["marks"])
    return {"h": h, "last": last, "dx": dx, "dz": dz, "dh0": dh0}


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "orth":
        m, n = sorted((case["rows"], case["cols"]))
        # a step: the Gram matrix and its square (symmetric: one half of each), and the product with X
        return {"bytes": 2 * size * case["batch"] * m * n, "flops": case["batch"] * STEPS * (m * m * n + m**3 + 2 * m * m * n)}
    e, rows = case["batch"] * case["time"] * case["dim"], case["batch"] * case["time"] * bool(case["marks"])
    # forward: x, z -> h.  Backward, after the rest of a network has run: dh, x, z -> dx, dz.
    passes = [3, 5] if case["train"] else [3]
    state = 8 * case["batch"] * case["dim"]
    return {"bytes": sum(p * size * e + rows + state for p in passes), "flops": 6 * e + (10 * e if case["train"] else 0)}


def _chain(a, b, first):
    """h_t = a_t h_{t-1} + b_t in 64 bits, in rows of about sqrt(T) steps: each step for all rows at once, then row by row."""
    n, t, d = a.shape
    size = max(1, math.isqrt(t))
    rows = -(-t // size)
    pad = rows * size - t
    a = torch.cat((a, a.new_ones(n, pad, d)), 1).view(n, rows, size, d)
    h = torch.cat((b, b.new_zeros(n, pad, d)), 1).view(n, rows, size, d)
    a, h = a.clone(), h.clone()
    for i in range(1, size):
        h[:, :, i] += a[:, :, i] * h[:, :, i - 1]
        a[:, :, i] *= a[:, :, i - 1]
    for r in range(rows):
        h[:, r] += a[:, r] * first[:, None]
        first = h[:, r, -1]
    return h.view(n, rows * size, d)[:, :t]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "orth":
        # the polynomial of the Gram matrix alone, times G at the end: X_k = Q_k G / |G|
        g = s["g"].double()
        tall = g.shape[1] > g.shape[2]
        g = g.mT if tall else g
        g = g / (torch.linalg.matrix_norm(g, keepdim=True) + EPS)
        gram = g @ g.mT
        eye = torch.eye(gram.shape[1], dtype=torch.float64, device="cuda").expand_as(gram)
        q = eye
        for _ in range(STEPS):
            p = COEFFS[0] * eye + COEFFS[1] * gram + COEFFS[2] * (gram @ gram)
            q, gram = p @ q, p @ gram @ p
        x = q @ g
        return (x.mT if tall else x).contiguous()
    f = torch.sigmoid(s["z"].double())
    x, other, factor = s["x"].double(), torch.sigmoid(-s["z"].double()), f
    if s["marks"] is not None:
        missing, first = (s["marks"] == 0)[..., None], (s["marks"] == 2)[..., None]
        x, other = x.masked_fill(missing, 0.0), other.masked_fill(missing, 0.0)
        factor = f.masked_fill(missing, 1.0).masked_fill(first, 0.0)
    h0 = s["h0"].double()
    h = _chain(factor, other * x, h0)
    out = {"h": h, "last": h[:, -1].clone()}
    if case["train"]:
        gap = torch.cat((h0[:, None], h[:, :-1]), 1)
        if s["marks"] is not None:
            gap = gap.masked_fill(first, 0.0)
        gap = (gap - x) * f * other
        # the costate mu_t = f_t lambda_t, which is what the step before receives
        g = s["dh"].double()
        mu = _chain(factor.flip(1), (factor * g).flip(1), torch.zeros_like(h0))
        # the last step's own part of dlast reaches step t through the product of the factors behind it
        mu += _chain(factor.flip(1), torch.zeros_like(g), s["dlast"].double())
        mu = mu.flip(1)
        lam = g + torch.cat((mu[:, 1:], s["dlast"].double()[:, None]), 1)
        out["dx"], out["dz"], out["dh0"] = other * lam, lam * gap, mu[:, 0].clone()
    return out
