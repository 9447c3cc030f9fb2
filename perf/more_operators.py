"""Performance cases of the operators that a training step of the predictors runs around its recurrence and its updates.

Three operators.  `embed`: the learned features of options (or of any tokens) looked up and scaled, and the gradient of
their table, summed over every place where a row was used.  `attend`: linear attention over a monitor's trace, whose state
decays at a rate of each head's own: whole traces forward, forward and backward as a training step runs them, and single
tokens against a state that a scheduler keeps.  `clip`: the norm of all gradients of a model, and the gradients scaled by it.
`run` computes them in elementary torch operations in 32 bits, or, where `own` is true, by the library's calls.

Sizes: 48 and 144 options of 8 features, 5 models of 12 -> 64 -> 64 -> 2 and 16 servers are this repository's own; the
others are generic.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


def _embed(rows, dim, tokens, dtype, train, pad):
    return {"op": "embed", "rows": rows, "dim": dim, "tokens": tokens, "dtype": dtype, "train": train, "pad": pad}


def _attend(batch, time, heads, dk, dv, dtype, mode, marks):
    return {"op": "attend", "batch": batch, "time": time, "heads": heads, "dk": dk, "dv": dv, "dtype": dtype, "mode": mode,
            "marks": marks}


def _clip(tensors, least, most, dtype, max_norm):
    return {"op": "clip", "tensors": tensors, "least": least, "most": most, "dtype": dtype, "max_norm": max_norm}


def listed():
    return [
        # the features of one configuration of six models with 24 options each: a decision's lookup, latency alone
        dict(_embed(144, 8, 6, "f32", False, False), name="embed_decision"),
        # a training step over 2,048 observations of each of five models: 48 options, each used by the hundred
        dict(_embed(48, 8, 10240, "f32", True, False), name="embed_options"),
        # a training step over a large vocabulary, where few rows are used often and most never; a padded batch
        dict(_embed(100003, 1024, 65536, "bf16", True, True), name="embed_vocabulary"),
        # one new sample of 16 servers' 8 features: a scheduler's decision tick, latency alone
        dict(_attend(16, 1, 2, 8, 8, "f32", "step", True), name="attend_tick"),
        # one token for each of 128 sequences in flight: the state is read and written once
        dict(_attend(128, 1, 16, 128, 128, "bf16", "step", False), name="attend_decode"),
        # a day of samples a second of 8 servers, some missing: the state rebuilt when a scheduler starts
        dict(_attend(8, 86400, 4, 16, 16, "f32", "forward", True), name="attend_day"),
        # a long prompt of one sequence, so that its heads' work has to be split along time
        dict(_attend(1, 65536, 16, 128, 128, "bf16", "forward", False), name="attend_prompt"),
        # a training step over many sequences
        dict(_attend(8, 4096, 16, 128, 128, "bf16", "train", False), name="attend_train"),
        # a training step on short packed traces with an odd length, odd heads, and widths that fill no tile
        dict(_attend(5, 2047, 7, 100, 72, "f16", "train", True), name="attend_train_odd"),
        # the gradients of five predictors and four gates: a small model's step, latency alone
        dict(_clip(7, 4, 20480, "f32", 1.0), name="clip_predictors"),
        # a network of many layers with odd sizes, some parameters in 32 bits
        dict(_clip(1500, 1, 200000, "mixed", 0.5), name="clip_many"),
        # a large network's matrices
        dict(_clip(24, 4000000, 40000000, "bf16", 1.0), name="clip_large"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    kind = rng.random()
    if kind < 0.3:
        while True:
            rows, dim, tokens = _log(rng, 2, 262144), _log(rng, 1, 4096), _log(rng, 1, 262144)
            if rows * dim <= 100_000_000 and tokens * dim <= 60_000_000:
                return _embed(rows, dim, tokens, dtype, rng.random() < 0.7, rng.random() < 0.5)
    if kind < 0.5:
        most = _log(rng, 1, 10_000_000)
        case = _clip(_log(rng, 1, 1000), _log(rng, 1, most), most, rng.choice([dtype, "mixed"]), rng.choice([0.1, 1.0, 10.0]))
        while sum(_sizes(case)) > 400_000_000:
            case["tensors"] = max(1, case["tensors"] // 2)
        return case
    mode = rng.choice(["step", "forward", "train", "train"])
    while True:
        case = _attend(_log(rng, 1, 256), 1 if mode == "step" else _log(rng, 1, 100000), _log(rng, 1, 32), _log(rng, 4, 128),
                       _log(rng, 4, 128), dtype, mode, rng.random() < 0.5)
        b, t, h, dk, dv = (case[n] for n in ("batch", "time", "heads", "dk", "dv"))
        chunks = -(-t // _chunk(t))
        if (b * t * h * max(dk, dv) <= 60_000_000 and b * h * chunks * dk * dv <= 250_000_000
                and b * h * chunks * chunks <= 100_000_000 and b * h * t * _chunk(t) <= 300_000_000):
            return case


def _sizes(case):
    """Elements of each tensor: the same for every seed."""
    r = random.Random(case["tensors"] * 7 + case["most"])
    return [_log(r, case["least"], case["most"]) for _ in range(case["tensors"])]


def _types(case):
    return [torch.float32 if case["dtype"] == "f32" or (case["dtype"] == "mixed" and i % 3 == 2) else
            torch.float16 if case["dtype"] == "f16" else torch.bfloat16 for i in range(case["tensors"])]


def _views(sizes, types, make):
    """(flat buffers, tensors): the tensors of a type lie one behind the other in a buffer, as a step's buckets do."""
    flat, at, views = {}, {}, []
    for t in sorted(set(types), key=str):
        flat[t] = make(sum(n for n, u in zip(sizes, types) if u == t), t)
        at[t] = 0
    for n, t in zip(sizes, types):
        views.append(flat[t][at[t]:at[t] + n])
        at[t] += n
    return list(flat.values()), views


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    if case["op"] == "clip":
        sizes, types = _sizes(case), _types(case)
        _, grads = _views(sizes, types, lambda n, t: torch.randn(n, device="cuda", generator=g, dtype=t))
        # layers' gradients differ in size by about a thousand
        size = torch.exp(7.0 * torch.rand(len(sizes), device="cuda", generator=g) - 9.0).tolist()
        for v, s in zip(grads, size):
            v.mul_(s)
        flat, outs = _views(sizes, types, lambda n, t: torch.zeros(n, device="cuda", dtype=t))
        return {"case": case, "grads": grads, "outs": outs, "flat": flat}
    dt = DTYPES[case["dtype"]]
    if case["op"] == "embed":
        r, d, n = case["rows"], case["dim"], case["tokens"]
        # how often a token is used falls as 1 / its rank: rank = rows^u - 1, dealt over the table by a stride
        u = torch.rand(n, device="cuda", generator=g, dtype=torch.float64)
        rank = (torch.exp(u * math.log(r + 1.0)) - 1.0).long().clamp_(0, r - 1)
        stride = 7919
        while math.gcd(stride, r) > 1:
            stride += 1
        ids = (rank * stride + 13) % r
        if case["pad"]:
            ids.masked_fill_(torch.rand(n, device="cuda", generator=g) < 0.06, -1)
        s = {"case": case, "table": (normal(r, d) / math.sqrt(d)).to(dt), "ids": ids, "scale": math.sqrt(d)}
        if case["train"]:
            s["dout"] = (0.01 * normal(n, d)).to(dt)
        return s
    b, t, h, dk, dv = (case[n] for n in ("batch", "time", "heads", "dk", "dv"))
    # memories from 2 to 2,000 samples over the heads
    memory = torch.exp(torch.linspace(math.log(2.0), math.log(2000.0), h, device="cuda"))
    s = {"case": case, "log_decay": torch.log1p(-1.0 / memory), "scale": dk ** -0.5, "marks": None,
         "state": normal(b, h, dk, dv)}
    lead = (b, h) if case["mode"] == "step" else (b, t, h)
    s["q"], s["k"], s["v"] = normal(*lead, dk).to(dt), normal(*lead, dk).to(dt), normal(*lead, dv).to(dt)
    if case["marks"]:
        # one sample in 20 missing (the monitor leaves NaN there), a new trace about every 5,000
        u = torch.rand(lead[:-1], device="cuda", generator=g)
        s["marks"] = torch.where(u < 0.05, 0, torch.where(u > 0.9998, 2, 1)).to(torch.uint8)
        gone = (s["marks"] == 0)[..., None, None]
        s["k"].masked_fill_(gone, float("nan"))
        s["v"].masked_fill_(gone, float("nan"))
    if case["mode"] == "train":
        s["do"], s["dlast"] = normal(b, t, h, dv).to(dt), normal(b, h, dk, dv)
    return s


def _plain_embed(s):
    ids, table = s["ids"], s["table"]
    live = (ids >= 0)[:, None]
    out = torch.where(live, table[ids.clamp(min=0)].float() * s["scale"], 0.0).to(table.dtype)
    if not s["case"]["train"]:
        return {"out": out}
    d = torch.where(live, s["dout"].float(), 0.0)
    total = torch.zeros(table.shape, device="cuda").index_add_(0, ids.clamp(min=0), d)
    return {"out": out, "dtable": (total * s["scale"]).to(table.dtype)}


def _plain_clip(s):
    squares = torch.stack([g.float().square().sum() for g in s["grads"]])
    norm = squares.sum().sqrt()
    factor = torch.where(torch.isfinite(norm), (s["case"]["max_norm"] / (norm + EPS)).clamp(max=1.0), 1.0)
    [o.copy_(g.float() * factor) for g, o in zip(s["grads"], s["outs"])]
    return {"norm": norm, "out": s["flat"]}


def _chunk(time):
    return 64 if time <= 8192 else 128 if time <= 32768 else 256


def _plain_step(s):
    live, keep = s["marks"], torch.exp(s["log_decay"])[:, None, None]
    k, v, state = s["k"].float(), s["v"].float(), s["state"]
    if live is not None:
        m = live[:, None, None, None]
        keep = torch.where(m == 0, 1.0, torch.where(m == 2, 0.0, keep))
        k, v = torch.where(m[..., 0] == 0, 0.0, k), torch.where(m[..., 0] == 0, 0.0, v)
    state.mul_(keep).add_(k[..., None] * v[..., None, :])
    o = s["scale"] * (s["q"].float()[..., None, :] @ state)[..., 0, :]
    return {"o": o.to(s["q"].dtype), "state": state}


def _plain_attend(s):
    b, t, h = s["q"].shape[:3]
    size = min(t, _chunk(t))
    n = -(-t // size)
    marks = s["marks"]
    part = lambda x: torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, n * size - t)).view(b, n, size, h, -1).permute(0, 3, 1, 2, 4)  # noqa: E731
    whole = lambda x: x.permute(0, 2, 3, 1, 4).reshape(b, n * size, h, -1)[:, :t].to(s["q"].dtype)  # noqa: E731
    q, k, v = part(s["q"]), part(s["k"]), part(s["v"])
    steps = torch.ones(b, n * size, device="cuda")
    steps[:, t:] = 0
    first = torch.zeros_like(steps)
    if marks is not None:
        steps[:, :t] = (marks != 0).float()
        first[:, :t] = (marks == 2).float()
        gone = (steps == 0).view(b, 1, n, size, 1)
        k, v = torch.where(gone, 0.0, k), torch.where(gone, 0.0, v)
    # samples seen and traces begun up to each step, and up to each chunk's start
    seen, trace = steps.cumsum(1), first.cumsum(1)
    starts = lambda x: torch.cat((torch.zeros_like(x[:, :1]), x[:, size - 1::size]), 1)  # noqa: E731
    seen0, trace0 = starts(seen), starts(trace)
    seen, trace = seen.view(b, n, size), trace.view(b, n, size)
    g = s["log_decay"]

    def decay(late, early, late_trace, early_trace):
        """What is left at `late` of what came in at `early`: [batch, heads, ...]."""
        gap = (late - early)[:, None]
        left = torch.exp(g.view(1, h, *[1] * (gap.dim() - 2)) * gap)
        return torch.where(((gap >= 0) & (late_trace == early_trace)[:, None]), left, 0.0)

    inner = decay(seen[..., :, None], seen[..., None, :], trace[..., :, None], trace[..., None, :]).tril()
    row = decay(seen, seen0[:, :-1, None], trace, trace0[:, :-1, None])[..., None]
    column = decay(seen0[:, 1:, None], seen, trace0[:, 1:, None], trace)[..., None]
    chain = decay(seen0[:, :, None], seen0[:, None], trace0[:, :, None], trace0[:, None]).tril()

    def along(chain, parts):
        return (chain @ parts.flatten(3)).view_as(parts)

    state = s["state"][:, :, None]
    states = along(chain, torch.cat((state, (k * column).mT @ v), 2))
    o = s["scale"] * ((inner * (q @ k.mT)) @ v + row * (q @ states[:, :, :-1]))
    out = {"o": whole(o), "last": states[:, :, -1].clone()}
    if s["case"]["mode"] == "forward":
        return out
    do = part(s["do"])
    back = along(chain.mT, torch.cat((s["scale"] * (q * row).mT @ do, s["dlast"][:, :, None]), 2))
    weights = s["scale"] * inner
    dp = weights * (do @ v.mT)
    out["dq"] = whole(dp @ k + s["scale"] * row * (do @ states[:, :, :-1].mT))
    out["dk"] = whole(dp.mT @ q + column * (v @ back[:, :, 1:].mT))
    out["dv"] = whole((weights * (q @ k.mT)).mT @ do + column * (k @ back[:, :, 1:]))
    out["dstate"] = back[:, :, 0].clone()
    return out


def run(state):
    s, case = state, state["case"]
    if not own:
        if case["op"] == "embed":
            return _plain_embed(s)
        if case["op"] == "clip":
            return _plain_clip(s)
        return _plain_step(s) if case["mode"] == "step" else _plain_attend(s)
    from paper_2609_02109_gb300 import mf

    if case["op"] == "embed":
        out = {"out": mf.embedding(s["table"], s["ids"], s["scale"])}
        if case["train"]:
            out["dtable"] = mf.embedding_backward(s["dout"], s["ids"], case["rows"], s["scale"])
        return out
    if case["op"] == "clip":
        return {"norm": mf.clip_gradients(s["grads"], case["max_norm"], eps=EPS, out=s["outs"]), "out": s["flat"]}
    if case["mode"] == "step":
        o = mf.linear_attention_step(s["q"], s["k"], s["v"], s["log_decay"], s["state"], s["marks"], s["scale"])
        return {"o": o, "state": s["state"]}
    if case["mode"] == "forward":
        o, last = mf.linear_attention(s["q"], s["k"], s["v"], s["log_decay"], s["state"], s["marks"], s["scale"])
        return {"o": o, "last": last}
    o, last, saved = mf.linear_attention(s["q"], s["k"], s["v"], s["log_decay"], s["state"], s["marks"], s["scale"], save=True)
    dq, dk, dv, dstate = mf.linear_attention_backward(s["do"], s["q"], s["k"], s["v"], s["log_decay"], saved, s["dlast"],
                                                      s["marks"], s["scale"])
    return {"o": o, "last": last, "dq": dq, "dk": dk, "dv": dv, "dstate": dstate}


def work(case):
    if case["op"] == "clip":
        values = sum(_sizes(case))
        size = sum(n * t.itemsize for n, t in zip(_sizes(case), _types(case)))
        return {"bytes": 2 * size + 4, "flops": 3 * values}
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "embed":
        # rows that no token names are not read; the gradient of every row is written
        n, d, r = case["tokens"], case["dim"], case["rows"]
        share = torch.log1p(1.0 / torch.arange(1, r + 1, dtype=torch.float64)) / math.log(r + 1.0)
        used = float(-torch.expm1(-n * share).sum())
        forward = size * d * (used + n) + 8 * n
        return {"bytes": forward + (size * d * (n + r) + 8 * n if case["train"] else 0), "flops": n * d * (2 if case["train"] else 1)}
    b, t, h, dk, dv = (case[x] for x in ("batch", "time", "heads", "dk", "dv"))
    rows, state = b * t * h, 4 * b * h * dk * dv
    forward = size * rows * 2 * (dk + dv) + 2 * state + b * t * bool(case["marks"])
    if case["mode"] != "train":
        return {"bytes": forward, "flops": rows * 5 * dk * dv}
    # backward, after the rest of a network has run: q, k, v and the output's gradient -> dq, dk, dv
    backward = size * rows * (4 * dk + 3 * dv) + 2 * state + b * t * bool(case["marks"])
    return {"bytes": forward + backward, "flops": rows * 17 * dk * dv}


def _exact_attend(s):
    """The state step by step, forward and back."""
    case = s["case"]
    step = case["mode"] == "step"
    q, k, v = ((x[:, None] if step else x).double() for x in (s["q"], s["k"], s["v"]))
    t = q.shape[1]
    keep = torch.exp(s["log_decay"].double())[None, None].expand(q.shape[:3])
    if s["marks"] is not None:
        marks = (s["marks"][:, None] if step else s["marks"])[..., None]
        keep = torch.where(marks == 0, 1.0, torch.where(marks == 2, 0.0, keep))
        gone = (marks == 0)[..., None]
        k, v = k.masked_fill(gone, 0.0), v.masked_fill(gone, 0.0)
    keep = keep[..., None, None]
    train = case["mode"] == "train"
    do = s["do"].double() * s["scale"] if train else None
    state = s["state"].double()
    o, dq = torch.empty_like(v), torch.empty_like(q)
    for i in range(t):
        state = torch.addcmul(k[:, i, :, :, None] * v[:, i, :, None], state, keep[:, i])
        torch.matmul(q[:, i, :, None], state, out=o[:, i, :, None])
        if train:
            torch.matmul(do[:, i, :, None], state.mT, out=dq[:, i, :, None])
    o *= s["scale"]
    if step:
        return {"o": o[:, 0], "state": state}
    out = {"o": o, "last": state}
    if train:
        back = s["dlast"].double()
        dk, dv = torch.empty_like(k), torch.empty_like(v)
        for i in reversed(range(t)):
            back = back + q[:, i, :, :, None] * do[:, i, :, None]
            torch.matmul(v[:, i, :, None], back.mT, out=dk[:, i, :, None])
            torch.matmul(k[:, i, :, None], back, out=dv[:, i, :, None])
            back = back * keep[:, i]
        out.update(dq=dq, dk=dk, dv=dv, dstate=back)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(s)
    if case["op"] == "clip":
        norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in s["grads"]))
        factor = min(1.0, case["max_norm"] / (norm + EPS))
        flat, outs = _views(_sizes(case), _types(case), lambda n, t: torch.empty(n, device="cuda", dtype=torch.float64))
        for g, o in zip(s["grads"], outs):
            o.copy_(g).mul_(factor)
        return {"norm": torch.tensor(norm, dtype=torch.float64), "out": flat}
    ids, table = s["ids"], s["table"].double()
    used = torch.nonzero(ids >= 0)[:, 0]
    out = torch.zeros(ids.shape[0], case["dim"], device="cuda", dtype=torch.float64)
    out[used] = s["scale"] * table[ids[used]]
    if not case["train"]:
        return {"out": out}
    total = torch.zeros_like(table)
    for at in used.split(8192):
        total.index_put_((ids[at],), s["dout"][at].double(), accumulate=True)
    return {"out": out, "dtable": s["scale"] * total}
