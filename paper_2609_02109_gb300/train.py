"""Fits the predictors of a problem to a monitor's trace, and learns the state that they see.

The paper trains one predictor per model on (local configuration, observed state) offline and leaves how the
runtime monitor smooths its samples open (Sec. III-A, III-B, Eq. 2, Eq. 6).  Here a trace of raw aggregate
samples (summed SM share, VRAM, bandwidth, N, scaled as the predictors see them) passes through the gated linear
recurrence, whose gates say how long each component is remembered and are learned with the predictors; the hidden
layers of all predictors are updated as one batch by their orthogonalised momentum.  ``fit`` returns weights in
the layout of ``prob["weights"]``, ready for ``mf.Context``.

    python -m paper_2609_02109_gb300.train       # a small synthetic run: loss, learned memories, a search
"""
from __future__ import annotations

import numpy as np
import torch
from torch.autograd.function import once_differentiable

from . import mf, workload


class _Recurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, z, h0, marks):
        h, last, saved = mf.recurrence(x, z, h0, marks, save=True)
        ctx.save_for_backward(x, z, saved, marks)
        ctx.has_h0 = h0 is not None
        return h, last

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, dlast):
        x, z, saved, marks = ctx.saved_tensors
        if dh.stride(-1) != 1 and dh.shape[-1] > 1:
            dh = dh.contiguous()
        dx, dz, dh0 = mf.recurrence_backward(dh, x, z, saved, None if dlast is None else dlast.contiguous(), marks)
        return dx, dz, dh0 if ctx.has_h0 else None, None


def recurrence(x, z, h0=None, marks=None):
    """mf.recurrence with gradients for x, z and h0: (h, last state).  (First derivatives: a second one raises.)"""
    return _Recurrence.apply(x, z, h0, marks)


class Muon:
    """Momentum whose update is orthogonalised, for tensors [..., rows, cols]: u = g + beta m (Nesterov's form) with
    m = beta m + g, then w -= lr sqrt(max(1, rows / cols)) orthogonalize(u)."""

    def __init__(self, params, lr: float = 0.02, beta: float = 0.95, steps: int = 5):
        self.params, self.lr, self.beta, self.steps = list(params), lr, beta, steps
        self.buffers = [torch.zeros_like(p) for p in self.params]

    @torch.no_grad()
    def step(self) -> None:
        for p, m in zip(self.params, self.buffers):
            if p.grad is None:  # (not part of this step's loss)
                continue
            m.mul_(self.beta).add_(p.grad)
            u = mf.orthogonalize(torch.add(p.grad, m, alpha=self.beta), steps=self.steps)
            p.sub_(u, alpha=self.lr * max(1.0, p.shape[-2] / p.shape[-1]) ** 0.5)

    def zero_grad(self) -> None:
        for p in self.params:
            p.grad = None


class Predictors:
    """The N predictors of a problem as batched float32 parameters [N, out, in] (Eq. 6; two hidden layers)."""

    def __init__(self, prob: dict, device="cuda"):
        n, d, h1, h2 = len(prob["n_options"]), prob["d_local"] + 4, prob["hidden1"], prob["hidden2"]
        if h2 < 1:
            raise ValueError("Predictors wants two hidden layers")
        flat = torch.as_tensor(prob["weights"], device=device).view(n, -1)
        shapes = ((h1, d), (h1,), (h2, h1), (h2,), (2, h2), (2,))
        parts = flat.split([int(np.prod(s)) for s in shapes], 1)
        self.w = [p.reshape(n, *s).clone().requires_grad_(True) for p, s in zip(parts, shapes)]

    def __call__(self, inputs: torch.Tensor) -> torch.Tensor:
        """inputs [N, samples, d_local + 4] -> (thr, lat) [N, samples, 2]."""
        w1, b1, w2, b2, w3, b3 = self.w
        h = torch.relu(torch.baddbmm(b1[:, None], inputs, w1.mT))
        h = torch.relu(torch.baddbmm(b2[:, None], h, w2.mT))
        return torch.baddbmm(b3[:, None], h, w3.mT)

    def packed(self) -> np.ndarray:
        """The weights in the layout of prob["weights"]."""
        return torch.cat([p.detach().flatten(1) for p in self.w], 1).flatten().cpu().numpy()


def synthetic_trace(prob: dict, traces: int, time: int, seed: int, device="cuda") -> dict:
    """Traces of a monitor in front of the problem's own predictors: the true state is a running mean of what
    runs (memories of about 8, 20, 50 and 150 samples), the monitor sees each sample with noise and misses one in
    20 (NaN); at random times model i runs option o_i and its throughput and latency are observed."""
    g = torch.Generator(device=device).manual_seed(seed)
    n = len(prob["n_options"])
    raw = torch.rand(traces, time, 4, device=device, generator=g)
    raw = 0.5 + 0.5 * torch.sin(torch.cumsum(raw - 0.5, 1))
    memory = torch.tensor([8.0, 20.0, 50.0, 150.0], device=device)
    state, _ = mf.recurrence(raw, torch.log(memory - 1).expand(traces, time, 4))
    seen = raw + 0.05 * torch.randn(raw.shape, device=device, generator=g)
    marks = (torch.rand(traces, time, device=device, generator=g) >= 0.05).to(torch.uint8)
    seen.masked_fill_((marks == mf.MARK_MISSING)[..., None], float("nan"))
    samples = traces * time // 8
    at = torch.randint(traces * time, (samples,), device=device, generator=g)
    first = np.concatenate([[0], np.cumsum(prob["n_options"])[:-1]])
    feats = torch.as_tensor(prob["local_feats"], device=device)
    rows = torch.stack([int(first[i]) + torch.randint(int(k), (samples,), device=device, generator=g)
                        for i, k in enumerate(prob["n_options"])])
    teacher = Predictors(prob, device)
    with torch.no_grad():
        inputs = torch.cat((feats[rows], state.reshape(-1, 4)[at].expand(n, samples, 4)), 2)
        target = teacher(inputs)
    return {"seen": seen, "marks": marks, "at": at, "rows": rows, "target": target, "memory": memory}


def fit(prob: dict, trace: dict, steps: int = 100, lr: float = 0.01, seed: int = 1) -> dict:
    """Fits new predictors and the state's gates to a trace (as of synthetic_trace).

    Returns weights (as prob["weights"]), the learned memories in samples, the last state of every trace, and the loss
    of every step."""
    device = trace["seen"].device
    start = dict(prob, weights=np.concatenate([
        workload.draw_weights(seed + 1000, i, prob["d_local"], prob["hidden1"], prob["hidden2"])
        for i in range(len(prob["n_options"]))]))
    net = Predictors(start, device)
    hidden, others = [net.w[0], net.w[2]], [net.w[1], net.w[3], net.w[4], net.w[5]]
    gates = torch.full((4,), 3.0, device=device, requires_grad=True)
    muon = Muon(hidden, lr=lr)
    rest = torch.optim.Adam([{"params": others, "lr": lr}, {"params": [gates], "lr": 5 * lr}])
    feats = torch.as_tensor(prob["local_feats"], device=device)[trace["rows"]]
    n, samples = trace["rows"].shape
    losses = []
    for _ in range(steps):
        state, _ = recurrence(trace["seen"], gates.expand(trace["seen"].shape), None, trace["marks"])
        inputs = torch.cat((feats, state.reshape(-1, 4)[trace["at"]].expand(n, samples, 4)), 2)
        loss = torch.nn.functional.mse_loss(net(inputs), trace["target"])
        muon.zero_grad()
        rest.zero_grad()
        loss.backward()
        muon.step()
        rest.step()
        losses.append(loss.detach())
    with torch.no_grad():  # the state that the learned gates make of the traces
        _, last = mf.recurrence(trace["seen"], gates.expand(trace["seen"].shape), None, trace["marks"])
    return {"weights": net.packed(), "memory": 1 + torch.exp(gates.detach()), "state": last,
            "loss": torch.stack(losses).cpu().numpy() if losses else np.zeros(0, np.float32)}


def main() -> None:
    prob = workload.paper_scale()
    trace = synthetic_trace(prob, 4, 4096, seed=7)
    got = fit(prob, trace)
    print(f"loss {got['loss'][0]:.4f} -> {got['loss'][-1]:.5f} in {len(got['loss'])} steps; memories "
          f"{[round(float(v), 1) for v in got['memory']]} samples (true: {[float(v) for v in trace['memory']]})")
    for name, weights in (("true predictors", prob["weights"]), ("fitted", got["weights"])):
        with mf.Context(dict(prob, weights=weights)) as ctx:
            res = ctx.search(8)
        print(f"{name}: best configuration {res['best_idx']}, J = {res['best_score']:.4f}, {res['count']} feasible")


if __name__ == "__main__":
    main()
