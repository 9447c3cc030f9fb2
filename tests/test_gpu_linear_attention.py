"""Linear attention on the GPU against the 64-bit steps, with derived bounds (tests/_attend_ref.py)."""
import numpy as np
import pytest

import _attend_ref as A

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


def kinds():
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


class Case:
    def __init__(self, kind, b, t, h, dk, dv, seed=0, marks="none", state=True, fast=1.0, layout="bthd", scale=0.7):
        import torch
        r = np.random.default_rng(seed + 1000 * t + dk)
        dt = kinds()[kind]
        self.kind, self.scale = kind, scale

        def seq(d):
            x = torch.tensor(r.standard_normal((b, t, h, d)), dtype=torch.float32).to(dt)
            if layout == "bhtd":
                return x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
            if layout == "padded":  # rows inside a wider tensor, at an odd offset
                wide = torch.zeros(b, t, h, d + 5, dtype=dt).cuda()
                wide[..., 3:3 + d] = x.cuda()
                return wide[..., 3:3 + d]
            if layout == "shared":  # one head, read by all
                return x[:, :, :1].cuda().expand(b, t, h, d)
            return x.cuda()

        self.q, self.k, self.v, self.do = seq(dk), seq(dk), seq(dv), seq(dv)
        # memories from one sample to a thousand
        memory = np.exp(r.uniform(0, np.log(1000.0) * fast, h))
        self.decay = torch.tensor(-1.0 / memory, dtype=torch.float32).cuda()
        self.state = torch.tensor(r.standard_normal((b, h, dk, dv)), dtype=torch.float32).cuda() if state else None
        self.dlast = torch.tensor(r.standard_normal((b, h, dk, dv)), dtype=torch.float32).cuda() if state else None
        self.marks = None
        if marks != "none":
            m = r.choice([0, 1, 2], (b, t), p={"some": [0.2, 0.77, 0.03], "missing": [1, 0, 0], "first": [0.3, 0, 0.7]}[marks])
            if marks == "some" and t > 128:
                m[0, :130] = 0          # a chunk without a sample
                m[-1, [31, 32, 127, 128]] = 2
            self.marks = torch.tensor(m.astype(np.uint8)).cuda()
            gone = (self.marks == 0)[..., None, None].expand_as(self.k)
            if layout != "shared":
                self.k[gone] = float("nan")
                self.v[(self.marks == 0)[..., None, None].expand_as(self.v)] = float("inf")

    def host(self):
        d = lambda x: None if x is None else x.double().cpu().numpy()  # noqa: E731
        k, v = d(self.k), d(self.v)
        marks = None if self.marks is None else self.marks.cpu().numpy()
        return d(self.q), k, v, d(self.decay), d(self.state), marks, float(np.float32(self.scale))

    def check(self, mf, grad=True):
        import torch
        args = (self.q, self.k, self.v, self.decay, self.state, self.marks, self.scale)
        o, last, saved = mf.linear_attention(*args, save=True)
        d = lambda x: x.double().cpu().numpy()  # noqa: E731
        host = self.host()
        want = A.attend(*host)
        bounds = A.attend_bounds(self.kind, None, None, *host)
        for name, got, exact, bound in zip(("o", "last"), (o, last), want, bounds):
            off = np.abs(d(got) - exact)
            assert got.shape == exact.shape and (off <= bound).all(), (name, (off / bound).max())
        plain = mf.linear_attention(*args)
        assert plain[0].equal(o) and plain[1].equal(last)
        if not grad:
            return
        got = mf.linear_attention_backward(self.do, self.q, self.k, self.v, self.decay, saved, self.dlast, self.marks, self.scale)
        dl = None if self.dlast is None else d(self.dlast)
        want = A.attend_grad(d(self.do), dl, *host)
        bounds = A.attend_bounds(self.kind, d(self.do), dl, *host)
        for name, g, exact, bound in zip(("dq", "dk", "dv", "dstate"), got, want, bounds):
            off = np.abs(d(g) - exact)
            if self.kind == "f16" and name != "dstate":
                # from 65520 on, halfway between the largest half and the next power of two, a value rounds to infinity
                beyond = (np.abs(exact) + bound >= 65520) & np.isinf(d(g)) & (np.sign(d(g)) == np.sign(exact))
                off[beyond] = 0
            assert g.shape == exact.shape and (off <= bound).all(), (name, (off / bound).max())
        again = mf.linear_attention_backward(self.do, self.q, self.k, self.v, self.decay, saved, self.dlast, self.marks, self.scale)
        assert all(x.equal(y) for x, y in zip(got, again))
        assert mf.check_operators() == mf.MF_OK
        torch.cuda.synchronize()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("t", [0, 1, 2, 8, 9, 31, 32, 33, 64, 127, 128, 129, 257, 700])
def test_lengths(mf, kind, t):
    Case(kind, 2, t, 3, 24, 20, marks="some").check(mf)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("t", [9, 19, 39, 40, 79])
@pytest.mark.parametrize("dk,dv", [(64, 64), (128, 72), (40, 24)])
def test_lengths_of_wide_heads(mf, kind, t, dk, dv):
    """On both sides of where chunks on the tensor cores take over from steps."""
    Case(kind, 2, t, 3, dk, dv, marks="some").check(mf)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(1, 1), (3, 7), (8, 8), (16, 64), (64, 16), (65, 64), (64, 64), (100, 72), (128, 1), (127, 128), (128, 128)])
def test_widths(mf, kind, dk, dv):
    Case(kind, 1, 200, 2, dk, dv).check(mf)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(5, 9), (128, 128), (64, 64)])
@pytest.mark.parametrize("marks", ["none", "some", "missing", "first"])
@pytest.mark.parametrize("state", [False, True])
def test_marks_and_states(mf, kind, dk, dv, marks, state):
    Case(kind, 2, 300, 2, dk, dv, marks=marks, state=state).check(mf)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", ["bhtd", "padded", "shared"])
@pytest.mark.parametrize("dk,dv", [(16, 16), (128, 64)])
def test_layouts(mf, kind, layout, dk, dv):
    Case(kind, 2, 150, 3, dk, dv, layout=layout, marks="none").check(mf)
    if layout != "shared":
        Case(kind, 2, 150, 3, dk, dv, layout=layout, marks="some").check(mf)


@pytest.mark.parametrize("kind,dk,dv,t", [("f32", 16, 16, 9000), ("bf16", 64, 64, 9000), ("f16", 128, 128, 5000), ("f32", 100, 40, 3000),
                                          ("bf16", 128, 128, 4100)])
def test_long_traces_that_are_split(mf, kind, dk, dv, t):
    c = Case(kind, 1, t, 2, dk, dv, marks="some")
    c.check(mf)
    saved = mf.linear_attention(c.q, c.k, c.v, c.decay, c.state, c.marks, c.scale, save=True)[2]
    assert saved.numel() > 2 * dk * dv  # several segments


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("decay", [0.0, -float("inf"), -40.0, -1e-7, 0.01])
@pytest.mark.parametrize("t", [5, 300])
def test_decays(mf, kind, decay, t):
    c = Case(kind, 1, t, 2, 16, 16, marks="some")
    c.decay.fill_(decay)
    c.check(mf)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(8, 8), (128, 128), (20, 33)])
def test_steps_are_the_sequence(mf, kind, dk, dv):
    """Single tokens one after the other, the state in place: the bounds of a sequence, and the states' bits equal to
    what the forward call makes of the same step."""
    import torch
    c = Case(kind, 3, 12, 2, dk, dv, marks="some")
    state, outs = c.state.clone(), []
    for i in range(12):
        before = state.clone()
        outs.append(mf.linear_attention_step(c.q[:, i], c.k[:, i], c.v[:, i], c.decay, state, c.marks[:, i], c.scale))
        one, last = mf.linear_attention(c.q[:, i:i + 1], c.k[:, i:i + 1], c.v[:, i:i + 1], c.decay, before, c.marks[:, i:i + 1], c.scale)
        assert one[:, 0].equal(outs[-1]) and last.equal(state)
        still = c.marks[:, i] == 0
        assert state[still].equal(before[still])
    host = c.host()
    want, bounds = A.attend(*host), A.attend_bounds(kind, None, None, *host)
    assert (np.abs(torch.stack(outs, 1).double().cpu().numpy() - want[0]) <= bounds[0]).all()
    assert (np.abs(state.double().cpu().numpy() - want[1]) <= bounds[1]).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(16, 24), (128, 128)])
@pytest.mark.parametrize("where", ["q", "k", "v", "do"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_where_it_belongs(mf, kind, dk, dv, where, value):
    """Results that depend on the value are not finite, results that do not are as without it, bit for bit."""
    import torch
    t, at = 400, 150
    c = Case(kind, 1, t, 2, dk, dv, state=True)
    c.decay.fill_(-0.01)
    c.marks = torch.ones(1, t, dtype=torch.uint8, device="cuda")
    c.marks[0, 200] = 2   # what is before ends here

    def run():
        o, last, saved = mf.linear_attention(c.q, c.k, c.v, c.decay, c.state, c.marks, c.scale, save=True)
        return (o, last, *mf.linear_attention_backward(c.do, c.q, c.k, c.v, c.decay, saved, c.dlast, c.marks, c.scale))

    clean = [x.clone() for x in run()]
    column = dk // 2 if where in "qk" else dv // 2
    getattr(c, where)[0, at, 1, column] = value
    o, last, dq, dkey, dvalue, dstate = run()
    touched = {}
    before, inside = slice(0, at + 1), slice(at, 200)
    every = slice(None)
    # (tensor, time, columns) that depend on the value; head 1 only
    if where == "q":
        touched = {"o": (slice(at, at + 1), every), "dk": (before, slice(column, column + 1)), "dv": (before, every)}
    elif where == "k":
        touched = {"o": (inside, every), "dq": (inside, slice(column, column + 1)), "dv": (slice(at, at + 1), every)}
    elif where == "v":
        touched = {"o": (inside, slice(column, column + 1)), "dq": (inside, every), "dk": (slice(at, at + 1), every)}
    else:
        touched = {"dq": (slice(at, at + 1), every), "dk": (before, every), "dv": (before, slice(column, column + 1))}
    for name, got, was in (("o", o, clean[0]), ("dq", dq, clean[2]), ("dk", dkey, clean[3]), ("dv", dvalue, clean[4])):
        mask = torch.zeros_like(got, dtype=torch.bool)
        if name in touched:
            times, columns = touched[name]
            mask[0, times, 1, columns] = True
        assert not torch.isfinite(got[mask]).any(), name
        assert torch.isfinite(got[~mask]).all(), name
        # (a part of bf16's sums is scaled by what its chunk holds, so that some results are rounded otherwise)
        assert got[~mask].equal(was[~mask]) or kind != "f32", name
    assert last.equal(clean[1]) if kind == "f32" else torch.isfinite(last).all()
    if where in ("q", "do"):
        mask = torch.zeros_like(dstate, dtype=torch.bool)
        mask[0, 1, column if where == "q" else every, column if where == "do" else every] = True
        assert not torch.isfinite(dstate[mask]).any() and torch.isfinite(dstate[~mask]).all()
    else:
        assert torch.isfinite(dstate).all()


def test_extreme_values(mf):
    """Rows of very large and very small values, whose products are ordinary: no overflow on the way."""
    import torch
    for kind, big in (("f32", 1e12), ("bf16", 1e12), ("f16", 2000.0)):
        c = Case(kind, 1, 300, 2, 64, 64, state=True)
        c.q /= big
        c.k *= big
        c.check(mf)
        c = Case(kind, 1, 300, 2, 128, 128, state=False)
        c.v *= big
        c.v[:, ::3] /= big * (1.0 if kind == "f16" else big)
        c.do /= 10.0
        c.q /= 100.0
        c.check(mf)


def test_on_another_stream_and_captured(mf):
    """On a stream of its own and in a graph, replayed on new values, with a graph of a call that shares the pool."""
    import torch
    c = Case("bf16", 2, 500, 2, 64, 64, marks="some")
    want = mf.linear_attention(c.q, c.k, c.v, c.decay, c.state, c.marks, c.scale)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = mf.linear_attention(c.q, c.k, c.v, c.decay, c.state, c.marks, c.scale)
    s.synchronize()
    assert all(x.equal(y) for x, y in zip(got, want))
    graphs, outs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()], []
    for g in graphs:
        with torch.cuda.graph(g, pool=graphs[0].pool() if outs else None):
            o, last, saved = mf.linear_attention(c.q, c.k, c.v, c.decay, c.state, c.marks, c.scale, save=True)
            outs.append((o, last, *mf.linear_attention_backward(c.do, c.q, c.k, c.v, c.decay, saved, c.dlast, c.marks, c.scale)))
    other = Case("bf16", 2, 500, 2, 64, 64, seed=9, marks="some")
    for n in ("q", "k", "v", "do", "state", "dlast", "marks"):
        getattr(c, n).copy_(getattr(other, n))
    o, last, saved = mf.linear_attention(c.q, c.k, c.v, c.decay, c.state, c.marks, c.scale, save=True)
    want = (o, last, *mf.linear_attention_backward(c.do, c.q, c.k, c.v, c.decay, saved, c.dlast, c.marks, c.scale))
    for g, out in zip(graphs, outs):
        g.replay()
        torch.cuda.synchronize()
        assert all(x.equal(y) for x, y in zip(out, want))


def test_many_heads_of_short_sequences(mf):
    """More rows than blocks of a launch run at a time."""
    for kind in ("f32", "bf16"):
        Case(kind, 70, 40, 30, 8, 12, marks="some").check(mf)
    Case("f32", 3000, 1, 30, 4, 4, marks="some").check(mf, grad=False)


def test_binding_refuses(mf):
    import torch
    c = Case("f32", 1, 4, 2, 8, 8)
    call = lambda **kw: mf.linear_attention(**{**dict(q=c.q, k=c.k, v=c.v, log_decay=c.decay, state=c.state), **kw})  # noqa: E731
    for kw in (dict(q=c.q.cpu()), dict(q=c.q.double()), dict(q=c.q[0]), dict(k=c.k.half()), dict(k=c.k[:, :, :, :4]),
               dict(v=c.v[:, :2]), dict(v=c.v.mT), dict(log_decay=None), dict(log_decay=c.decay[:1]), dict(log_decay=c.decay.double()),
               dict(state=c.state.half()), dict(state=c.state.mT), dict(state=c.state[:, :1]),
               dict(marks=torch.ones(1, 4, device="cuda")), dict(marks=torch.ones(1, 3, dtype=torch.uint8, device="cuda")),
               dict(scale=float("nan")), dict(q=torch.zeros(1, 4, 2, 129, device="cuda"), k=torch.zeros(1, 4, 2, 129, device="cuda"))):
        with pytest.raises(mf.MFError) as e:
            call(**kw)
        assert e.value.status == mf.MF_EINVAL
    step = lambda **kw: mf.linear_attention_step(**{**dict(q=c.q[:, 0], k=c.k[:, 0], v=c.v[:, 0], log_decay=c.decay, state=c.state), **kw})  # noqa: E731
    for kw in (dict(state=None), dict(q=c.q), dict(state=c.state.clone().requires_grad_()), dict(marks=torch.ones(2, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(mf.MFError):
            step(**kw)
    saved = mf.linear_attention(c.q, c.k, c.v, c.decay, save=True)[2]
    for kw in (dict(saved=None), dict(saved=saved[:-1]), dict(do=c.do[:, :2]), dict(dlast=c.state.half())):
        with pytest.raises(mf.MFError):
            mf.linear_attention_backward(**{**dict(do=c.do, q=c.q, k=c.k, v=c.v, log_decay=c.decay, saved=saved), **kw})


@pytest.mark.parametrize("shape", [(0, 5, 2, 4, 4), (2, 5, 0, 4, 4), (2, 0, 2, 4, 4), (2, 5, 2, 0, 4), (2, 5, 2, 4, 0), (2, 40, 2, 0, 4), (2, 40, 2, 4, 0)])
def test_sizes_of_zero(mf, shape):
    b, t, h, dk, dv = shape
    for kind in ("f32", "bf16"):
        Case(kind, b, t, h, dk, dv).check(mf)


def test_waits_that_run_out_are_told():
    """The tensor-core passes' bounded waits, made to give up: the status says so, and the next call is as ever."""
    import torch
    from paper_2609_02109_gb300 import mf
    c = Case("bf16", 1, 1000, 2, 128, 128)
    args = (c.q, c.k, c.v, c.decay, c.state, None, c.scale)
    want = mf.linear_attention(*args)
    mf.debug_operators_wait_test(2)
    try:
        mf.linear_attention(*args)
    finally:
        mf.debug_operators_wait_test(0)
    assert mf.check_operators() == mf.MF_ETIMEOUT
    got = mf.linear_attention(*args)
    torch.cuda.synchronize()
    assert mf.check_operators() == mf.MF_OK and all(x.equal(y) for x, y in zip(got, want))
