"""Linear attention on every way that operands take: whatever the strides and alignment, the bits are equal; two threads."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


def laid_out(x, pad, at):
    """The same values inside rows that are `pad` wider, from column `at` on."""
    import torch
    b, t, h, d = x.shape
    wide = torch.full((b, t, h, d + pad), 7.0, dtype=x.dtype, device="cuda")
    wide[..., at:at + d] = x
    return wide[..., at:at + d]


def by_heads(x):
    """The same values, heads before time."""
    return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)


def run(mf, q, k, v, do, decay, state, marks):
    o, last, saved = mf.linear_attention(q, k, v, decay, state, marks, 0.3, save=True)
    return (o, last, *mf.linear_attention_backward(do, q, k, v, decay, saved, state, marks, 0.3))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dk,dv", [(8, 8), (16, 32), (32, 16), (24, 20), (32, 48), (64, 64), (128, 64), (64, 128), (72, 104), (100, 40), (128, 128)])
@pytest.mark.parametrize("b,t,h", [(2, 300, 2), (1, 2000, 1)])
def test_layouts_give_equal_bits(mf, kind, dk, dv, b, t, h):
    import torch
    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[kind]
    g = torch.Generator(device="cuda").manual_seed(dk + 7 * dv)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, k, v, do = (normal(b, t, h, d).to(dt) for d in (dk, dk, dv, dv))
    decay, state = -torch.rand(h, device="cuda", generator=g) / 10, normal(b, h, dk, dv)
    marks = (torch.rand(b, t, device="cuda", generator=g) > 0.1).to(torch.uint8)
    marks[:, t // 2] = 2
    want = run(mf, q, k, v, do, decay, state, marks)
    for change in (by_heads, lambda x: laid_out(x, 16 - x.shape[3] % 8, 8), lambda x: laid_out(x, 12 - x.shape[3] % 4, 4),
                   lambda x: laid_out(x, 3, 1)):
        got = run(mf, *map(change, (q, k, v, do)), decay, state, marks.t().contiguous().t())
        assert all(x.equal(y) for x, y in zip(got, want))
    assert mf.check_operators() == mf.MF_OK


def test_results_next_to_others_stay_as_they_are(mf):
    """Through the C ABI: results into rows of a wider tensor, on every width of stores."""
    import ctypes as C
    import torch
    for dt, kind in ((torch.bfloat16, 1), (torch.float16, 2), (torch.float32, 0)):
        for dk, dv, pad in ((64, 72, 8), (64, 72, 4), (64, 72, 3), (16, 12, 5)):
            b, t, h = 2, 200, 3
            g = torch.Generator(device="cuda").manual_seed(3)
            q, k, v = (torch.randn(b, t, h, d, device="cuda", generator=g).to(dt) for d in (dk, dk, dv))
            decay = torch.tensor([-0.1, -0.01, 0.0], device="cuda")
            want, _ = mf.linear_attention(q, k, v, decay)
            wide = torch.full((b, t + 1, h, dv + pad), 9.0, dtype=dt, device="cuda")
            heads = lambda x, n: mf._Heads(x.data_ptr(), *x.stride()[:3])  # noqa: E731
            p = mf._LinearAttention(type=kind, batch=b, time=t, heads=h, dim_k=dk, dim_v=dv, q=heads(q, dk), k=heads(k, dk), v=heads(v, dv),
                                    d_log_decay=decay.data_ptr(), d_state=None, d_marks=None, scale=1.0, o=heads(wide, dv), d_last=None,
                                    d_saved=None, d_status=None)
            need = C.c_uint64()
            assert mf.lib().mf_linear_attention_sizes(kind, b, t, h, dk, dv, None, C.byref(need), None) == mf.MF_OK
            work = torch.empty(need.value + 16, dtype=torch.uint8, device="cuda")
            assert mf.lib().mf_linear_attention_forward(C.byref(p), work.data_ptr(), need.value, None) == mf.MF_OK
            torch.cuda.synchronize()
            assert wide[:, :t, :, :dv].equal(want)
            assert (wide[:, t] == 9).all() and (wide[..., dv:] == 9).all()


def test_two_threads_at_once(mf):
    import threading
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    cases = []
    for dt in (torch.bfloat16, torch.float32):
        q, k, v = (torch.randn(1, 3000, 2, 128, device="cuda", generator=g).to(dt) for _ in range(3))
        decay = torch.tensor([-0.1, -0.01], device="cuda")
        cases.append((q, k, v, decay, mf.linear_attention(q, k, v, decay)))
    torch.cuda.synchronize()
    bad = []

    def work(case):
        q, k, v, decay, want = case
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got = mf.linear_attention(q, k, v, decay)
                torch.cuda.current_stream().synchronize()
                bad.extend(0 for x, y in zip(got, want) if not x.equal(y))

    threads = [threading.Thread(target=work, args=(c,)) for c in cases for _ in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not bad and mf.check_operators() == mf.MF_OK
