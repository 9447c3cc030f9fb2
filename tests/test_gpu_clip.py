"""Clipping by the norm of many tensors on the GPU."""
import numpy as np
import pytest

from _ops_ref import TYPE_U, U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mf():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_02109_gb300 import mf as m
    return m


def tensors(sizes, mix, seed=0, size=1.0):
    import torch
    dts = {"f": torch.float32, "b": torch.bfloat16, "h": torch.float16}
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(size * torch.randn(n, device="cuda", generator=g)).to(dts[mix[i % len(mix)]]) for i, n in enumerate(sizes)]


def check(mf, grads, max_norm, eps=1e-6, apart=False):
    """The norm: each square one rounding; sums of at most 2^14 / 512 squares a thread, then of chunks (up to 2^10), lanes,
    warps and blocks: fewer than 64 + chunks roundings in a row, halved by the square root, and one more for it.  The
    factor: two roundings more; the product one, and one to the type."""
    import torch
    kind = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}
    host = [g.double().cpu().numpy() for g in grads]
    want = np.sqrt(sum((h ** 2).sum() for h in host))
    chunks = max([1] + [-(-h.size // 16384) for h in host])
    rel = U * (64 + chunks)
    out = [torch.full_like(g, 7.0) for g in grads] if apart else None
    before = [g.clone() for g in grads]
    norm = mf.clip_gradients(grads, max_norm, eps, out)
    assert norm.shape == () and norm.dtype == torch.float32 and abs(float(norm) - want) <= rel * want
    factor = min(1.0, max_norm / (want + eps)) if want + eps > 0 else 1.0
    for g, b, o, h in zip(grads, before, out or grads, host):
        if apart:
            assert g.equal(b)
        k = kind[g.dtype]
        tiny = 2.0 ** -25 if k == "f16" else 1e-44
        assert (np.abs(o.double().cpu().numpy() - factor * h) <= (rel + 4 * U + TYPE_U[k] * 1.001) * factor * np.abs(h) + tiny).all()
        if factor == 1.0:
            assert o.equal(b)


SETS = {"predictors": ([5 * 64 * 12, 320, 20480, 320, 640, 10, 4], "f"), "one": ([1], "b"), "odd": ([3, 0, 17, 16385, 1, 4097], "fbh"),
        "mixed": (list(range(0, 300)), "fbh"), "large": ([1 << 20, 3, 999999], "bf"), "many": ([1 + i % 7 for i in range(2500)], "hb"),
        "chunks": ([16384 * 9 + 5] * 3, "h"), "none": ([], "f"), "empty": ([0, 0], "f")}


@pytest.mark.parametrize("name", list(SETS))
@pytest.mark.parametrize("max_norm", [0.0, 0.5, 1e9, float("inf")])
@pytest.mark.parametrize("apart", [False, True])
def test_sets(mf, name, max_norm, apart):
    sizes, mix = SETS[name]
    check(mf, tensors(sizes, mix), max_norm, apart=apart)


@pytest.mark.parametrize("size,mix", [(1e-30, "f"), (1e30, "f"), (1e-38, "f"), (1e15, "b"), (1e-6, "h"), (1e4, "h")])
def test_very_small_and_large_values(mf, size, mix):
    """Squares outside float32."""
    check(mf, tensors([20000, 7, 600000], mix, size=size), 1.0, eps=0.0, apart=True)
    check(mf, tensors([2000, 7], mix, size=size), 1.0, eps=0.0)


def test_sizes_far_apart_in_one_set(mf):
    for a, b in ((1e25, 1.0), (1.0, 1e-25), (1e25, 1e-25), (1e-20, 1e-21)):
        check(mf, tensors([1000], "f", size=a) + tensors([100000], "f", seed=1, size=b), 0.3)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n", [100, 700000])
def test_a_norm_that_is_not_finite_scales_nothing(mf, value, n):
    import torch
    grads = tensors([50, n], "f")
    grads[1][n // 2] = value
    before = [g.clone() for g in grads]
    out = [torch.empty_like(g) for g in grads]
    assert not torch.isfinite(mf.clip_gradients(grads, 1.0, out=out))
    assert not torch.isfinite(mf.clip_gradients(grads, 1.0))
    for g, o, b in zip(grads, out, before):
        assert torch.equal(g.nan_to_num(-7.0), b.nan_to_num(-7.0)) and torch.equal(o.nan_to_num(-7.0), b.nan_to_num(-7.0))


def test_zeros(mf):
    import torch
    for max_norm in (0.0, 1.0):
        grads = [torch.zeros(5, device="cuda"), torch.zeros(70, device="cuda")]
        assert float(mf.clip_gradients(grads, max_norm, eps=0.0)) == 0.0 and not grads[1].any()


def test_layouts(mf):
    """Axes in another order, offsets that are odd, inputs and outputs whose addresses differ modulo 16."""
    import torch
    base = torch.randn(40, 30, 5, device="cuda")
    flat = torch.randn(100003, device="cuda").bfloat16()
    grads = [base.permute(2, 0, 1), flat[1:50000], flat[50001:50002], flat[50003:], torch.randn(6, 1, 4, device="cuda").mT,
             torch.randn(300, 200, device="cuda").t()]
    out = [torch.empty(5, 40, 30, device="cuda").as_strided(g.shape, g.stride()) if i == 0 else torch.empty_like(g) for i, g in enumerate(grads)]
    assert all(o.stride() == g.stride() for o, g in zip(out, grads))
    check(mf, grads, 1.0)
    base = torch.randn(20001, device="cuda").half()
    check(mf, [base[3:]], 1.0, apart=True)
    o = torch.zeros(20010, device="cuda").half()
    mf.clip_gradients([base[3:]], 1.0, out=[o[4:4 + 19998]])
    # (equal bits where addresses are alike modulo 16: the norm's additions go by them)
    same = torch.empty(20001, device="cuda").half()
    same[3:] = base[3:]
    mf.clip_gradients([same[3:]], 1.0)
    assert o[4:4 + 19998].equal(same[3:]) and not o[:4].any() and not o[4 + 19998:].any()


def test_rows_beside_the_tensors_stay(mf):
    import torch
    flat = torch.ones(50000, device="cuda")
    mf.clip_gradients([flat[5:1000], flat[1003:40000]], 0.1)
    assert flat[:5].eq(1).all() and flat[1000:1003].eq(1).all() and flat[40000:].eq(1).all() and flat[5] < 0.1


def test_streams_graphs_and_equal_bits(mf):
    import torch
    for sizes in ([100, 3000], [900000, 5, 70000]):
        grads = tensors(sizes, "fb")
        outs = [torch.empty_like(g) for g in grads]
        want = mf.clip_gradients(grads, 0.5, out=outs)
        want, wanted = want.clone(), [o.clone() for o in outs]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            norm = mf.clip_gradients(grads, 0.5, out=outs)
        s.synchronize()
        assert norm.equal(want) and all(o.equal(w) for o, w in zip(outs, wanted))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            norm = mf.clip_gradients(grads, 0.5, out=outs)
        for g in grads:
            g.mul_(3)
        graph.replay()
        torch.cuda.synchronize()
        assert abs(float(norm) / float(want) - 3) < 1e-2


def test_binding_refuses(mf):
    import torch
    g = torch.randn(8, 6, device="cuda")
    for args, kw in (([[g, g]], {}), ([[g.cpu()]], {}), ([[g.double()]], {}), ([[g[:, :3]]], {}), ([[g, g[2:4]]], {}),
                     ([[g]], dict(out=[g[:4]])), ([[g]], dict(out=[g.half()])), ([[g]], dict(out=[])), ([[g[:4]]], dict(out=[g[2:6]])),
                     ([[g]], dict(eps=-1.0)), ([[g.clone().requires_grad_()]], {}), ([[g, 3.0]], {}), ([[g.expand(2, 8, 6)]], {})):
        with pytest.raises(mf.MFError) as e:
            mf.clip_gradients(*args, 1.0, **kw)
        assert e.value.status == mf.MF_EINVAL
    for bad in (-1.0, float("nan")):
        with pytest.raises(mf.MFError):
            mf.clip_gradients([g], bad)
