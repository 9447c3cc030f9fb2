"""The embedding and its table's gradient on the GPU."""
import numpy as np
import pytest

import _attend_ref as A
from _ops_ref import TYPE_U, U

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


def check(mf, kind, rows, dim, ids, scale=1.7, wide=True, layout="plain", seed=1):
    import torch
    r = np.random.default_rng(seed)
    dt = kinds()[kind]
    n = ids.size

    def tensor(count):
        x = torch.tensor(r.standard_normal((count, dim)), dtype=torch.float32).to(dt).cuda()
        if layout == "plain":
            return x
        out = torch.zeros(count, dim + 7, dtype=dt, device="cuda")  # rows of an odd stride, at an odd offset
        out[:, 1:1 + dim] = x
        return out[:, 1:1 + dim]

    table, dout = tensor(rows), tensor(n)
    d_ids = torch.tensor(ids.astype(np.int64 if wide else np.int32)).cuda()
    d = lambda x: x.double().cpu().numpy()  # noqa: E731
    s = float(np.float32(scale))
    out = mf.embedding(table, d_ids, scale)
    want = np.where((ids >= 0)[:, None], s * d(table)[np.maximum(ids, 0)], 0) if rows else np.zeros((n, dim))
    tiny = 2.0 ** -25 if kind == "f16" else 1e-45
    # one rounding in fp32 and one to the type
    assert (np.abs(d(out) - want) <= (U + TYPE_U[kind] * (1 + U)) * np.abs(want) + tiny).all()
    grad = mf.embedding_backward(dout, d_ids, rows, scale)
    want, bound = A.embedding_grad(d(dout), ids, rows, s)
    off = np.abs(d(grad) - want)
    assert grad.shape == (rows, dim) and (off <= bound + TYPE_U[kind] * (np.abs(want) + bound) + tiny).all(), (off - bound).max()
    assert grad.equal(mf.embedding_backward(dout, d_ids, rows, scale))
    assert mf.check_operators() == mf.MF_OK


IDS = {
    "spread": lambda r, rows, n: r.integers(0, rows, n),
    "one": lambda r, rows, n: np.full(n, rows - 1),
    "few": lambda r, rows, n: r.choice([0, rows // 2, rows - 1], n, p=[0.9, 0.05, 0.05]),
    "padded": lambda r, rows, n: np.where(r.random(n) < 0.3, -1, r.integers(0, rows, n)),
    "none": lambda r, rows, n: np.full(n, -1),
    "sorted": lambda r, rows, n: np.sort(r.integers(0, rows, n)),
}


@pytest.mark.parametrize("ids", list(IDS))
@pytest.mark.parametrize("rows,dim,n", [(48, 8, 10240), (1, 1, 1), (2, 3, 500), (1000, 64, 300), (5, 130, 4097), (70000, 16, 6000),
                                         (300, 700, 2500), (40, 6, 16384), (40, 6, 16385), (2000, 12, 1700), (2000, 12, 1900),
                                        (1023, 9, 2048), (1024, 9, 2049), (1025, 33, 3)])
def test_ids(mf, ids, rows, dim, n):
    check(mf, "f32", rows, dim, IDS[ids](np.random.default_rng(3), rows, n))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", ["plain", "odd"])
@pytest.mark.parametrize("dim", [1, 2, 4, 6, 8, 15, 128, 129, 520])
@pytest.mark.parametrize("wide", [False, True])
def test_types_and_layouts(mf, kind, layout, dim, wide):
    check(mf, kind, 37, dim, IDS["padded"](np.random.default_rng(dim), 37, 1000), wide=wide, layout=layout)


@pytest.mark.parametrize("rows,dim,n", [(300000, 4, 200000), (3, 5, 300000), (1 << 21, 1, 150000)])
def test_many_tokens(mf, rows, dim, n):
    """More tiles of the sort than a block counts by itself, three digits, rows used by the hundred thousand."""
    check(mf, "f32", rows, dim, IDS["few" if rows < 10 else "padded"](np.random.default_rng(4), rows, n))


@pytest.mark.parametrize("rows,dim,n", [(0, 4, 0), (5, 0, 3), (5, 4, 0), (0, 4, 3)])
def test_sizes_of_zero(mf, rows, dim, n):
    check(mf, "bf16", rows, dim, np.full(n, -1))


def test_invalid_ids_are_zeros_and_told(mf):
    import torch
    table = torch.randn(6, 5, device="cuda")
    ids = torch.tensor([0, 6, -1, 5, -2, 1 << 40], device="cuda")
    out = mf.embedding(table, ids)
    assert out[[0, 3]].equal(table[[0, 5]]) and not out[[1, 2, 4, 5]].any()
    assert mf.check_operators() == mf.MF_EDEVICE and mf.check_operators() == mf.MF_OK
    grad = mf.embedding_backward(torch.ones(6, 5, device="cuda"), ids, 6)
    assert grad.sum(1).tolist() == [5.0, 0, 0, 0, 0, 5.0]
    assert mf.check_operators() == mf.MF_EDEVICE
    mf.embedding(table, torch.tensor([-1, 2], device="cuda"))
    assert mf.check_operators() == mf.MF_OK


def test_padding_hides_what_is_not_finite(mf):
    import torch
    dout = torch.full((4, 3), float("nan"), device="cuda")
    dout[1] = 2.0
    grad = mf.embedding_backward(dout, torch.tensor([-1, 3, -1, 0], device="cuda"), 5)
    assert grad[3].tolist() == [2.0] * 3 and torch.isnan(grad[0]).all() and not grad[[1, 2, 4]].any()
    table = torch.full((3, 2), float("nan"), device="cuda")
    table[1] = 1.0
    assert mf.embedding(table, torch.tensor([[1, -1]], device="cuda")).tolist() == [[[1.0, 1.0], [0.0, 0.0]]]


def test_shapes_streams_and_graphs(mf):
    import torch
    table = torch.randn(50, 12, device="cuda")
    ids = torch.randint(0, 50, (3, 4, 700), device="cuda", dtype=torch.int32)
    out = mf.embedding(table, ids, 2.0)
    assert out.shape == (3, 4, 700, 12) and out.equal(2 * table[ids.long()])
    want = mf.embedding_backward(out, ids, 50, 0.5)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = mf.embedding_backward(mf.embedding(table, ids, 2.0), ids, 50, 0.5)
    s.synchronize()
    assert got.equal(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = mf.embedding_backward(mf.embedding(table, ids, 2.0), ids, 50, 0.5)
    ids.copy_(torch.randint(0, 50, ids.shape, device="cuda", dtype=torch.int32))
    table.mul_(1.5)
    graph.replay()
    assert got.equal(mf.embedding_backward(mf.embedding(table, ids, 2.0), ids, 50, 0.5))
    wide = torch.randn(2, 700, 12, device="cuda").expand(2, 700, 12)
    assert mf.embedding_backward(wide, ids[0, :2].contiguous(), 50).shape == (50, 12)
    same = torch.randn(1, 12, device="cuda").expand(700, 12)  # one row for all tokens
    one = mf.embedding_backward(same, ids[0, 0], 50)
    assert one.equal(mf.embedding_backward(same.contiguous(), ids[0, 0], 50))


def test_binding_refuses(mf):
    import torch
    table, ids = torch.randn(6, 5, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    for args in ((table.cpu(), ids), (table, ids.cpu()), (table, ids.float()), (table.double(), ids), (table[0], ids),
                 (table.mT, ids), (table, torch.zeros(8, dtype=torch.int64, device="cuda")[::2]), (table, ids, float("nan"))):
        with pytest.raises(mf.MFError) as e:
            mf.embedding(*args)
        assert e.value.status == mf.MF_EINVAL
    dout = torch.randn(4, 5, device="cuda")
    for args in ((dout[:3], ids, 6), (dout.mT, ids, 6), (dout, ids, -1), (dout.double(), ids, 6), (dout, ids.cpu(), 6),
                 (dout, ids, 6, float("inf")), (torch.randn(2, 5, 2, device="cuda").mT, ids.view(2, 2), 6)):
        with pytest.raises(mf.MFError):
            mf.embedding_backward(*args)
