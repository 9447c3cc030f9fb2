"""Linear attention, the embedding and clipping without a GPU: their formulas against differences, and what is refused."""
import ctypes as C

import numpy as np
import pytest

import _attend_ref as A


@pytest.fixture(scope="module")
def mf():
    from paper_2609_02109_gb300 import build
    build.build()
    from paper_2609_02109_gb300 import mf as mod
    return mod


@pytest.mark.parametrize("with_marks", [False, True])
def test_the_gradient_of_attention_is_that_of_differences(with_marks):
    r = np.random.default_rng(5)
    b, t, h, dk, dv = 2, 17, 2, 3, 4
    q, k, v, do = (r.standard_normal((b, t, h, d)) for d in (dk, dk, dv, dv))
    state, dlast = r.standard_normal((b, h, dk, dv)), r.standard_normal((b, h, dk, dv))
    marks = r.integers(0, 3, (b, t)).astype(np.uint8) if with_marks else None
    decay = np.array([-0.1, -1.5])

    def loss(q, k, v, state):
        o, last, _ = A.attend(q, k, v, decay, state, marks, 0.7)
        return (o * do).sum() + (last * dlast).sum()

    got = A.attend_grad(do, dlast, q, k, v, decay, state, marks, 0.7)
    eps = 1e-5  # central differences: the loss is quadratic in no input, so only its rounding is left: 1e-15 100 / eps
    for n, grad in enumerate(got):
        args = [q, k, v, state]
        for _ in range(12):
            at = tuple(r.integers(0, m) for m in args[n].shape)
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[n][at] += eps
            down[n][at] -= eps
            assert abs((loss(*up) - loss(*down)) / (2 * eps) - grad[at]) < 1e-7


def test_chunks_give_what_steps_give():
    """The form by chunks (products within a chunk, and the state before it) equals the steps."""
    r = np.random.default_rng(6)
    t, d, size = 24, 3, 8
    q, k, v = (r.standard_normal((1, t, 1, d)) for _ in range(3))
    decay = np.array([-0.2])
    o, last, _ = A.attend(q, k, v, decay, None, None, 1.0)
    s = np.zeros((d, d))
    for c in range(0, t, size):
        x, y, z = (a[0, c:c + size, 0] for a in (q, k, v))
        n = np.arange(1, size + 1)
        w = np.tril(np.exp(decay[0] * (n[:, None] - n[None])))
        got = (w * (x @ y.T)) @ z + np.exp(decay[0] * n)[:, None] * (x @ s)
        assert np.abs(got - o[0, c:c + size, 0]).max() < 1e-12
        s = np.exp(decay[0] * size) * s + (y * np.exp(decay[0] * (size - n))[:, None]).T @ z
    assert np.abs(s - last[0, 0]).max() < 1e-12


# -- what the C ABI refuses, before anything runs ---------------------------------------------
P = 0x10000  # an address that is never read


def _attend(mf, cls, **over):
    b, t, h, dk, dv = 2, 5, 3, 4, 6
    kw = dict(type=0, batch=b, time=t, heads=h, dim_k=dk, dim_v=dv, d_log_decay=P, d_marks=None, scale=1.0, d_status=None)
    seq = lambda d: mf._Heads(P, t * h * d, h * d, d)  # noqa: E731
    kw.update(q=seq(dk), k=seq(dk), v=seq(dv))
    if cls is mf._LinearAttention:
        kw.update(d_state=None, o=seq(dv), d_last=None, d_saved=None)
    else:
        kw.update(d_saved=P, dout=seq(dv), d_dlast=None, dq=seq(dk), dk=seq(dk), dv=seq(dv), d_dstate=None)
    kw.update({n: mf._Heads(*v) if isinstance(v, tuple) else v for n, v in over.items()})
    return cls(**kw)


BAD = [dict(type=3), dict(type=-1), dict(batch=-1), dict(time=-1), dict(heads=-1), dict(dim_k=-1), dict(dim_v=129),
       dict(dim_k=129), dict(time=1 << 31), dict(batch=1 << 20, heads=1 << 20), dict(q=(None, 60, 12, 4)),
       dict(k=(P + 2, 60, 12, 4)), dict(v=(P, -1, 18, 6)), dict(q=(P, 60, 1 << 60, 4)), dict(d_log_decay=None),
       dict(d_log_decay=P + 1), dict(scale=float("nan")), dict(scale=float("inf")), dict(d_marks=P, marks_stride_time=-1),
       dict(d_status=P + 2)]


@pytest.mark.parametrize("over", BAD + [dict(o=(None, 90, 18, 6)), dict(o=(P, 0, 18, 6)), dict(o=(P, 90, 18, 5)), dict(o=(P, 90, 12, 6)),
                                        dict(d_state=P + 1), dict(d_last=P + 2), dict(d_saved=P + 3)])
def test_attention_refuses(mf, over):
    p = _attend(mf, mf._LinearAttention, **over)
    assert mf.lib().mf_linear_attention_forward(C.byref(p), None, 0, None) == mf.MF_EINVAL
    assert mf.lib().mf_last_error().startswith(b"mf_linear_attention_forward: ")


@pytest.mark.parametrize("over", BAD + [dict(dout=(None, 90, 18, 6)), dict(dq=(P, 0, 12, 4)), dict(dk=(P, 60, 12, 3)),
                                        dict(dv=(P + 1, 90, 18, 6)), dict(d_saved=None), dict(d_dlast=P + 1), dict(d_dstate=P + 2)])
def test_the_gradient_of_attention_refuses(mf, over):
    p = _attend(mf, mf._LinearAttentionGrad, **over)
    assert mf.lib().mf_linear_attention_backward(C.byref(p), None, 0, None) == mf.MF_EINVAL
    assert mf.lib().mf_last_error().startswith(b"mf_linear_attention_backward: ")


def _embed(mf, cls, **over):
    kw = dict(type=1, id_bits=64, rows=7, dim=4, tokens=5, d_ids=P, scale=1.0, d_status=None)
    kw.update(dict(d_table=P, table_stride=4, d_out=P, out_stride=4) if cls is mf._Embedding else
              dict(d_dout=P, dout_stride=4, d_dtable=P, dtable_stride=4))
    kw.update(over)
    return cls(**kw)


EMBED_BAD = [dict(type=3), dict(id_bits=16), dict(rows=-1), dict(dim=-1), dict(tokens=-1), dict(rows=1 << 31), dict(dim=1 << 31),
             dict(rows=1 << 30, dim=1 << 30), dict(d_ids=None), dict(d_ids=P + 4), dict(scale=float("inf")),
             dict(scale=float("nan")), dict(d_status=P + 1)]


@pytest.mark.parametrize("over", EMBED_BAD + [dict(d_table=None), dict(d_table=P + 1), dict(table_stride=-1), dict(d_out=None),
                                              dict(d_out=P + 1), dict(out_stride=3), dict(out_stride=1 << 60)])
def test_the_embedding_refuses(mf, over):
    assert mf.lib().mf_embedding_forward(C.byref(_embed(mf, mf._Embedding, **over)), None) == mf.MF_EINVAL
    assert mf.lib().mf_last_error().startswith(b"mf_embedding_forward: ")


@pytest.mark.parametrize("over", EMBED_BAD + [dict(d_dout=None), dict(d_dout=P + 1), dict(dout_stride=-1), dict(d_dtable=None),
                                              dict(d_dtable=P + 1), dict(dtable_stride=3)])
def test_the_gradient_of_the_embedding_refuses(mf, over):
    p = _embed(mf, mf._EmbeddingGrad, **over)
    assert mf.lib().mf_embedding_backward(C.byref(p), P, 1 << 30, None) == mf.MF_EINVAL
    assert mf.lib().mf_last_error().startswith(b"mf_embedding_backward: ")


@pytest.mark.parametrize("work,size", [(None, 1 << 30), (P + 8, 1 << 30), (P, 16)])
def test_workspaces_are_checked(mf, work, size):
    p = _embed(mf, mf._EmbeddingGrad, rows=70000)
    assert mf.lib().mf_embedding_backward(C.byref(p), work, size, None) == mf.MF_EINVAL
    assert b"d_work" in mf.lib().mf_last_error()


def _clip(mf, ins, outs, sizes, types, max_norm=1.0, eps=0.0, norm=P, **over):
    n = len(ins)
    keep = ((C.c_uint64 * n)(*ins), (C.c_uint64 * n)(*outs), (C.c_int64 * n)(*sizes), (C.c_int32 * n)(*types))
    args = dict(count=n, d_in=C.addressof(keep[0]), d_out=C.addressof(keep[1]), sizes=C.addressof(keep[2]),
                types=C.addressof(keep[3]), max_norm=max_norm, eps=eps, d_norm=norm)
    args.update(over)
    p = mf._Clip(**args)
    status = mf.lib().mf_clip_gradients(C.byref(p), P, 0, None)  # (no scratch: a large call that is fine otherwise ends there)
    return status, mf.lib().mf_last_error().decode()


FOUR = dict(ins=[P, P + 64], outs=[P, P + 64], sizes=[8, 8], types=[0, 1])
LARGE = 1 << 20  # values: a tensor that makes a call large


def _with_large(ins, outs, sizes, types, **more):
    far = P + (1 << 30)
    return dict(ins=ins + [far], outs=outs + [far], sizes=sizes + [LARGE], types=types + [0], **more)


@pytest.mark.parametrize("over", [
    dict(count=-1), dict(count=1 << 31), dict(sizes=[8, -1]), dict(sizes=[8, 1 << 40]),
    dict(sizes=[1 << 39, 1 << 39]), dict(types=[0, 3]), dict(ins=[P + 2, P + 64], outs=[P + 2, P + 64]),
    dict(ins=[0, P + 64], outs=[0, P + 64]), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=-1.0),
    dict(eps=float("inf")), dict(norm=P + 1),
    dict(ins=[P, P], outs=[P, P]),                          # a tensor twice
    dict(ins=[P, P + 31], outs=[P, P + 31], types=[0, 0], sizes=[8, 1]),
    dict(ins=[P, P + 16], outs=[P, P + 16]),                # tensors that overlap
    dict(ins=[P, P + 64], outs=[P + 4, P + 64]),            # an output over its own input's other values
    dict(ins=[P, P + 64], outs=[P + 64, P + 128]),          # an output over another input
    dict(ins=[P, P + 256], outs=[P + 512, P + 512])])       # two outputs
def test_clipping_refuses(mf, over):
    status, text = _clip(mf, **{**FOUR, **over})
    assert status == mf.MF_EINVAL and text.startswith("mf_clip_gradients: ") and "d_work" not in text


def test_clipping_refuses_missing_arrays(mf):
    for name in ("d_in", "d_out", "sizes", "types"):
        n, kinds = (C.c_int64 * 2)(8, 8), (C.c_int32 * 2)(0, 0)
        args = dict(count=2, d_in=C.addressof(n), d_out=C.addressof(n), sizes=C.addressof(n), types=C.addressof(kinds))
        p = mf._Clip(**{**args, name: None}, max_norm=1.0, eps=0.0, d_norm=P)
        assert mf.lib().mf_clip_gradients(C.byref(p), P, 0, None) == mf.MF_EINVAL
        assert b"NULL" in mf.lib().mf_last_error()


@pytest.mark.parametrize("kw", [FOUR, dict(FOUR, outs=[P + 256, P + 512]), dict(FOUR, ins=[P + 64, P], outs=[P + 64, P]),
                                dict(FOUR, ins=[P, P], outs=[P + 64, P + 128]),       # an input twice, outputs apart
                                dict(FOUR, sizes=[0, 8], ins=[0, P], outs=[0, P]), dict(FOUR, max_norm=float("inf")),
                                dict(FOUR, max_norm=0.0)])
def test_what_clipping_takes(mf, kw):
    """Everything but the scratch memory is fine."""
    status, text = _clip(mf, **_with_large(**kw))
    assert status == mf.MF_EINVAL and "d_work is too small" in text


def test_bindings_pack_the_structures(mf):
    """The packed arguments have the structures' sizes and fields."""
    for pack, cls in ((mf._PACK_ATTEND, mf._LinearAttention), (mf._PACK_ATTEND_GRAD, mf._LinearAttentionGrad),
                      (mf._PACK_EMBEDDING, mf._Embedding), (mf._PACK_EMBEDDING, mf._EmbeddingGrad), (mf._PACK_CLIP, mf._Clip)):
        flat = []

        def fields(c):
            for _, kind in c._fields_:
                if hasattr(kind, "_fields_"):
                    fields(kind)
                else:
                    flat.append(kind)

        fields(cls)
        values = [float(i) if kind is C.c_float else i for i, kind in enumerate(flat, 1)]
        got, back = cls.from_buffer_copy(pack(*values).ljust(C.sizeof(cls), b"\0")), []

        def read(v):
            for name, kind in v._fields_:
                x = getattr(v, name)
                if hasattr(kind, "_fields_"):
                    read(x)
                else:
                    back.append(x)

        read(got)
        assert back == values
