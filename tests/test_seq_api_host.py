"""Refusals of attention over sequences and of the floating-point embedding: every one comes before any device work, so
it is seen without a GPU.  Addresses are numbers that nothing reads."""
import ctypes

import pytest

from paper_2306_04235_gb300 import mnmt

A = 1 << 20  # an aligned address


def shape(n=2, q_rows=10, k_rows=12, hq=4, hkv=2, d=64, dtype=mnmt.BF16, causal=True, scale=0.125, q_start=A, k_start=A, **kw):
    return mnmt.AttentionShape(n, q_rows, k_rows, hq, hkv, d, dtype, causal, scale, q_start, k_start, **kw)


def h(heads=4, d=64, at=A, row=None, head=None):
    return mnmt.Heads(at, heads * d if row is None else row, d if head is None else head)


def refused(call, *args):
    with pytest.raises(mnmt.MnmtError) as e:
        call(*args)
    assert e.value.code == mnmt.EINVAL, e.value
    return str(e.value)


def forward(s, q=None, k=None, v=None, o=None, lse=None, ws=A, status=None):
    mnmt.mnmt_attention_forward(s, q or h(at=A), k or h(2, at=2 * A), v or h(2, at=3 * A), o or h(at=4 * A), lse, ws, status)


@pytest.mark.parametrize("kw", [dict(n=-1), dict(q_rows=-1), dict(k_rows=(1 << 30) + 1), dict(hq=0), dict(hkv=0), dict(hq=5), dict(hq=1, hkv=2),
                                dict(hq=8192, hkv=8192), dict(d=0), dict(d=12), dict(d=136), dict(dtype=mnmt.F32), dict(dtype=7), dict(scale=0.0),
                                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q_start=None), dict(k_start=None),
                                dict(q_rows=1 << 30, hq=64, hkv=1),
                                dict(q_start=A + 2), dict(k_len=A + 1), dict(q_len=A + 3)])
def test_shapes(kw):
    refused(forward, shape(**kw))


@pytest.mark.parametrize("kw", [dict(q=h(at=0)), dict(q=h(at=A + 8)), dict(k=h(2, at=A + 2)), dict(q=h(row=252)), dict(q=h(row=260)), dict(k=h(2, row=64)),
                                dict(q=h(head=32)), dict(q=h(row=64, head=64)), dict(o=h(row=64, head=576)), dict(q=h(row=1 << 40)), dict(o=h(at=A)),
                                dict(o=h(at=2 * A)), dict(lse=A + 1), dict(ws=None), dict(ws=A + 8), dict(status=A + 2)])
def test_operands(kw):
    refused(lambda: forward(shape(), **kw))


def test_layouts_that_are_taken():
    """A head per row, and a row per head; a stride that nothing steps over is not looked at.  (With no sequences the call
    ends before the device is used, or where there is none, with another code.)"""
    for s, kw in [(shape(n=0), {}), (shape(n=0), dict(q=h(row=64, head=640))), (shape(n=0, q_rows=1), dict(q=h(row=1), o=h(at=4 * A, row=0))),
                  (shape(n=0, hq=1, hkv=1), dict(q=h(1, head=3), k=h(1, at=2 * A), v=h(1, at=3 * A), o=h(1, at=4 * A)))]:
        try:
            forward(s, **kw)
        except mnmt.MnmtError as e:
            assert e.code == mnmt.ECUDA, e


def test_null_structures():
    L = mnmt.lib()
    assert L.mnmt_attention_forward(None, h(), h(2), h(2), h(at=4 * A), None, A, None, None) == mnmt.EINVAL
    for i in range(4):
        ops = [h(at=A), h(2, at=2 * A), h(2, at=3 * A), h(at=4 * A)]
        ops[i] = ctypes.POINTER(mnmt.Heads)()
        assert L.mnmt_attention_forward(shape(), *ops, None, A, None, None) == mnmt.EINVAL
    assert L.mnmt_attention_forward_workspace(None) == 0


def test_token():
    s = shape(n=3, q_rows=4)
    refused(mnmt.mnmt_attention_token, s, h(at=A), h(2, at=2 * A), h(2, at=3 * A), h(at=4 * A), None, A)
    assert mnmt.mnmt_attention_token_workspace(s) == 0
    refused(mnmt.mnmt_attention_token, shape(n=4, q_rows=4, k_start=None), h(at=A), h(2, at=2 * A), h(2, at=3 * A), h(at=4 * A), None, A)


def backward(s, **kw):
    ops = dict(q=h(at=A), k=h(2, at=2 * A), v=h(2, at=3 * A), o=h(at=4 * A), lse=9 * A, g=h(at=5 * A), dq=h(at=6 * A), dk=h(2, at=7 * A),
               dv=h(2, at=8 * A), ws=A, status=None) | kw
    mnmt.mnmt_attention_backward(s, ops["q"], ops["k"], ops["v"], ops["o"], ops["lse"], ops["g"], ops["dq"], ops["dk"], ops["dv"], ops["ws"], ops["status"])


@pytest.mark.parametrize("kw", [dict(lse=None), dict(g=h(at=0)), dict(dq=h(at=A)), dict(dq=h(at=5 * A)), dict(dk=h(2, at=8 * A)), dict(dv=h(2, at=3 * A)),
                                dict(dk=h(2, at=7 * A, row=100)), dict(ws=None), dict(dv=h(2, at=6 * A))])
def test_backward(kw):
    refused(lambda: backward(shape(), **kw))


def test_workspaces():
    """Sizes come from the shape alone, without its arrays, and a buffer has to be given whatever they are."""
    for f in (mnmt.mnmt_attention_forward_workspace, mnmt.mnmt_attention_backward_workspace):
        assert f(shape(q_start=None, k_start=None)) > 0 and f(shape(n=0, q_rows=0, k_rows=0)) > 0 and f(shape(d=4)) == 0
    assert mnmt.mnmt_attention_token_workspace(shape(n=5, q_rows=5, k_start=None)) > 0
    big = shape(n=1 << 20, q_rows=1 << 29, k_rows=1 << 29, hq=32, hkv=8, d=128)
    assert mnmt.mnmt_attention_backward_workspace(big) >= 32 * (1 << 29) * 4
    assert [mnmt.mnmt_embed_backward_workspace(*x) > 0 for x in [(0, 1, 1), (10, 100, 64), (1 << 30, 1 << 30, 8), (-1, 5, 5), (5, 0, 5), (5, 5, 0)]] == \
        [True, True, True, False, False, False]


def embed(T=4, V=100, d=64, dt=mnmt.BF16, ldt=64, ids=A, table=A, out=2 * A, ot=mnmt.F32, ldo=64, scale=1.0, **kw):
    mnmt.mnmt_embed(ids, T, table, dt, ldt, V, d, scale, out, ot, ldo, **kw)


@pytest.mark.parametrize("kw", [dict(T=-1), dict(V=0), dict(d=0), dict(dt=5), dict(ot=-1), dict(ldt=63), dict(ldo=10), dict(ids=None), dict(ids=A + 2),
                                dict(table=None), dict(table=A + 1), dict(out=None), dict(out=A), dict(out=2 * A + 2), dict(scale=float("nan")),
                                dict(pe=A, ldpe=64, P=0, table=4 * A), dict(pe=A, ldpe=8, P=9, table=4 * A), dict(pe=A, ldpe=64, P=9, pos=A + 1),
                                dict(pe=2 * A, ldpe=64, P=9), dict(status=A + 1), dict(ldt=1 << 40)])
def test_embed(kw):
    refused(lambda: embed(**kw))


def embed_backward(T=4, V=100, d=64, gt=mnmt.BF16, ldg=64, ids=A, g=A, out=2 * A, ot=mnmt.F32, ldo=64, scale=1.0, acc=False, ws=A, status=None):
    mnmt.mnmt_embed_backward(ids, T, g, gt, ldg, scale, -1, V, d, out, ot, ldo, acc, ws, status)


@pytest.mark.parametrize("kw", [dict(T=-1), dict(V=0), dict(d=0), dict(gt=5), dict(ot=-1), dict(ldg=63), dict(ldo=10), dict(ids=None), dict(g=None),
                                dict(out=None), dict(out=A), dict(scale=float("inf")), dict(ws=None), dict(ws=A + 8), dict(status=A + 1)])
def test_embed_backward(kw):
    refused(lambda: embed_backward(**kw))
