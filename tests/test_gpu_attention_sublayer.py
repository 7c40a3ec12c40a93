"""The operators of a training step in a row, as a decoder's self-attention sublayer uses them: embedding, 4-bit linear,
attention, 4-bit linear, dropout onto the residual, and back to the table.  Each stage is held to its 64-bit form on what
the stage before it left."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import attention_sublayer as example  # noqa: E402
from seq_plain import Case, check  # noqa: E402

pytestmark = pytest.mark.gpu


def values(m, rows, cols):
    """The values of a packed matrix in 64 bits."""
    from paper_2306_04235_gb300 import mnmt

    v = torch.empty((rows, cols), device="cuda")
    mnmt.mnmt_fp4_dequantize(m, v, mnmt.F32, cols)
    return v.double()


def near(got, want, mag, terms, dtype):
    """A sum of `terms` products whose magnitudes add up to mag, in fp32, rounded to dtype."""
    u = torch.finfo(dtype).eps / 2
    return bool(((got.double() - want).abs() <= (terms + 8) * 2.0 ** -23 * mag + u * want.abs() + 1e-30).all())


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("lens", [[46], [20, 128, 1, 77, 100, 13], [300, 5]])
def test_stages(fmt, lens):
    s = example.Sublayer(d=256, heads=4, kv_heads=2, vocab=500, lens=lens, fmt=fmt, p=0.1, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(0, 500, (s.T,), generator=gen, device="cuda", dtype=torch.int32)
    s.forward(ids)
    g = torch.randn((s.T, s.d), generator=gen, device="cuda") * 1e-2
    s.backward(g)
    torch.cuda.synchronize()
    assert int(s.status) == 0 and int(s.qkv.status) == 0 and int(s.wo.status) == 0
    # embedding
    x = s.table[ids.long()].double() * s.scale + s.pe[s.pos.long()].double()
    assert near(s.x, x, x.abs() + s.pe[s.pos.long()].double().abs(), 2, torch.bfloat16)
    # the linears on what was quantised
    for lin, y in ((s.qkv, s.qkv.y), (s.wo, s.wo.y)):
        a, w = values(lin.xq, s.T, lin.K), values(lin.wq, lin.N, lin.K)
        assert near(y, a @ w.t() + lin.b.double(), a.abs() @ w.abs().t(), lin.K, torch.bfloat16)
    # attention, forward and back
    c = Case(s.q, s.k, s.v, s.attn.scale, True, s.starts, s.starts)
    o, lse, bo, bl = c.forward()
    check("o", s.o, o, bo)
    check("lse", s.lse, lse, bl)
    for name, got, (want, bound) in zip(("dq", "dk", "dv"), (s.dq, s.dk, s.dv), c.backward(s.wo.gx.view_as(s.o), s.o)):
        check(name, got, want, bound)
    # the linear's input gradient goes to the table: straight through, then the tokens' sums
    gx = s.qkv.gx.double()
    want = torch.zeros((500, s.d), dtype=torch.float64, device="cuda").index_add_(0, ids.long(), gx) * s.scale
    mag = torch.zeros((500, s.d), dtype=torch.float64, device="cuda").index_add_(0, ids.long(), gx.abs()) * s.scale
    assert near(s.gtable, want, mag, s.T, torch.float32)


def test_serving_continues_a_prompt():
    """One token more through the single-token form against the cache is the last row of a prompt that holds it."""
    s = example.Sublayer(d=256, heads=4, kv_heads=2, vocab=300, lens=[37], fmt="mx", p=0.0, seed=5)
    ids = torch.arange(37, dtype=torch.int32, device="cuda") * 7
    s.forward(ids)
    cache = example.Cache(s, 64)
    cache.fill(s.k[:36], s.v[:36])
    o = cache.step(s.q[36:37], s.k[36:37], s.v[36:37])
    torch.cuda.synchronize()
    full = Case(s.q, s.k, s.v, s.attn.scale, True, [0, 37], [0, 37]).forward()
    check("o", o, full[0][36:], full[2][36:])


def test_training_runs():
    losses, s = example.train(steps=6)
    assert all(x == x and x < float("inf") for x in losses)
    assert bool(torch.isfinite(s.gtable).all()) and bool(s.gtable.any())
