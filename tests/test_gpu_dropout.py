"""Counter-based dropout on the GPU against the plain definition: elements bit
for bit, the gain's gradient to the rounding of its sum (terms in fp32 chains of
at most 1024 elements per thread and fp64 above: 2^-24 (1024 + 2) of the sum of
magnitudes), and gradients against differences."""
import numpy as np
import pytest

import fp4_plain as P
from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": (mnmt.F32, torch.float32), "bf16": (mnmt.BF16, torch.bfloat16), "f16": (mnmt.F16, torch.float16)}
SEED, OFFSET = 0x9E3779B97F4A7C15, (5 << 32) | 77


def strided(a, dtype, pad, off=0):
    M, K = a.shape
    buf = torch.full((M * (K + pad) + off,), 7.0, dtype=dtype, device="cuda")
    v = buf[off:].view(M, K + pad)[:, :K]
    v.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return v


def host(t):
    torch.cuda.synchronize()
    return t.float().cpu().numpy()


def rounded(v, dt):
    return torch.from_numpy(np.ascontiguousarray(v, np.float32)).to(dt).float().numpy()


def draw(M, d, seed=0):
    return np.random.default_rng(seed + M * 31 + d).standard_normal((M, d)).astype(np.float32)


@pytest.mark.parametrize("M,d", [(1, 1), (1, 7), (1, 768), (3, 9), (30, 64), (5, 1001), (257, 40)])
@pytest.mark.parametrize("ty,oty", [("bf16", "bf16"), ("f32", "f32"), ("f16", "f32"), ("bf16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("relu,resid,p,pad,off", [(0, 0, 0.1, 0, 0), (1, 1, 0.3, 8, 0), (0, 1, 0.0, 5, 1), (1, 0, 1.0, 0, 0)])
def test_forward_and_backward(M, d, ty, oty, relu, resid, p, pad, off):
    (xt, xdt), (ot, odt) = TYPES[ty], TYPES[oty]
    x = strided(draw(M, d), xdt, pad, off)
    r = strided(draw(M, d, 1) + np.float32(0.5), odt, pad, off) if resid else None
    out = strided(np.zeros((M, d), np.float32), odt, pad, off)
    gamma, ld = 0.75, d + pad
    mnmt.mnmt_dropout(x, xt, ld, r, ld, gamma, p, SEED, OFFSET, relu, M, d, out, ot, ld)
    keep, s = P.keep(M, d, p, SEED, OFFSET)
    xh = host(x)
    v = np.where(keep, (np.maximum(xh, 0) if relu else xh) * np.float32(s), np.float32(0))
    want = np.float32(gamma) * host(r) + v if resid else v
    assert np.array_equal(host(out), rounded(want, odt))

    g = strided(draw(M, d, 2), odt, pad, off)
    gx = strided(np.zeros((M, d), np.float32), xdt, pad, off)
    gr = strided(np.zeros((M, d), np.float32), odt, pad, off) if resid else None
    gg = torch.full((1,), 9.0, device="cuda") if resid else None
    ws = torch.empty(mnmt.DROPOUT_WORKSPACE, dtype=torch.uint8, device="cuda")
    args = (g, ot, ld, x, xt, ld, r, ld, gamma, p, SEED, OFFSET, relu, M, d)
    mnmt.mnmt_dropout_backward(*args, gx, ld, gr, ld, gg, ws)
    gh = host(g)
    live = keep & (xh > 0) if relu else keep
    assert np.array_equal(host(gx), rounded(np.where(live, gh * np.float32(s), 0), xdt))
    if resid:
        assert np.array_equal(host(gr), rounded(np.float32(gamma) * gh, odt))
        t = gh.astype(np.float64) * host(r)
        assert abs(float(gg.item()) - t.sum()) <= 2.0 ** -24 * 1026 * np.abs(t).sum()
        first = gg.item()
        mnmt.mnmt_dropout_backward(*args, None, 0, None, 0, gg, ws)
        assert gg.item() == first  # the same order each time, whatever else is asked for


def test_in_place_and_rows_alone():
    """out over x or r; a row's numbers do not depend on what else is drawn."""
    M, d = 9, 200
    x, r = torch.from_numpy(draw(M, d)).cuda(), torch.from_numpy(draw(M, d, 1)).cuda()
    out = torch.empty_like(x)
    mnmt.mnmt_dropout(x, mnmt.F32, d, r, d, 0.5, 0.4, 3, 9, 0, M, d, out, mnmt.F32, d)
    a, b = x.clone(), r.clone()
    mnmt.mnmt_dropout(a, mnmt.F32, d, r, d, 0.5, 0.4, 3, 9, 0, M, d, a, mnmt.F32, d)
    mnmt.mnmt_dropout(x, mnmt.F32, d, b, d, 0.5, 0.4, 3, 9, 0, M, d, b, mnmt.F32, d)
    assert torch.equal(a, out) and torch.equal(b, out)
    one = torch.empty((1, d), device="cuda")
    mnmt.mnmt_dropout(x, mnmt.F32, d, r, d, 0.5, 0.4, 3, 9, 0, 1, d, one, mnmt.F32, d)
    assert torch.equal(one[0], out[0])
    g = torch.from_numpy(draw(M, d, 2)).cuda()
    gx, gr = torch.empty_like(g), torch.empty_like(g)
    mnmt.mnmt_dropout_backward(g, mnmt.F32, d, None, mnmt.F32, d, None, 0, 0.5, 0.4, 3, 9, 0, M, d, gx, d, gr, d)
    h = g.clone()
    mnmt.mnmt_dropout_backward(h, mnmt.F32, d, None, mnmt.F32, d, None, 0, 0.5, 0.4, 3, 9, 0, M, d, h, d)
    assert torch.equal(h, gx)


def test_special_values():
    """What is dropped is zero even where it is infinite or NaN; ReLU keeps a NaN; other seeds and offsets draw other numbers."""
    d = 4096
    x = torch.full((1, d), float("nan"), device="cuda")
    out = torch.empty_like(x)
    for relu in (0, 1):
        mnmt.mnmt_dropout(x, mnmt.F32, d, None, 0, 1.0, 0.5, 1, 0, relu, 1, d, out, mnmt.F32, d)
        keep, _ = P.keep(1, d, 0.5, 1, 0)
        assert np.array_equal(np.isnan(host(out)), keep) and (host(out)[~keep] == 0).all()
    masks = []
    for seed, off in ((1, 0), (2, 0), (1, 1), (1, 1 << 32), (1 | 1 << 32, 0)):
        mnmt.mnmt_dropout(x, mnmt.F32, d, None, 0, 1.0, 0.5, seed, off, 0, 1, d, out, mnmt.F32, d)
        masks.append(np.isnan(host(out)))
    for i in range(len(masks)):
        for j in range(i):
            assert 0.4 < (masks[i] != masks[j]).mean() < 0.6


def test_gradients_by_differences():
    """out is linear in x (where x > 0 stays), r and gamma: with steps that are powers of two the differences of
    sum(g out) give the gradients to the rounding of fp32."""
    M, d, p, h = 4, 60, 0.25, 2.0 ** -3
    x, r, g = np.abs(draw(M, d)) + np.float32(0.5), draw(M, d, 1), draw(M, d, 2)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda()
    ws = torch.empty(mnmt.DROPOUT_WORKSPACE, dtype=torch.uint8, device="cuda")
    gx, gr, gg = torch.empty((M, d), device="cuda"), torch.empty((M, d), device="cuda"), torch.empty(1, device="cuda")
    mnmt.mnmt_dropout_backward(dev(g), mnmt.F32, d, dev(x), mnmt.F32, d, dev(r), d, 0.5, p, 11, 22, 1, M, d, gx, d, gr, d, gg, ws)

    def loss(x, r, gamma):
        out = torch.empty((M, d), device="cuda")
        mnmt.mnmt_dropout(dev(x), mnmt.F32, d, dev(r), d, gamma, p, 11, 22, 1, M, d, out, mnmt.F32, d)
        return (g.astype(np.float64) * host(out)).sum()

    tol = 2.0 ** -22 * np.abs(g).max() * 16 / h
    for i, j in [(0, 0), (1, 7), (2, 8), (3, 59), (2, 31)]:
        e = np.zeros((M, d), np.float32)
        e[i, j] = h
        assert abs((loss(x + e, r, 0.5) - loss(x - e, r, 0.5)) / (2 * h) - host(gx)[i, j]) <= tol
        assert abs((loss(x, r + e, 0.5) - loss(x, r - e, 0.5)) / (2 * h) - host(gr)[i, j]) <= tol
    assert abs((loss(x, r, 0.5 + h) - loss(x, r, 0.5 - h)) / (2 * h) - gg.item()) <= tol * M * d


def test_empty_and_refusals():
    x = torch.zeros((4, 8), device="cuda")
    ws = torch.empty(mnmt.DROPOUT_WORKSPACE, dtype=torch.uint8, device="cuda")
    mnmt.mnmt_dropout(None, mnmt.F32, 8, None, 0, 1.0, 0.1, 0, 0, 0, 0, 8, None, mnmt.F32, 8)
    gg = torch.ones(1, device="cuda")
    mnmt.mnmt_dropout_backward(None, mnmt.F32, 8, None, mnmt.F32, 8, None, 8, 1.0, 0.1, 0, 0, 0, 0, 8, ggamma=gg, workspace=ws)
    assert gg.item() == 0.0

    def refused(f, *a, **k):
        with pytest.raises(mnmt.MnmtError) as ei:
            f(*a, **k)
        assert ei.value.code == mnmt.EINVAL and str(ei.value)

    D, B = mnmt.mnmt_dropout, mnmt.mnmt_dropout_backward
    for p in (-0.1, 1.1, float("nan")):
        refused(D, x, mnmt.F32, 8, None, 0, 1.0, p, 0, 0, 0, 4, 8, x, mnmt.F32, 8)
    refused(D, x, 7, 8, None, 0, 1.0, 0.1, 0, 0, 0, 4, 8, x, mnmt.F32, 8)
    refused(D, x, mnmt.F32, 7, None, 0, 1.0, 0.1, 0, 0, 0, 4, 8, x, mnmt.F32, 8)
    refused(D, x, mnmt.F32, 8, None, 0, 1.0, 0.1, 0, 0, 0, 4, 8, None, mnmt.F32, 8)
    refused(D, x, mnmt.F32, 8, None, 0, 1.0, 0.1, 0, 0, 0, -1, 8, x, mnmt.F32, 8)
    refused(D, x, mnmt.F32, 8, None, 0, 1.0, 0.1, 0, 0, 0, 4, 0, x, mnmt.F32, 8)
    refused(D, x, mnmt.F32, 8, x.data_ptr() + 1, 8, 1.0, 0.1, 0, 0, 0, 4, 8, x, mnmt.F32, 8)
    refused(D, x, mnmt.F32, 8, None, 0, 1.0, 0.1, 0, 0, 0, 4, 8, x, mnmt.BF16, 8)
    refused(B, x, mnmt.F32, 8, None, mnmt.F32, 8, None, 0, 1.0, 0.1, 0, 0, 0, 4, 8)
    refused(B, x, mnmt.F32, 8, None, mnmt.F32, 8, None, 0, 1.0, 0.1, 0, 0, 1, 4, 8, x, 8)
    refused(B, x, mnmt.F32, 8, None, mnmt.F32, 8, x, 8, 1.0, 0.1, 0, 0, 0, 4, 8, ggamma=gg)
    refused(B, x, mnmt.F32, 8, None, mnmt.F32, 8, None, 8, 1.0, 0.1, 0, 0, 0, 4, 8, ggamma=gg, workspace=ws)
    refused(B, x, mnmt.F32, 8, None, mnmt.F32, 8, None, 8, 1.0, 0.1, 0, 0, 0, 4, 8, x, 8, x, 8)
