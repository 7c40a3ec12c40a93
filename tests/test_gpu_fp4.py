"""Microscaled 4-bit floating point on the GPU: quantisation bit for bit against
the plain definition, products and gradients against 64 bits.

Tolerances.  Codes, scales and values are defined to the last bit.  A product's
terms are exact and its sum runs in fp32: each of at most K/16 + 16 partial sums
loses at most 2^-23 of the sum of magnitudes A = sum |x w|, and the output is
rounded once: |y - y64| <= (K/16 + 16) 2^-23 A + u |y64| with u = 2^-23, 2^-8,
2^-11 for fp32, bf16, fp16 (plus the smallest fp16 step)."""
import numpy as np
import pytest

import fp4_plain as P
from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FMT = {"mx": mnmt.FP4_MX, "nv": mnmt.FP4_NV}
TYPES = {"f32": (mnmt.F32, torch.float32), "bf16": (mnmt.BF16, torch.bfloat16), "f16": (mnmt.F16, torch.float16)}
UNIT = {"f32": 2.0 ** -23, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
G = {"mx": 1.0, "nv": float(np.float32(0.0021))}


def strided(a, dtype, pad, off=0):
    """a as a view of a wider device buffer, its first element `off` elements in."""
    M, K = a.shape
    buf = torch.full((M * (K + pad) + off,), 7.0, dtype=dtype, device="cuda")
    v = buf[off:].view(M, K + pad)[:, :K]
    v.copy_(torch.from_numpy(np.ascontiguousarray(a)))
    return v


def host(t):
    torch.cuda.synchronize()
    return t.float().cpu().numpy()


def buffers(M, K, fmt, fill=0xA5):
    c = torch.full((max(M, 1), mnmt.mnmt_fp4_pitch(K)), fill, dtype=torch.uint8, device="cuda")
    s = torch.full((max(16, mnmt.mnmt_fp4_scale_bytes(M, K, FMT[fmt])),), fill, dtype=torch.uint8, device="cuda")
    return c, s


def packed(x, fmt):
    """x [M][K] quantised by the plain definition: the matrix and its values (float64)."""
    byte, code, v, inside = P.quantize(x, fmt, G[fmt])
    c, s = P.pack(byte, code, x.shape[1])
    c, s = torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()
    return mnmt.Fp4(x.shape[0], x.shape[1], FMT[fmt], G[fmt], c, s), v.astype(np.float64), inside


def inputs(rng, M, K, scale=1.0):
    x = rng.standard_normal((M, K)) * scale
    x *= np.exp2(rng.integers(-6, 7, (M, 1)))
    return x.astype(np.float32)


SHAPES = [(1, 1), (1, 16), (1, 33), (3, 31), (4, 512), (17, 257), (128, 64), (129, 129), (200, 1000), (2, 2049)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M,K", SHAPES)
@pytest.mark.parametrize("pad,off", [(0, 0), (8, 0), (5, 3)])
def test_quantize(fmt, ty, M, K, pad, off):
    rng = np.random.default_rng(M * 1000 + K)
    code, dt = TYPES[ty]
    x = strided(inputs(rng, M, K), dt, pad, off)
    v = strided(np.zeros((M, K), np.float32), dt, pad, off)
    c, s = buffers(M, K, fmt)
    mnmt.mnmt_fp4_quantize(mnmt.Fp4(M, K, FMT[fmt], G[fmt], c, s), x, code, K + pad, v, K + pad)
    byte, cd, val, inside = P.quantize(host(x), fmt, G[fmt])
    pc, ps = P.pack(byte, cd, K)
    assert np.array_equal(c.cpu().numpy(), pc)
    assert np.array_equal(s.cpu().numpy()[:ps.size], ps)
    want = torch.from_numpy(val).to(dt).float().numpy()
    assert np.array_equal(host(v), want)
    # values alone, in place; and from the packed form
    y = x.clone() if not pad and not off else x
    mnmt.mnmt_fp4_quantize(mnmt.Fp4(M, K, FMT[fmt], G[fmt]), y, code, K + pad, y, K + pad)
    assert np.array_equal(host(y), want)
    v.zero_()
    mnmt.mnmt_fp4_dequantize(mnmt.Fp4(M, K, FMT[fmt], G[fmt], c, s), v, code, K + pad)
    assert np.array_equal(host(v), want)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M,K,pad,off", [(1, 1, 0, 0), (5, 31, 0, 0), (130, 520, 8, 0), (7, 515, 3, 1)])
def test_quantize_backward(fmt, ty, M, K, pad, off):
    rng = np.random.default_rng(K)
    code, dt = TYPES[ty]
    x = strided(inputs(rng, M, K, 0.3), dt, pad, off)
    g = strided(rng.standard_normal((M, K)).astype(np.float32), dt, pad, off)
    gx = strided(np.zeros((M, K), np.float32), dt, pad, off)
    q = mnmt.Fp4(M, K, FMT[fmt], G[fmt])
    mnmt.mnmt_fp4_quantize_backward(q, x, code, K + pad, g, K + pad, gx, K + pad)
    inside = P.quantize(host(x), fmt, G[fmt])[3]
    want = np.where(inside, host(g), 0)
    assert np.array_equal(host(gx), want)
    if K > 100:
        assert 0 < (~inside).sum() < inside.size / 4  # some elements were held at 6
    mnmt.mnmt_fp4_quantize_backward(q, x, code, K + pad, g, K + pad, g, K + pad)
    assert np.array_equal(host(g), want)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_special_values(fmt):
    """Zeros, subnormals, the largest numbers, ties, infinities and NaN: a block with one of the last two is NaN as a
    whole, its neighbours are untouched, its gradient is zero."""
    B = P.BLOCK[fmt]
    x = np.zeros((12, 4 * B), np.float32)
    x[1, :B] = np.float32(2.0 ** -149)
    x[2, :B] = np.linspace(-2.0 ** -126, 2.0 ** -126, B)
    x[3, :B] = np.float32(3.4e38)
    x[4, B:2 * B] = np.linspace(-8, 8, B)
    x[5, :B] = np.resize([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], B)
    x[6, 3] = np.inf
    x[7, B + 1] = -np.inf
    x[8, 2 * B + 5] = np.nan
    x[8, 3 * B:] = 1.0
    x[9, :] = -0.0
    x[10, :] = 1e-30
    x[11, ::3] = np.float32(-7.5) * np.float32(G[fmt])
    M, K = x.shape
    c, s = buffers(M, K, fmt)
    xd, v = torch.from_numpy(x).cuda(), torch.empty((M, K), device="cuda")
    mnmt.mnmt_fp4_quantize(mnmt.Fp4(M, K, FMT[fmt], G[fmt], c, s), xd, mnmt.F32, K, v, K)
    byte, cd, val, inside = P.quantize(x, fmt, G[fmt])
    pc, ps = P.pack(byte, cd, K)
    assert np.array_equal(c.cpu().numpy(), pc) and np.array_equal(s.cpu().numpy(), ps)
    assert np.array_equal(host(v), val, equal_nan=True)
    assert np.isnan(val[6, :B]).all() and not np.isnan(val[6, B:]).any() and np.isnan(val[8]).sum() == B
    g = torch.ones((M, K), device="cuda")
    mnmt.mnmt_fp4_quantize_backward(mnmt.Fp4(M, K, FMT[fmt], G[fmt]), xd, mnmt.F32, K, g, K, g, K)
    assert np.array_equal(host(g), inside.astype(np.float32))
    # a NaN block makes NaN of its rows' products, and of no other
    w = torch.empty((40, K), device="cuda").normal_()
    wc, ws = buffers(40, K, fmt)
    wq = mnmt.Fp4(40, K, FMT[fmt], G[fmt], wc, ws)
    mnmt.mnmt_fp4_quantize(wq, w, mnmt.F32, K)
    for rows in (slice(0, 12), slice(5, 9)):
        xs = xd[rows].clone()
        n = xs.shape[0]
        xs[xs.abs() > 1e30] = 5.0  # the largest numbers stay out of the products: their sum overflows
        xs[torch.isinf(xd[rows])] = float("inf")
        xc, xsc = buffers(n, K, fmt)
        y = torch.empty((n, 40), device="cuda")
        mnmt.mnmt_fp4_linear(mnmt.Fp4(n, K, FMT[fmt], G[fmt], xc, xsc), wq, xs, mnmt.F32, K, None, False, y, mnmt.F32, 40)
        assert np.array_equal(np.isnan(host(y)).all(1), np.isnan(val[rows]).any(1))
        assert np.array_equal(np.isnan(host(y)).any(1), np.isnan(val[rows]).any(1))


LINEAR = [(1, 1, 1), (1, 64, 64), (1, 2048, 512), (2, 100, 33), (4, 130, 1000), (8, 512, 256), (16, 48, 96), (17, 300, 512), (33, 77, 129),
          (64, 256, 2048), (127, 129, 65), (128, 128, 128), (130, 1000, 384), (257, 264, 640), (512, 96, 4096), (1000, 513, 250)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", LINEAR)
@pytest.mark.parametrize("ty,out,relu,bias,pad", [("bf16", "bf16", True, True, 0), ("f32", "f32", False, False, 0), ("f16", "f16", False, True, 5),
                                                  ("bf16", "f32", False, True, 8)])
def test_linear(fmt, M, N, K, ty, out, relu, bias, pad):
    rng = np.random.default_rng(M + 7 * N + 13 * K)
    (xt, xdt), (yt, ydt) = TYPES[ty], TYPES[out]
    wq, w, _ = packed(rng.standard_normal((N, K)).astype(np.float32) * np.float32(0.05), fmt)
    x = strided(rng.standard_normal((M, K)).astype(np.float32), xdt, pad)
    b = rng.standard_normal(N).astype(np.float32) if bias else None
    bd = torch.from_numpy(b).cuda() if bias else None
    c, s = buffers(M, K, fmt)
    xq = mnmt.Fp4(M, K, FMT[fmt], G[fmt], c, s)
    y = strided(np.full((M, N), 3.0, np.float32), ydt, pad)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_fp4_linear(xq, wq, x, xt, K + pad, bd, relu, y, yt, N + pad, status)
    byte, cd, v, _ = P.quantize(host(x), fmt, G[fmt])
    pc, ps = P.pack(byte, cd, K)
    assert np.array_equal(c.cpu().numpy(), pc) and np.array_equal(s.cpu().numpy()[:ps.size], ps)
    v = v.astype(np.float64)
    want = v @ w.T + (b if bias else 0)
    mag = np.abs(v) @ np.abs(w).T + (np.abs(b) if bias else 0)
    if relu:
        want = np.maximum(want, 0)
    tol = (K / 16 + 16) * 2.0 ** -23 * mag + UNIT[out] * np.abs(want) + (2.0 ** -24 if out == "f16" else 0)
    got = host(y).astype(np.float64)
    assert (np.abs(got - want) <= tol).all()
    assert int(status.item()) == 0
    # nothing beside the N columns was written; the packed operand gives the same again
    if pad:
        full = torch.as_strided(y, (M, N + pad), (N + pad, 1))
        assert (host(full)[:, N:] == 7.0).all()
    y2 = strided(np.zeros((M, N), np.float32), ydt, pad)
    mnmt.mnmt_fp4_linear(xq, wq, None, 0, 0, bd, relu, y2, yt, N + pad, status)
    assert np.array_equal(host(y2), host(y))


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K,out,pad", [(2100, 2500, 320, "bf16", 0), (2100, 2500, 320, "f32", 3), (4096, 1536, 1100, "f16", 0), (385, 9000, 64, "f32", 0),
                                           (9000, 385, 544, "bf16", 1)])
def test_linear_of_many_tiles(fmt, M, N, K, out, pad):
    """Grids of more tiles than SMs: several tiles per CTA, on CTA pairs."""
    rng = np.random.default_rng(M + N + K)
    yt, ydt = TYPES[out]
    wq, w, _ = packed(rng.standard_normal((N, K)).astype(np.float32) * np.float32(0.05), fmt)
    x = strided(rng.standard_normal((M, K)).astype(np.float32), torch.bfloat16, 0)
    b = rng.standard_normal(N).astype(np.float32)
    c, s = buffers(M, K, fmt)
    y = strided(np.full((M, N), 3.0, np.float32), ydt, pad)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_fp4_linear(mnmt.Fp4(M, K, FMT[fmt], G[fmt], c, s), wq, x, mnmt.BF16, K, torch.from_numpy(b).cuda(), True, y, yt, N + pad, status)
    v = P.quantize(host(x), fmt, G[fmt])[2].astype(np.float64)
    want = np.maximum(v @ w.T + b, 0)
    mag = np.abs(v) @ np.abs(w).T + np.abs(b)
    tol = (K / 16 + 16) * 2.0 ** -23 * mag + UNIT[out] * np.abs(want) + (2.0 ** -24 if out == "f16" else 0)
    assert (np.abs(host(y).astype(np.float64) - want) <= tol).all() and int(status.item()) == 0
    if pad:
        assert (host(torch.as_strided(y, (M, N + pad), (N + pad, 1)))[:, N:] == 7.0).all()


def gradient_case(fmt, M, N, K, ty, wty, pad, seed=0):
    rng = np.random.default_rng(seed + M + 7 * N + 13 * K)
    x = strided(rng.standard_normal((M, K)).astype(np.float32), TYPES[ty][1], pad)
    w = strided(rng.standard_normal((N, K)).astype(np.float32) * np.float32(0.05), TYPES[wty][1], pad)
    g = strided(rng.standard_normal((M, N)).astype(np.float32), torch.bfloat16, pad)
    xq, xv, xin = packed(host(x), fmt)
    wq, wv, win = packed(host(w), fmt)
    return x, w, g, xq, xv, xin, wq, wv, win


BACKWARD = [(1, 1, 1), (1, 64, 64), (3, 100, 33), (46, 1024, 256), (130, 129, 65), (128, 256, 128), (300, 77, 1000), (1025, 264, 200), (2000, 40, 96)]


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", BACKWARD)
@pytest.mark.parametrize("ty,wty,pad", [("bf16", "f32", 0), ("f32", "bf16", 8), ("f16", "f32", 5)])
def test_linear_backward(fmt, M, N, K, ty, wty, pad):
    x, w, g, xq, xv, xin, wq, wv, win = gradient_case(fmt, M, N, K, ty, wty, pad)
    gx = strided(np.full((M, K), 3.0, np.float32), TYPES[ty][1], pad)
    gw = strided(np.full((N, K), 3.0, np.float32), torch.float32, pad)
    gb = torch.full((N,), 3.0, device="cuda")
    ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(xo, wo, gx, gw, gb):
        mnmt.mnmt_fp4_linear_backward(xq, wq, g, N + pad, xo, TYPES[ty][0], K + pad, wo, TYPES[wty][0], K + pad, ws, gx, K + pad, gw, K + pad, gb,
                                      status)

    def near(got, want, mag, n, unit):
        return (np.abs(host(got).astype(np.float64) - want) <= (n / 16 + 16) * 2.0 ** -23 * mag + unit * np.abs(want) + (2.0 ** -24 if unit == UNIT["f16"] else 0)).all()

    G64 = host(g).astype(np.float64)
    wx, ww = G64 @ wv, G64.T @ xv
    mx, mw = np.abs(G64) @ np.abs(wv), np.abs(G64).T @ np.abs(xv)
    run(x, w, gx, gw, gb)
    assert near(gx, np.where(xin, wx, 0), mx, N, UNIT[ty]) and near(gw, np.where(win, ww, 0), mw, M, UNIT["f32"])
    assert near(gb, G64.sum(0), np.abs(G64).sum(0), M, UNIT["f32"])
    assert (host(gx)[~xin] == 0).all() and (host(gw)[~win] == 0).all()
    # the same again bit for bit; no masks; one output at a time
    first = [host(t).copy() for t in (gx, gw, gb)]
    run(x, w, gx, gw, gb)
    assert all(np.array_equal(a, host(b)) for a, b in zip(first, (gx, gw, gb)))
    gx.fill_(3.0), gw.fill_(3.0), gb.fill_(3.0)
    run(None, None, gx, None, None)
    assert near(gx, wx, mx, N, UNIT[ty]) and (host(gw) == 3).all() and (host(gb) == 3).all()
    run(None, None, None, gw, None)
    assert near(gw, ww, mw, M, UNIT["f32"]) and (host(gb) == 3).all()
    run(None, None, None, None, gb)
    assert np.array_equal(host(gb), first[2])
    assert int(status.item()) == 0


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K,pad", [(3000, 1100, 1300, 0), (700, 5003, 2056, 3), (20000, 520, 264, 8), (300, 16000, 500, 0),
                                       (9001, 200, 72, 3)])
def test_linear_backward_of_many_tiles(fmt, M, N, K, pad):
    """Grids of CTA pairs and long sums, against float64."""
    x, w, g, xq, xv, xin, wq, wv, win = gradient_case(fmt, M, N, K, "bf16", "f32", pad)
    gx = strided(np.full((M, K), 3.0, np.float32), torch.bfloat16, pad)
    gw = strided(np.full((N, K), 3.0, np.float32), torch.float32, pad)
    gb = torch.full((N,), 3.0, device="cuda")
    ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_fp4_linear_backward(xq, wq, g, N + pad, x, mnmt.BF16, K + pad, w, mnmt.F32, K + pad, ws, gx, K + pad, gw, K + pad, gb, status)
    d = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda().double()
    G64, X64, W64 = g.double(), d(xv), d(wv)
    for got, want, mag, inside, n, unit in ((gx, G64 @ W64, G64.abs() @ W64.abs(), xin, N, UNIT["bf16"]),
                                            (gw, G64.t() @ X64, G64.abs().t() @ X64.abs(), win, M, UNIT["f32"])):
        want = want * d(inside)
        assert ((got.double() - want).abs() <= (n / 16 + 16) * 2.0 ** -23 * mag + unit * want.abs()).all()
        rel = ((got.double() - want).norm() / want.norm()).item()
        assert rel <= unit + n / 16 * 2.0 ** -24
        if pad:
            full = torch.as_strided(got, (got.shape[0], K + pad), (K + pad, 1))
            assert (full[:, K:] == 7.0).all()
    assert ((gb.double() - G64.sum(0)).abs() <= (M / 16 + 16) * 2.0 ** -23 * G64.abs().sum(0)).all() and int(status.item()) == 0


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_linear_gradient_by_differences(fmt):
    """The linear is linear in each operand: changing one code by one step changes sum(G y) by the gradient times
    the step (no masks, fp32)."""
    M, N, K = 5, 70, 96
    x, w, g, xq, xv, _, wq, wv, _ = gradient_case(fmt, M, N, K, "f32", "f32", 0)
    gx, gw = torch.empty((M, K), device="cuda"), torch.empty((N, K), device="cuda")
    ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    mnmt.mnmt_fp4_linear_backward(xq, wq, g, N, None, mnmt.F32, K, None, mnmt.F32, K, ws, gx, K, gw, K)
    G64 = host(g).astype(np.float64)

    def loss(a, b):
        y = torch.empty((M, N), device="cuda")
        mnmt.mnmt_fp4_linear(a, b, None, 0, 0, None, False, y, mnmt.F32, N)
        return (G64 * host(y)).sum()

    mag = np.abs(G64).sum() * np.abs(xv).max() * np.abs(wv).max() * K * 2.0 ** -22
    base = loss(xq, wq)
    for mat, v, grad in ((xq, xv, gx), (wq, wv, gw)):
        for r, k in [(0, 0), (v.shape[0] - 1, K - 1), (2, 33)]:
            codes = mat.buffers[0].clone()
            codes[r, k // 2] ^= 8 << (4 * (k % 2))  # the sign of one element
            flipped = mnmt.Fp4(mat.rows, mat.cols, mat.format, mat.tensor_scale, codes, mat.buffers[1])
            new = loss(flipped, wq) if mat is xq else loss(xq, flipped)
            assert abs((new - base) - (-2 * v[r, k]) * float(host(grad)[r, k])) <= 2 * mag


def test_empty():
    """No rows: nothing is read, and sums over nothing are zero."""
    w, _, _ = packed(np.ones((8, 40), np.float32), "mx")
    e = mnmt.Fp4(0, 40, mnmt.FP4_MX)
    mnmt.mnmt_fp4_quantize(e, None, mnmt.F32, 40, None, 40)
    mnmt.mnmt_fp4_linear(e, w, None, 0, 0, None, False, None, mnmt.F32, 8)
    ws = torch.empty(max(16, mnmt.mnmt_fp4_linear_backward_workspace(0, 8, 40)), dtype=torch.uint8, device="cuda")
    gw, gb = torch.ones((8, 40), device="cuda"), torch.ones(8, device="cuda")
    mnmt.mnmt_fp4_linear_backward(e, w, None, 8, None, mnmt.F32, 40, None, mnmt.F32, 40, ws, None, 0, gw, 40, gb)
    assert (host(gw) == 0).all() and (host(gb) == 0).all()
    x, _, _ = packed(np.ones((3, 40), np.float32), "mx")
    gx = torch.ones((3, 40), device="cuda")
    mnmt.mnmt_fp4_linear_backward(x, e, None, 0, None, mnmt.F32, 40, None, mnmt.F32, 40, ws, gx, 40)
    assert (host(gx) == 0).all()
    y = torch.ones((3, 8), device="cuda")
    mnmt.mnmt_fp4_linear(x, mnmt.Fp4(0, 40, mnmt.FP4_MX), None, 0, 0, None, False, y, mnmt.F32, 8)
    assert (host(y) == 1).all()


def test_other_stream():
    """Work runs on the stream it is given."""
    rng = np.random.default_rng(1)
    wq, w, _ = packed(rng.standard_normal((64, 128)).astype(np.float32), "mx")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a = torch.randn((2048, 2048), device="cuda")
        for _ in range(20):
            a = a @ a * 1e-3
        x = (a[:40, :128] * 0 + 1).to(torch.bfloat16).contiguous()
        c, s = buffers(40, 128, "mx")
        y = torch.empty((40, 64), device="cuda")
        mnmt.mnmt_fp4_linear(mnmt.Fp4(40, 128, mnmt.FP4_MX, 1.0, c, s), wq, x, mnmt.BF16, 128, None, False, y, mnmt.F32, 64, stream=side)
    want = np.broadcast_to(w.sum(1), (40, 64))
    assert np.abs(host(y) - want).max() <= 24 * 2.0 ** -23 * np.abs(w).sum(1).max()


def test_refusals():
    x = torch.zeros((4, 64), device="cuda")
    c, s = buffers(4, 64, "mx")
    q = mnmt.Fp4(4, 64, mnmt.FP4_MX, 1.0, c, s)

    def refused(f, *a, **k):
        with pytest.raises(mnmt.MnmtError) as ei:
            f(*a, **k)
        assert ei.value.code == mnmt.EINVAL and str(ei.value)

    Q = mnmt.mnmt_fp4_quantize
    refused(Q, q, None, mnmt.F32, 64)
    refused(Q, q, x, 3, 64)
    refused(Q, q, x, mnmt.F32, 63)
    refused(Q, q, x.data_ptr() + 2, mnmt.F32, 64)
    refused(Q, mnmt.Fp4(4, 64, mnmt.FP4_MX), x, mnmt.F32, 64)
    refused(Q, mnmt.Fp4(4, 64, mnmt.FP4_MX, 1.0, c, None), x, mnmt.F32, 64)
    refused(Q, mnmt.Fp4(4, 64, 2, 1.0, c, s), x, mnmt.F32, 64)
    refused(Q, mnmt.Fp4(-1, 64, 0, 1.0, c, s), x, mnmt.F32, 64)
    refused(Q, mnmt.Fp4(4, 0, 0, 1.0, c, s), x, mnmt.F32, 64)
    refused(Q, mnmt.Fp4(4, 64, 0, 1.0, c.data_ptr() + 8, s), x, mnmt.F32, 64)
    for g in (0.0, -1.0, float("nan"), float("inf"), 1e-38):
        refused(Q, mnmt.Fp4(4, 64, mnmt.FP4_NV, g, c, s), x, mnmt.F32, 64)
    refused(mnmt.mnmt_fp4_dequantize, mnmt.Fp4(4, 64, 0), x, mnmt.F32, 64)
    refused(mnmt.mnmt_fp4_dequantize, q, x, mnmt.F32, 60)
    refused(mnmt.mnmt_fp4_quantize_backward, q, x, mnmt.F32, 64, None, 64, x, 64)
    y = torch.zeros((4, 8), device="cuda")
    wc, wsc = buffers(8, 64, "mx")
    w = mnmt.Fp4(8, 64, mnmt.FP4_MX, 1.0, wc, wsc)
    L = mnmt.mnmt_fp4_linear
    refused(L, q, mnmt.Fp4(8, 32, 0, 1.0, wc, wsc), x, mnmt.F32, 64, None, False, y, mnmt.F32, 8)
    refused(L, q, mnmt.Fp4(8, 64, 1, 1.0, wc, wsc), x, mnmt.F32, 64, None, False, y, mnmt.F32, 8)
    refused(L, q, w, x, mnmt.F32, 64, None, False, y, mnmt.F32, 7)
    refused(L, q, w, x, mnmt.F32, 64, None, False, None, mnmt.F32, 8)
    refused(L, q, w, x, mnmt.F32, 64, None, False, y, 5, 8)
    refused(L, mnmt.Fp4(4, 64, 0), w, x, mnmt.F32, 64, None, False, y, mnmt.F32, 8)
    refused(L, q, w, x, mnmt.F32, 64, y.data_ptr() + 1, False, y, mnmt.F32, 8)
    B = mnmt.mnmt_fp4_linear_backward
    g = torch.zeros((4, 8), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(4, 8, 64), dtype=torch.uint8, device="cuda")
    gx = torch.zeros((4, 64), device="cuda")
    refused(B, q, w, None, 8, x, mnmt.F32, 64, None, 0, 0, ws, gx, 64)
    refused(B, q, w, g, 7, x, mnmt.F32, 64, None, 0, 0, ws, gx, 64)
    refused(B, q, w, g, 8, x, mnmt.F32, 64, None, 0, 0, None, gx, 64)
    refused(B, q, w, g, 8, x, 9, 64, None, 0, 0, ws, gx, 64)
    refused(B, q, w, g, 8, x, mnmt.F32, 64, None, 0, 0, ws, gx, 60)
    assert mnmt.mnmt_fp4_linear_backward_workspace(-1, 8, 64) == 0
