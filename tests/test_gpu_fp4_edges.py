"""4-bit floating-point operators and dropout where sizes, scales and offsets are
unusual: block scales far apart (a stale scale or slot would show), row counts on
either side of the kernels' limits, offsets beyond 32 bits, stream capture,
operands written by the kernel before."""
import numpy as np
import pytest

import fp4_plain as P
from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FMT = {"mx": mnmt.FP4_MX, "nv": mnmt.FP4_NV}


def empty(rows, cols, fmt, g=1.0):
    return mnmt.Fp4(rows, cols, FMT[fmt], g, torch.empty((rows, mnmt.mnmt_fp4_pitch(cols)), dtype=torch.uint8, device="cuda"),
                    torch.empty(mnmt.mnmt_fp4_scale_bytes(rows, cols, FMT[fmt]), dtype=torch.uint8, device="cuda"))


def values(q):
    v = torch.empty((q.rows, q.cols), device="cuda")
    mnmt.mnmt_fp4_dequantize(q, v, mnmt.F32, q.cols)
    return v


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,N,K", [(2100, 2500, 4096), (300, 5000, 2000), (130, 600, 8192), (40, 3000, 1500), (6, 900, 4096)])
def test_scales_far_apart(fmt, M, N, K):
    """Neighbouring blocks of rows differ by factors of up to 2^12, independently in both operands: each output is
    dominated by a few blocks, so a product with another block's scale is off by orders of magnitude.  Tolerance as
    for any product: (K/16 + 16) 2^-23 of the sum of magnitudes."""
    gen = torch.Generator(device="cuda").manual_seed(K)

    def draw(rows):
        x = torch.randn((rows, K), generator=gen, device="cuda")
        s = torch.randint(-6, 7, (rows, -(-K // 16)), generator=gen, device="cuda").float().exp2().repeat_interleave(16, 1)[:, :K]
        q = empty(rows, K, fmt, 0.03125)
        mnmt.mnmt_fp4_quantize(q, (x * s).contiguous(), mnmt.F32, K)
        return q

    xq, wq = draw(M), draw(N)
    y = torch.empty((M, N), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_fp4_linear(xq, wq, None, 0, 0, None, False, y, mnmt.F32, N, status)
    xv, wv = values(xq).double(), values(wq).double()
    want, mag = xv @ wv.t(), xv.abs() @ wv.abs().t()
    assert ((y.double() - want).abs() <= (K / 16 + 16) * 2.0 ** -23 * mag + 2.0 ** -23 * want.abs()).all()
    assert int(status.item()) == 0


@pytest.mark.parametrize("fmt", ["mx", "nv"])
@pytest.mark.parametrize("M,K", [(1, 32768), (1, 32769), (8, 4096), (8, 4097), (9, 64), (7, 31), (2, 16384), (3, 16384)])
def test_row_counts_at_the_kernels_limits(fmt, M, K):
    """Rows and depths on both sides of what the kernel for a few rows takes: the same product either way."""
    rng = np.random.default_rng(K)
    N = 70
    x = torch.from_numpy(rng.standard_normal((M, K)).astype(np.float32)).cuda().to(torch.bfloat16)
    g = 0.002
    wq, xq = empty(N, K, fmt, g), empty(M, K, fmt, g)
    mnmt.mnmt_fp4_quantize(wq, torch.from_numpy(rng.standard_normal((N, K)).astype(np.float32)).cuda(), mnmt.F32, K)
    y = torch.empty((M, N), device="cuda")
    mnmt.mnmt_fp4_linear(xq, wq, x, mnmt.BF16, K, None, False, y, mnmt.F32, N)
    byte, code, v, _ = P.quantize(x.float().cpu().numpy(), fmt, g)
    pc, ps = P.pack(byte, code, K)
    assert np.array_equal(xq.buffers[0].cpu().numpy(), pc) and np.array_equal(xq.buffers[1].cpu().numpy(), ps)
    wv = values(wq).double().cpu().numpy()
    want, mag = v.astype(np.float64) @ wv.T, np.abs(v.astype(np.float64)) @ np.abs(wv).T
    assert (np.abs(y.double().cpu().numpy() - want) <= (K / 16 + 16) * 2.0 ** -23 * mag + 2.0 ** -23 * np.abs(want)).all()


def test_offsets_beyond_32_bits():
    """Rows whose first element lies beyond 2^31 elements: strided input and output of a product, quantisation with
    its values, its gradient, and dropout; the last rows against the plain definitions."""
    M, N, K, ld = 70000, 40, 48, 32000  # M ld = 2.24e9 elements
    big = torch.empty((M, ld), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((M, ld), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = big[:, :K]
    x.copy_(torch.randn((M, K), generator=gen, device="cuda"))
    wq, xq = empty(N, K, "mx"), empty(M, K, "mx")
    w = torch.randn((N, K), generator=gen, device="cuda")
    mnmt.mnmt_fp4_quantize(wq, w, mnmt.F32, K)
    mnmt.mnmt_fp4_linear(xq, wq, x, mnmt.BF16, ld, None, False, out, mnmt.BF16, ld)
    tail = slice(M - 200, M)
    xt = x[tail].float().cpu().numpy()
    v = P.quantize(xt, "mx")[2].astype(np.float64)
    want = v @ values(wq).double().cpu().numpy().T
    got = out[tail, :N].double().cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 1e-4).all()
    assert (out[tail, N:2 * N] == 0).all()
    mnmt.mnmt_fp4_quantize(xq, x, mnmt.BF16, ld, out, ld)
    assert np.array_equal(out[tail, :K].float().cpu().numpy(), torch.from_numpy(P.quantize(xt, "mx")[2]).to(torch.bfloat16).float().numpy())
    mnmt.mnmt_fp4_quantize_backward(xq, x, mnmt.BF16, ld, x, ld, out, ld)
    assert np.array_equal(out[tail, :K].float().cpu().numpy(), np.where(P.quantize(xt, "mx")[3], xt, 0))
    mnmt.mnmt_dropout(x, mnmt.BF16, ld, None, 0, 1.0, 0.25, 5, 6, False, M, K, out, mnmt.BF16, ld)
    keep, s = P.keep(M, K, 0.25, 5, 6)
    d = np.where(keep[tail], xt * np.float32(s), np.float32(0))
    assert np.array_equal(out[tail, :K].float().cpu().numpy(), torch.from_numpy(d).to(torch.bfloat16).float().numpy())
    mnmt.mnmt_dropout_backward(x, mnmt.BF16, ld, None, mnmt.BF16, ld, None, 0, 1.0, 0.25, 5, 6, False, M, K, out, ld)
    assert np.array_equal(out[tail, :K].float().cpu().numpy(), torch.from_numpy(d).to(torch.bfloat16).float().numpy())


def test_capture_and_replay():
    """Every operator can be captured into a graph; replayed on new inputs it computes on those."""
    M, N, K = 150, 200, 96
    x = torch.empty((M, K), dtype=torch.bfloat16, device="cuda")
    g = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    w = torch.randn((N, K), device="cuda")
    xq, wq = empty(M, K, "mx"), empty(N, K, "mx")
    y, z = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
    gx, gw, gb = torch.empty((M, K), dtype=torch.bfloat16, device="cuda"), torch.empty((N, K), device="cuda"), torch.empty(N, device="cuda")
    gz, gg = torch.empty((M, N), dtype=torch.bfloat16, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    wd = torch.empty(mnmt.DROPOUT_WORKSPACE, dtype=torch.uint8, device="cuda")

    def step(stream):
        mnmt.mnmt_fp4_quantize(wq, w, mnmt.F32, K, stream=stream)
        mnmt.mnmt_fp4_linear(xq, wq, x, mnmt.BF16, K, None, False, y, mnmt.BF16, N, stream=stream)
        mnmt.mnmt_dropout(y, mnmt.BF16, N, g, N, 0.5, 0.3, 1, 2, True, M, N, z, mnmt.BF16, N, stream=stream)
        mnmt.mnmt_dropout_backward(g, mnmt.BF16, N, y, mnmt.BF16, N, z, N, 0.5, 0.3, 1, 2, True, M, N, gz, N, None, 0, gg, wd, stream=stream)
        mnmt.mnmt_fp4_linear_backward(xq, wq, gz, N, x, mnmt.BF16, K, w, mnmt.F32, K, ws, gx, K, gw, K, gb, stream=stream)

    def fill(seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        x.copy_(torch.randn((M, K), generator=gen, device="cuda"))
        g.copy_(torch.randn((M, N), generator=gen, device="cuda"))

    outs = (y, z, gz, gg, gx, gw, gb)
    fill(1)
    step(torch.cuda.current_stream())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        step(side)
        graph.capture_end()
    fill(2)
    step(torch.cuda.current_stream())
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    for t in outs:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(want, outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", ["mx", "nv"])
def test_back_to_back_operators_see_each_other(fmt):
    """A chain of calls without synchronisation, each reading what the one before wrote, gives what the same chain
    gives with a synchronisation after every call (32 times over)."""
    M, d, F = 96, 192, 320
    gen = torch.Generator(device="cuda").manual_seed(4)
    w1, w2 = torch.randn((F, d), generator=gen, device="cuda") * 0.05, torch.randn((d, F), generator=gen, device="cuda") * 0.05
    q1, q2 = empty(F, d, fmt, 1e-4), empty(d, F, fmt, 1e-4)
    xq, hq = empty(M, d, fmt, 0.01), empty(M, F, fmt, 0.01)

    def run(sync):
        r = torch.ones((M, d), device="cuda")
        x, h, v = (torch.empty((M, n), dtype=torch.bfloat16, device="cuda") for n in (d, F, d))
        for i in range(32):
            mnmt.mnmt_dropout(r, mnmt.F32, d, None, 0, 1.0, 0.1, 7, 3 * i, False, M, d, x, mnmt.BF16, d)
            sync()
            mnmt.mnmt_fp4_quantize(q1, w1, mnmt.F32, d)
            mnmt.mnmt_fp4_quantize(q2, w2, mnmt.F32, F)
            sync()
            mnmt.mnmt_fp4_linear(xq, q1, x, mnmt.BF16, d, None, True, h, mnmt.BF16, F)
            sync()
            mnmt.mnmt_fp4_linear(hq, q2, h, mnmt.BF16, F, None, False, v, mnmt.BF16, d)
            sync()
            mnmt.mnmt_dropout(v, mnmt.BF16, d, r, d, 0.9, 0.1, 7, 3 * i + 1, False, M, d, r, mnmt.F32, d)
            sync()
        torch.cuda.synchronize()
        return r

    assert torch.equal(run(lambda: None), run(torch.cuda.synchronize))
