"""Sums of many terms of one sign in the 4-bit floating-point operators: what the tensor
core's truncating accumulator loses must not grow with their length."""
import pytest

from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": (mnmt.F32, torch.float32, 2.0 ** -24), "bf16": (mnmt.BF16, torch.bfloat16, 2.0 ** -8), "f16": (mnmt.F16, torch.float16, 2.0 ** -11)}


def empty(rows, cols, fmt=mnmt.FP4_MX, g=1.0):
    return mnmt.Fp4(rows, cols, fmt, g, torch.empty((rows, mnmt.mnmt_fp4_pitch(cols)), dtype=torch.uint8, device="cuda"),
                    torch.empty(mnmt.mnmt_fp4_scale_bytes(rows, cols, fmt), dtype=torch.uint8, device="cuda"))


def values(q):
    v = torch.empty((q.rows, q.cols), device="cuda")
    mnmt.mnmt_fp4_dequantize(q, v, mnmt.F32, q.cols)
    return v


@pytest.mark.parametrize("out", ["bf16", "f16"])
def test_input_gradient_over_many_outputs(out):
    """gX in 16 bits of a layer so wide that its sums would fill the accumulator: 40 tiles of 256 x 256 on 76 pairs, which
    are not split.  An MMA of 16 terms loses at most 2^-24 of the sum on average, and at most 512 of them follow each
    other: a bias of at most 2^-15 of the sum (all terms have one sign), beside the output's rounding."""
    M, N, K = 2560, 131072, 1024
    ty, dt, unit = TYPES[out]
    gen = torch.Generator(device="cuda").manual_seed(7)
    G = (torch.rand((M, N), generator=gen, device="cuda", dtype=torch.float32) + 0.5).mul_(2.0 ** -8).to(torch.bfloat16)
    w = torch.rand((N, K), generator=gen, device="cuda") + 0.25
    wq, xq = empty(N, K), empty(M, K)
    mnmt.mnmt_fp4_quantize(wq, w, mnmt.F32, K)
    mnmt.mnmt_fp4_quantize(xq, torch.zeros((M, K), device="cuda"), mnmt.F32, K)
    ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    gx = torch.empty((M, K), dtype=dt, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_fp4_linear_backward(xq, wq, G, N, None, ty, K, None, mnmt.F32, K, ws, gx, K, status=status)
    rows = torch.arange(0, M, 10, device="cuda")
    want = G[rows].double() @ values(wq).double()
    rel = (gx[rows].double() - want) / want
    assert int(status.item()) == 0
    assert float(rel.abs().max()) <= unit + 2.0 ** -15
    # the roundings of 262144 outputs cancel
    assert abs(float(rel.mean())) <= 2.0 ** -15


@pytest.mark.parametrize("fmt,g", [(mnmt.FP4_MX, 1.0), (mnmt.FP4_NV, 2.0 ** -9)])
@pytest.mark.parametrize("M,N,K", [(16, 128, 262144), (128, 19200, 65536), (300, 20000, 65536), (17, 40, 4160)])
@pytest.mark.parametrize("out", ["f32", "f16"])
def test_linear_of_long_rows(M, N, K, out, fmt, g):
    """Each kind of tile (128 x 64, 128 x 128, pairs).  At most 128 MMAs of 64 terms follow each other in the accumulator
    for fp32 outputs and 1024 for 16-bit ones, each losing 2^-25 of the sum on average (half a last bit), at most 2^-24;
    the few sums taken out are added in fp32: a bias of 2^-18 or 2^-14 of the sum, beside the output's rounding.  Every third block or so of
    W has one large element, so that block scales (and with them the bits of the terms) differ."""
    ty, dt, unit = TYPES[out]
    lost = 2.0 ** -18 if out == "f32" else 2.0 ** -14
    gen = torch.Generator(device="cuda").manual_seed(K)
    x = torch.rand((M, K), generator=gen, device="cuda") + 0.25
    w = torch.rand((N, K), generator=gen, device="cuda").mul_(0.5).add_(0.1)
    w[:, ::96] *= 7
    xq, wq = empty(M, K, fmt, g), empty(N, K, fmt, g)
    mnmt.mnmt_fp4_quantize(xq, x, mnmt.F32, K)
    mnmt.mnmt_fp4_quantize(wq, w, mnmt.F32, K)
    del x, w
    scale = 2.0 ** -6 if out == "f16" else 1.0  # of x, by way of its scales: sums within fp16's range
    if out == "f16":
        if fmt == mnmt.FP4_NV:
            xq.tensor_scale = g * scale
        else:
            s = xq.buffers[1]
            s.copy_(torch.where(s > 0, s.int() - 6, 0).to(torch.uint8))
    y = torch.empty((M, N), dtype=dt, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_fp4_linear(xq, wq, None, 0, 0, None, False, y, ty, N, status)
    cols = torch.arange(0, N, max(1, N // 500), device="cuda")
    want = values(xq).double() @ values(wq)[cols].double().t()
    rel = (y[:, cols].double() - want) / want
    assert int(status.item()) == 0 and float(want.min()) > 0
    assert float(rel.abs().max()) <= unit + 2 * lost
    assert abs(float(rel.mean())) <= lost + unit / rel.numel() ** 0.5


@pytest.mark.parametrize("products", [True, False])
@pytest.mark.parametrize("M,N", [(1 << 22, 8), ((1 << 22) - 511, 7)])
def test_bias_gradient_of_many_rows(M, N, products):
    """Columns of ones with 1 + 7/128 in every 512th row: sums of 512 rows are exact, and a chain of thousands of them
    rounds each the same way.  At most 512 + 512 additions in fp32, 64 bits above, one rounding: 2^-24 (1024 + 2)."""
    K = 8
    G = torch.ones((M, N), dtype=torch.bfloat16, device="cuda")
    G[::512] = 1 + 7 / 128
    xq, wq = empty(M, K), empty(N, K)
    mnmt.mnmt_fp4_quantize(xq, torch.ones((M, K), dtype=torch.bfloat16, device="cuda"), mnmt.BF16, K)
    mnmt.mnmt_fp4_quantize(wq, torch.ones((N, K), device="cuda"), mnmt.F32, K)
    ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    gx = torch.empty((M, K), dtype=torch.bfloat16, device="cuda") if products else None
    gw = torch.empty((N, K), device="cuda") if products else None
    gb = torch.empty(N, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mnmt.mnmt_fp4_linear_backward(xq, wq, G, N, None, mnmt.BF16, K, None, mnmt.F32, K, ws, gx, K, gw, K, gb, status)
    want = G.double().sum(0)
    assert int(status.item()) == 0
    assert ((gb.double() - want).abs() <= 2.0 ** -24 * 1026 * want).all()
