"""Output gradients inside a wider buffer that TMA reads where it lies (rows on 16 bytes,
a width that is no multiple of 8): what stands beside the columns is never used, even
where it is not a number."""
import pytest

from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def packed(x):
    rows, cols = x.shape
    q = mnmt.Fp4(rows, cols, mnmt.FP4_MX, 1.0, torch.empty((rows, mnmt.mnmt_fp4_pitch(cols)), dtype=torch.uint8, device="cuda"),
                 torch.empty(mnmt.mnmt_fp4_scale_bytes(rows, cols, mnmt.FP4_MX), dtype=torch.uint8, device="cuda"))
    mnmt.mnmt_fp4_quantize(q, x, mnmt.F32, cols)
    return q


@pytest.mark.parametrize("M,N,K", [(1, 1, 8), (46, 77, 40), (130, 1001, 256), (2100, 2507, 512), (300, 9, 64), (64, 32003, 512)])
@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
def test_columns_beside_the_gradient(M, N, K, fill):
    gen = torch.Generator(device="cuda").manual_seed(N)
    ld = -(-N // 8) * 8
    wide = torch.full((M, ld), fill, dtype=torch.bfloat16, device="cuda")
    wide[:, :N] = torch.randn((M, N), generator=gen, device="cuda")
    zeros = torch.where(torch.arange(ld, device="cuda") < N, wide, torch.zeros_like(wide))
    xq, wq = packed(torch.randn((M, K), generator=gen, device="cuda")), packed(torch.randn((N, K), generator=gen, device="cuda"))
    ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    outs = []
    for G in (zeros, wide):
        gx, gw, gb = torch.empty((M, K), device="cuda"), torch.empty((N, K), device="cuda"), torch.empty(N, device="cuda")
        mnmt.mnmt_fp4_linear_backward(xq, wq, G, ld, None, mnmt.F32, K, None, mnmt.F32, K, ws, gx, K, gw, K, gb)
        outs.append((gx, gw, gb))
    for a, b in zip(*outs):
        assert bool(torch.isfinite(a).all()) and torch.equal(a, b)
