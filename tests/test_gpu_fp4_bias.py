"""The bias gradient of the 4-bit floating-point linear: row counts on either side of
where its blocks of rows change, columns that end inside eight, gradients whose rows
TMA can and cannot read, with and without the products beside it."""
import pytest

from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def empty(rows, cols):
    return mnmt.Fp4(rows, cols, mnmt.FP4_MX, 1.0, torch.zeros((rows, mnmt.mnmt_fp4_pitch(cols)), dtype=torch.uint8, device="cuda"),
                    torch.zeros(mnmt.mnmt_fp4_scale_bytes(rows, cols, mnmt.FP4_MX), dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("products", [True, False])
@pytest.mark.parametrize("pad,off", [(0, 0), (8, 0), (3, 1)])
@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 63, 64, 65, 100, 333, 1000, 5003, 16400])
@pytest.mark.parametrize("N", [1, 7, 8, 255, 256, 257, 771, 2056])
def test_bias_gradient(M, N, pad, off, products):
    """Against the sum in 64 bits.  A term passes through at most M additions in fp32: M 2^-24 of the sum of
    magnitudes (with a little for terms of the second order).  The columns beside G hold NaN, the bytes past the
    workspace stay as they are, and a second call gives the same bits."""
    K = 40
    gen = torch.Generator(device="cuda").manual_seed(M * 4099 + N)
    wide = torch.full((M * (N + pad) + off + 64,), float("nan"), dtype=torch.bfloat16, device="cuda")
    G = wide[off:off + M * (N + pad)].view(M, N + pad)[:, :N]
    G.copy_(torch.randn((M, N), generator=gen, device="cuda"))
    size = mnmt.mnmt_fp4_linear_backward_workspace(M, N, K)
    ws = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    xq, wq = empty(M, K), empty(N, K)
    gx = torch.empty((M, K), device="cuda") if products else None
    gw = torch.empty((N, K), device="cuda") if products else None
    out = []
    for _ in range(2):
        gb = torch.full((N + 1,), 7.0, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        mnmt.mnmt_fp4_linear_backward(xq, wq, G, N + pad, None, mnmt.F32, K, None, mnmt.F32, K, ws, gx, K, gw, K, gb, status)
        assert int(status.item()) == 0 and float(gb[N].item()) == 7.0
        out.append(gb[:N])
    want, mag = G.double().sum(0), G.double().abs().sum(0)
    assert ((out[0].double() - want).abs() <= (M + 1) * 2.0 ** -24 * mag).all()
    assert torch.equal(out[0], out[1])
    assert bool((ws[size:] == 0xA5).all())
    if products:  # zero codes
        assert not bool(gx.any()) and not bool(gw.any())
