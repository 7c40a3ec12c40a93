"""Outputs of the 4-bit floating-point linear and of its gradients whose rows start
anywhere: the bits of an output with aligned rows, and nothing beside the rows."""
import pytest

from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": (mnmt.F32, torch.float32), "bf16": (mnmt.BF16, torch.bfloat16), "f16": (mnmt.F16, torch.float16)}


def packed(rows, cols, gen):
    q = mnmt.Fp4(rows, cols, mnmt.FP4_MX, 1.0, torch.empty((rows, mnmt.mnmt_fp4_pitch(cols)), dtype=torch.uint8, device="cuda"),
                 torch.empty(mnmt.mnmt_fp4_scale_bytes(rows, cols, mnmt.FP4_MX), dtype=torch.uint8, device="cuda"))
    x = torch.randn((rows, cols), generator=gen, device="cuda")
    mnmt.mnmt_fp4_quantize(q, x, mnmt.F32, cols)
    return x, q


class Out:
    """rows x cols from element `off` of a buffer on, rows `pad` elements apart, 5 everywhere else."""

    def __init__(self, rows, cols, dtype, pad, off):
        self.ld = cols + pad
        self.buf = torch.full((off + rows * self.ld + 64,), 5.0, dtype=dtype, device="cuda")
        self.at = self.buf[off:off + rows * self.ld].view(rows, self.ld)
        self.cols = cols

    def rest(self):
        """Whether what lies beside the rows is as it was (the rows themselves are overwritten here)."""
        self.at[:, :self.cols] = 5.0
        return bool((self.buf == 5.0).all())


PLACES = [(0, 0), (1, 0), (2, 0), (4, 0), (8, 0), (0, 1), (0, 2), (6, 2), (4, 4), (3, 5), (8, 8)]


@pytest.mark.parametrize("pad,off", PLACES)
@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("M,N,K", [(40, 33, 64), (129, 65, 100), (300, 200, 520), (513, 190, 64), (4001, 2050, 130), (2100, 2500, 4300)])
def test_linear_output(M, N, K, out, pad, off):
    ty, dtype = TYPES[out]
    gen = torch.Generator(device="cuda").manual_seed(M)
    xq, wq = packed(M, K, gen)[1], packed(N, K, gen)[1]
    n8 = -(-N // 8) * 8
    bias = torch.randn(N, generator=gen, device="cuda")
    want, got = Out(M, N, dtype, n8 - N, 0), Out(M, N, dtype, pad, off)
    for o in (want, got):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        mnmt.mnmt_fp4_linear(xq, wq, None, 0, 0, bias, False, o.at, ty, o.ld, status)
        assert int(status.item()) == 0
    assert torch.equal(want.at[:, :N], got.at[:, :N])
    assert float(want.at[:, :N].float().abs().max()) > 1.0
    assert want.rest() and got.rest()


@pytest.mark.parametrize("pad,off", PLACES)
@pytest.mark.parametrize("out", list(TYPES))
@pytest.mark.parametrize("M,N,K", [(46, 100, 40), (300, 200, 131), (33, 2500, 260), (2500, 70, 300), (1500, 2100, 1030)])
def test_gradients(M, N, K, out, pad, off):
    ty, dtype = TYPES[out]
    gen = torch.Generator(device="cuda").manual_seed(K)
    (x, xq), (w, wq) = packed(M, K, gen), packed(N, K, gen)
    x = x.to(dtype)
    G = torch.randn((M, N), generator=gen, device="cuda").to(torch.bfloat16)
    ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, N, K), dtype=torch.uint8, device="cuda")
    k8 = -(-K // 8) * 8
    pairs = []
    for p, o in ((k8 - K, 0), (pad, off)):
        gx, gw = Out(M, K, dtype, p, o), Out(N, K, torch.float32, p, o)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        mnmt.mnmt_fp4_linear_backward(xq, wq, G, N, x, ty, K, w, mnmt.F32, K, ws, gx.at, gx.ld, gw.at, gw.ld, None, status)
        assert int(status.item()) == 0
        pairs.append((gx, gw))
    for want, got in zip(*pairs):
        assert torch.equal(want.at[:, :K], got.at[:, :K])
        assert float(want.at[:, :K].float().abs().max()) > 1.0
        assert want.rest() and got.rest()
