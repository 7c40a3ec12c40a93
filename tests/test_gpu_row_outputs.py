"""Outputs of the element-wise operators (4-bit quantisation, dropout) whose rows start
anywhere: the bits of an output with aligned rows, and nothing beside the rows."""
import pytest

from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": (mnmt.F32, torch.float32), "bf16": (mnmt.BF16, torch.bfloat16), "f16": (mnmt.F16, torch.float16)}
PLACES = [(0, 0), (1, 0), (8, 0), (0, 1), (3, 5), (6, 2), (16, 16)]


class Out:
    """rows x cols from element `off` of a buffer on, rows `pad` elements apart, 5 everywhere else."""

    def __init__(self, rows, cols, dtype, pad, off, a=None):
        self.ld = cols + pad
        self.buf = torch.full((off + rows * self.ld + 64,), 5.0, dtype=dtype, device="cuda")
        self.at = self.buf[off:off + rows * self.ld].view(rows, self.ld)
        self.cols = cols
        if a is not None:
            self.at[:, :cols] = a

    @property
    def rows(self):
        return self.at[:, :self.cols]

    def rest(self):
        """Whether what lies beside the rows is as it was (the rows themselves are overwritten here)."""
        self.rows[:] = 5.0
        return bool((self.buf == 5.0).all())


@pytest.mark.parametrize("pad,off", PLACES)
@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M,d", [(1, 1), (3, 7), (5, 31), (40, 64), (33, 130), (7, 515), (130, 1001)])
def test_quantize(M, d, ty, pad, off):
    code, dtype = TYPES[ty]
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn((M, d), generator=gen, device="cuda").to(dtype)
    g = torch.randn((M, d), generator=gen, device="cuda").to(dtype)
    d16 = -(-d // 16) * 16
    got = []
    for p, o in ((d16 - d, 0), (pad, off)):
        src, up, val, deq, gx = (Out(M, d, dtype, p, o, a) for a in (x, g, None, None, None))
        q = mnmt.Fp4(M, d, mnmt.FP4_NV, 0.01, torch.empty((M, mnmt.mnmt_fp4_pitch(d)), dtype=torch.uint8, device="cuda"),
                     torch.empty(mnmt.mnmt_fp4_scale_bytes(M, d, mnmt.FP4_NV), dtype=torch.uint8, device="cuda"))
        mnmt.mnmt_fp4_quantize(q, src.at, code, src.ld, val.at, val.ld)
        mnmt.mnmt_fp4_dequantize(q, deq.at, code, deq.ld)
        mnmt.mnmt_fp4_quantize_backward(q, src.at, code, src.ld, up.at, up.ld, gx.at, gx.ld)
        assert torch.equal(val.rows, deq.rows)
        got.append([val.rows.clone(), gx.rows.clone(), q.buffers[0], q.buffers[1]])
        assert torch.equal(src.rows, x) and torch.equal(up.rows, g)
        assert all(b.rest() for b in (src, up, val, deq, gx))
    for a, b in zip(*got):
        assert torch.equal(a, b)


@pytest.mark.parametrize("pad,off", PLACES)
@pytest.mark.parametrize("ty,rty", [("bf16", "f32"), ("f16", "f16"), ("f32", "bf16")])
@pytest.mark.parametrize("M,d", [(1, 1), (3, 7), (5, 31), (40, 64), (33, 130), (7, 515), (130, 1001)])
def test_dropout(M, d, ty, rty, pad, off):
    (code, dtype), (rcode, rdtype) = TYPES[ty], TYPES[rty]
    gen = torch.Generator(device="cuda").manual_seed(d)
    x = torch.randn((M, d), generator=gen, device="cuda").to(dtype)
    r = torch.randn((M, d), generator=gen, device="cuda").to(rdtype)
    g = torch.randn((M, d), generator=gen, device="cuda").to(rdtype)
    ws = torch.empty(mnmt.DROPOUT_WORKSPACE, dtype=torch.uint8, device="cuda")
    d16 = -(-d // 16) * 16
    got = []
    for p, o in ((d16 - d, 0), (pad, off)):
        sx, gx = Out(M, d, dtype, p, o, x), Out(M, d, dtype, p, o)
        sr, sg, out, gr = (Out(M, d, rdtype, p, o, a) for a in (r, g, None, None))
        gg = torch.full((3,), 5.0, device="cuda")
        mnmt.mnmt_dropout(sx.at, code, sx.ld, sr.at, sr.ld, 0.75, 0.25, 11, 3, True, M, d, out.at, rcode, out.ld)
        mnmt.mnmt_dropout_backward(sg.at, rcode, sg.ld, sx.at, code, sx.ld, sr.at, sr.ld, 0.75, 0.25, 11, 3, True, M, d, gx.at, gx.ld,
                                   gr.at, gr.ld, gg[1:], ws)
        assert float(gg[0].item()) == 5.0 and float(gg[2].item()) == 5.0
        got.append([out.rows.clone(), gx.rows.clone(), gr.rows.clone(), gg])
        assert torch.equal(sx.rows, x) and torch.equal(sr.rows, r) and torch.equal(sg.rows, g)
        assert all(b.rest() for b in (sx, sr, sg, out, gx, gr))
    for a, b in zip(*got):
        assert torch.equal(a, b)
