"""Products of 4-bit floating-point operands whose block scales lie at the ends of their
range: single factors leave fp32 where the sum of the products does not."""
import numpy as np
import pytest

import fp4_plain as P
from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

FMT = {"mx": mnmt.FP4_MX, "nv": mnmt.FP4_NV}


def packed(x, fmt, g):
    byte, code, v, _ = P.quantize(x, fmt, g)
    c, s = P.pack(byte, code, x.shape[1])
    c, s = torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()
    return mnmt.Fp4(x.shape[0], x.shape[1], FMT[fmt], g, c, s), v.astype(np.float64)


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 70, 96), (3, 70, 96), (8, 70, 512), (16, 70, 96), (300, 200, 512)])
@pytest.mark.parametrize("fmt,ex,ew", [("mx", 125, -123), ("mx", -123, 125), ("mx", 120, -120), ("mx", -120, 120), ("mx", 60, 60), ("mx", 0, 118),
                                       ("mx", -124, 0), ("nv", 100, -80), ("nv", -80, 100)])
def test_scales_at_the_ends(fmt, ex, ew, M, N, K, own):
    """Elements of up to 2^ex and 2^ew (NV: by way of the tensor scale), whole columns of blocks zero, so that a block's
    sum of zero meets the other operand's largest scale.  Tolerance as for any product: (K/16 + 16) 2^-23 of the sum
    of magnitudes, 2^-23 of the result; results below fp32's normal numbers in steps of 2^-149 per block."""
    rng = np.random.default_rng(K + M)

    def draw(rows, e):
        x = rng.uniform(-1, 1, (rows, K)).astype(np.float32)
        x[:, 32:64] = 0
        return np.ldexp(x, e).astype(np.float32)

    gx, gw = (float(2.0 ** (e - 11)) if fmt == "nv" else 1.0 for e in (ex, ew))
    x = draw(M, ex)
    (xq, xv), (wq, wv) = packed(x, fmt, gx), packed(draw(N, ew), fmt, gw)
    y = torch.empty((M, N), device="cuda")
    mnmt.mnmt_fp4_linear(xq, wq, torch.from_numpy(x).cuda() if own else None, mnmt.F32, K, None, False, y, mnmt.F32, N)
    want, mag = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    assert np.abs(want).max() < 2.0 ** 127 and np.abs(want).max() > 0
    got = y.cpu().numpy().astype(np.float64)
    assert (np.abs(got - want) <= (K / 16 + 16) * 2.0 ** -23 * mag + 2.0 ** -23 * np.abs(want) + K / 16 * 2.0 ** -149).all()
