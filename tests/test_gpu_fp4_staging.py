"""Gradients of the 4-bit floating-point linear where one product of a launch is stored
by TMA and the other, after it on the same CTAs, from registers through the same staging
blocks: odd widths beside a split product (its parts always go by TMA), widths that are
a multiple of 4 but not of 8 (fp32 rows end on 16 bytes, 16-bit ones do not), rows of one
output that start anywhere.

The reference is the same call with the width rounded up to a multiple of 8 and zero
columns at the end, all of whose stores go by TMA: the tiles, the parts and the order of
every sum are the same, so the columns that both have are the same bits."""
import pytest

from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TIMES = 100


def packed(x):
    rows, cols = x.shape
    q = mnmt.Fp4(rows, cols, mnmt.FP4_MX, 1.0, torch.empty((rows, mnmt.mnmt_fp4_pitch(cols)), dtype=torch.uint8, device="cuda"),
                 torch.empty(mnmt.mnmt_fp4_scale_bytes(rows, cols, mnmt.FP4_MX), dtype=torch.uint8, device="cuda"))
    mnmt.mnmt_fp4_quantize(q, x, mnmt.F32, cols)
    return q


# M, N, K, elements between rows beside K (gX, gW)
CASES = [(64, 32000, 2047, 0, 0), (512, 32000, 1021, 0, 0), (2048, 32000, 509, 0, 0), (8000, 512, 509, 0, 0), (16384, 8192, 2044, 0, 0),
         (700, 5003, 2056, 3, 3), (700, 5003, 2056, 0, 3)]


@pytest.mark.parametrize("masks", [False, True])
@pytest.mark.parametrize("M,N,K,padx,padw", CASES)
def test_products_stored_differently(M, N, K, padx, padw, masks):
    gen = torch.Generator(device="cuda").manual_seed(K)
    K8 = -(-K // 8) * 8
    G = torch.randn((M, N), generator=gen, device="cuda").to(torch.bfloat16)
    wide = []
    for rows in (M, N):
        x = torch.zeros((rows, K8), device="cuda")
        x[:, :K] = torch.randn((rows, K), generator=gen, device="cuda")
        wide.append(x)

    def call(k, gx, gw):
        x, w = (t[:, :k].contiguous() for t in wide)
        xq, wq = packed(x), packed(w)
        ws = torch.empty(mnmt.mnmt_fp4_linear_backward_workspace(M, N, k), dtype=torch.uint8, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        xo, wo = (x.to(torch.bfloat16), w) if masks else (None, None)

        def go():
            mnmt.mnmt_fp4_linear_backward(xq, wq, G, N, xo, mnmt.BF16, k, wo, mnmt.F32, k, ws, gx, gx.shape[1], gw, gw.shape[1], None, status)
            return status

        return go

    want = torch.empty((M, K8), dtype=torch.bfloat16, device="cuda"), torch.empty((N, K8), device="cuda")
    assert int(call(K8, *want)().item()) == 0
    got = torch.empty((M, K + padx), dtype=torch.bfloat16, device="cuda"), torch.empty((N, K + padw), device="cuda")
    go = call(K, *got)
    same = torch.ones(1, dtype=torch.bool, device="cuda")
    for _ in range(TIMES):
        for t in got:
            t.fill_(7.0)
        status = go()
        for a, b in zip(want, got):
            same &= (a[:, :K] == b[:, :K]).all()
    assert bool(same.item()) and int(status.item()) == 0
    assert float(want[0].float().abs().max()) > 1.0 and float(want[1].abs().max()) > 1.0
