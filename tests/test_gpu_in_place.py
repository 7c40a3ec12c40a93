"""In-place calls of quantisation and dropout: with the operand's own row stride they
give the bits of the call into another buffer, with another stride (rows written over
before they are read) they are refused; one row has no stride."""
import pytest

from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

D = 40
F = mnmt.F32


def matrix(seed, M, ld):
    return torch.randn((M, ld), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


# a call: its aliased output's operand, f(operand, its stride, the other operands' stride, output, its stride, M)
def quantize(t, ld, other, out, ldo, M):
    mnmt.mnmt_fp4_quantize(mnmt.Fp4(M, D, mnmt.FP4_MX), t, F, ld, out, ldo)


def quantize_backward_x(t, ld, other, out, ldo, M):
    mnmt.mnmt_fp4_quantize_backward(mnmt.Fp4(M, D, mnmt.FP4_MX), t, F, ld, other, D, out, ldo)


def quantize_backward_g(t, ld, other, out, ldo, M):
    mnmt.mnmt_fp4_quantize_backward(mnmt.Fp4(M, D, mnmt.FP4_MX), other, F, D, t, ld, out, ldo)


def dropout_r(t, ld, other, out, ldo, M):
    mnmt.mnmt_dropout(other, F, D, t, ld, 0.5, 0.3, 1, 2, False, M, D, out, F, ldo)


def dropout_backward_gx_x(t, ld, other, out, ldo, M):
    mnmt.mnmt_dropout_backward(other, F, D, t, F, ld, None, 0, 0.5, 0.3, 1, 2, True, M, D, out, ldo)


def dropout_backward_gr_g(t, ld, other, out, ldo, M):
    mnmt.mnmt_dropout_backward(t, F, ld, None, F, 0, None, 0, 0.5, 0.3, 1, 2, False, M, D, None, 0, out, ldo)


CALLS = [quantize, quantize_backward_x, quantize_backward_g, dropout_r, dropout_backward_gx_x, dropout_backward_gr_g]


@pytest.mark.parametrize("call", CALLS)
def test_same_stride(call):
    M, ld = 300, D + 5
    t, other, out = matrix(1, M, ld), matrix(2, M, D), torch.zeros((M, ld), device="cuda")
    call(t, ld, other, out, ld, M)
    before = t.clone()
    call(t, ld, other, t, ld, M)
    assert torch.equal(t[:, :D], out[:, :D]) and torch.equal(t[:, D:], before[:, D:]) and not torch.equal(t, before)


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("ld,ldo", [(D, D + 8), (D + 8, D)])
def test_other_stride(call, ld, ldo):
    M = 4
    t, other = matrix(1, M, D + 8), matrix(2, M, D)
    before = t.clone()
    with pytest.raises(mnmt.MnmtError) as ei:
        call(t, ld, other, t, ldo, M)
    assert ei.value.code == mnmt.EINVAL and "in place" in str(ei.value)
    torch.cuda.synchronize()
    assert torch.equal(t, before)
    # one row: no stride to differ; no rows: nothing to do
    out = torch.zeros((1, D + 8), device="cuda")
    call(t, ld, other, out, ldo, 1)
    call(t, ld, other, t, ldo, 1)
    assert torch.equal(t[0, :D], out[0, :D]) and torch.equal(t[1:], before[1:])
    call(t, ld, other, t, ldo, 0)
