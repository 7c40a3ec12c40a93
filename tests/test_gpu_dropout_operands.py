"""Dropout's backward pass where some of its outputs are not asked for: their operands
are neither needed nor read."""
import pytest

from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": (mnmt.F32, torch.float32), "bf16": (mnmt.BF16, torch.bfloat16), "f16": (mnmt.F16, torch.float16)}


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M,d,pad", [(1, 7, 0), (33, 64, 0), (130, 1001, 3)])
def test_gain_and_residual_alone_need_no_x(ty, M, d, pad):
    """With ReLU and without gx: the same bits from x of any type, from no x, and beside gx."""
    xt, dt = TYPES[ty]
    gen = torch.Generator(device="cuda").manual_seed(d)
    ld = d + pad
    x = torch.randn((M, ld), generator=gen, device="cuda").to(dt)
    g, r = torch.randn((M, d), generator=gen, device="cuda"), torch.randn((M, d), generator=gen, device="cuda")
    ws = torch.empty(mnmt.DROPOUT_WORKSPACE, dtype=torch.uint8, device="cuda")

    def call(x, gx):
        gr, gg = torch.empty((M, d), device="cuda"), torch.empty(1, device="cuda")
        mnmt.mnmt_dropout_backward(g, mnmt.F32, d, x, xt, ld, r, d, 0.75, 0.3, 5, 6, True, M, d, gx, ld, gr, d, gg, ws)
        return gr, gg

    want = call(x, torch.empty_like(x))
    for got in (call(x, None), call(None, None)):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(want[0], g * 0.75)
