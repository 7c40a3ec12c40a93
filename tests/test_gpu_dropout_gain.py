"""The gradient of dropout's residual gain over matrices so large that a lane visits
thousands of elements: its sum in fp32 does not grow with them."""
import pytest

from paper_2306_04235_gb300 import mnmt

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"bf16": (mnmt.BF16, torch.bfloat16), "f16": (mnmt.F16, torch.float16)}


@pytest.mark.parametrize("ty", list(TYPES))
@pytest.mark.parametrize("M,d", [(131072, 8192), (131071, 8191), (1 << 20, 1023)])
def test_gain_of_a_large_matrix(ty, M, d):
    """Every product is 1 + 2^-5 + 3 2^-14, exact in fp32, and so is any sum of up to 512 of them; a chain of thousands
    rounds each the same way.  A chain of at most 512 products in fp32, 64 bits above, one rounding: 2^-24 (512 + 2)."""
    t, dt = TYPES[ty]
    g = torch.full((M, d), 1 + 3 / 128, dtype=dt, device="cuda")
    r = torch.full((M, d), 1 + 1 / 128, dtype=dt, device="cuda")
    gg = torch.zeros(1, device="cuda")
    ws = torch.empty(mnmt.DROPOUT_WORKSPACE, dtype=torch.uint8, device="cuda")
    mnmt.mnmt_dropout_backward(g, t, d, None, t, d, r, d, 1.0, 0.1, 1, 2, False, M, d, ggamma=gg, workspace=ws)
    want = M * d * (1 + 3 / 128) * (1 + 1 / 128)
    assert abs(float(gg.item()) - want) <= 2.0 ** -24 * 514 * want
