"""fp16 attention where one key's score stands far above many others': the others' weights, each below what fp16 holds beside
1, are part of the sum and have to be part of the result."""
import math

import pytest

torch = pytest.importorskip("torch")
from paper_2306_04235_gb300 import mnmt  # noqa: E402
from test_gpu_seq_attn import BF, FP, TYPES, dev  # noqa: E402

pytestmark = pytest.mark.gpu


def operands(n, d, at, bits, v_top, v_rest, dtype):
    """Keys whose scores are 0 but for one, `bits` powers of two above, at row `at`, and their values."""
    k, v = torch.zeros((n, 1, d), dtype=dtype, device="cuda"), torch.full((n, 1, d), v_rest, dtype=dtype, device="cuda")
    k[at, 0, 0] = bits * math.log(2.0)
    v[at] = v_top
    top = float(k[at, 0, 0].double()) / math.log(2.0)  # what the type made of it
    w = 2.0 ** -top
    return k, v, top, (v_top + (n - 1) * w * v_rest) / (1 + (n - 1) * w), (abs(v_top) + (n - 1) * w * abs(v_rest)) / (1 + (n - 1) * w), math.log(2.0) * top + math.log1p((n - 1) * w)


def hold(o, lse, n, want, mag, want_lse, dtype):
    """A weight is rounded by half a step of its type, relative, but in fp16 by 2^-25 (half its smallest step) at least, which is
    2^-32 of the largest or less, as weights are taken 2^7 larger or more.  Sums: n / 8 truncating steps of 2^-23 in the tensor core (8
    products each at least), n / 8 rounded ones of 2^-24 in a lane's share of the weights' sum (the token form's four lanes
    add pairs), which log-sum-exp has too.  Scores of up to 64 powers of two: 2^-24 64 ln 2 < 2^-18 of a weight.  The result's own
    rounding."""
    u, z = torch.finfo(dtype).eps / 2, 2.0 ** -25 if dtype == FP else 0.0
    small = n * 2.0 ** -32 if dtype == FP else 0.0
    bound = small + (u + (n / 8 + 2) * 2.0 ** -23 + 2.0 ** -18) * mag + (u + (n / 8 + 8) * 2.0 ** -24) * abs(want) + z
    off = (o.double() - want).abs().max()
    assert float(off) <= bound, (float(o.double().flatten()[0]), want, bound)
    assert float((lse.double() - want_lse).abs().max()) <= 2.0 ** -18 + (n / 8 + 8) * 2.0 ** -24 + 2.0 ** -22 * abs(want_lse)


VALUES = [(1.0, 1.0), (0.0, 1.0), (1.0, -1.0)]


@pytest.mark.parametrize("v_top,v_rest", VALUES)
@pytest.mark.parametrize("bits", [12.0, 25.2, 28.0])
@pytest.mark.parametrize("n,at", [(32768, 0), (32768, 32767), (32768, 20001), (300, 7)])
@pytest.mark.parametrize("d,hq", [(64, 80), (128, 80), (64, 1), (128, 2)])  # a CTA per head, and clusters
def test_forward(d, hq, n, at, bits, v_top, v_rest):
    for dtype in (FP, BF):
        k, v, top, want, mag, want_lse = operands(n, d, at, bits, v_top, v_rest, dtype)
        q = torch.zeros((128, hq, d), dtype=dtype, device="cuda")
        q[:, :, 0] = 1.0
        o, lse = torch.empty_like(q), torch.empty((hq, 128), device="cuda")
        s = mnmt.AttentionShape(1, 128, n, hq, 1, d, TYPES[dtype], False, 1.0, dev([0, 128]), dev([0, n]))
        ws = torch.empty(mnmt.mnmt_attention_forward_workspace(s), dtype=torch.uint8, device="cuda")
        H = mnmt.heads
        mnmt.mnmt_attention_forward(s, H(q), H(k), H(v), H(o), lse, ws)
        torch.cuda.synchronize()
        hold(o, lse, n, want, mag, want_lse, dtype)


@pytest.mark.parametrize("v_top,v_rest", VALUES)
@pytest.mark.parametrize("bits", [12.0, 25.2, 28.0])
@pytest.mark.parametrize("n,at", [(32768, 0), (32768, 32767), (32768, 20001), (300, 7)])
@pytest.mark.parametrize("d,B", [(64, 3000), (128, 3000), (64, 1), (128, 3)])  # a warp per sequence, and runs of keys
def test_token(d, B, n, at, bits, v_top, v_rest):
    dtype = FP
    k, v, top, want, mag, want_lse = operands(n, d, at, bits, v_top, v_rest, dtype)
    q = torch.zeros((B, 1, d), dtype=dtype, device="cuda")
    q[:, :, 0] = 1.0
    o, lse = torch.empty_like(q), torch.empty((1, B), device="cuda")
    s = mnmt.AttentionShape(B, B, n, 1, 1, d, TYPES[dtype], False, 1.0, None, dev([0] * B), k_len=dev([n] * B))
    ws = torch.empty(mnmt.mnmt_attention_token_workspace(s), dtype=torch.uint8, device="cuda")
    H = mnmt.heads
    mnmt.mnmt_attention_token(s, H(q), H(k), H(v), H(o), lse, ws)
    torch.cuda.synchronize()
    hold(o, lse, n, want, mag, want_lse, dtype)


@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_rise_by_less_than_the_slack(d):
    """Scores that grow towards the keys that are walked last, in steps that do and do not move the maximum: the largest weights
    stay within fp16, in both forms, and the result is the formula's (values 1: the mean of ones is 1)."""
    n = 1024
    for step in (0.05, 7.0, 8.0, 9.0, 15.0, 16.0):  # powers of two a tile of 64 keys
        k = torch.zeros((n, 1, d), dtype=FP, device="cuda")
        k[:, 0, 0] = ((n - 1 - torch.arange(n, device="cuda")) // 64 * step * math.log(2.0)).to(FP)
        v = torch.ones((n, 1, d), dtype=FP, device="cuda")
        q = torch.zeros((128, 1, d), dtype=FP, device="cuda")
        q[:, :, 0] = 1.0
        x = k[:, 0, 0].double()
        for token in (False, True):
            B = 128
            s = mnmt.AttentionShape(B, B, n, 1, 1, d, mnmt.F16, False, 1.0, None, dev([0] * B), k_len=dev([n] * B)) if token else \
                mnmt.AttentionShape(1, 128, n, 1, 1, d, mnmt.F16, False, 1.0, dev([0, 128]), dev([0, n]))
            o, lse = torch.empty_like(q), torch.empty((1, 128), device="cuda")
            size = mnmt.mnmt_attention_token_workspace(s) if token else mnmt.mnmt_attention_forward_workspace(s)
            H = mnmt.heads
            (mnmt.mnmt_attention_token if token else mnmt.mnmt_attention_forward)(s, H(q), H(k), H(v), H(o), lse, torch.empty(size, dtype=torch.uint8, device="cuda"))
            torch.cuda.synchronize()
            # each weight 2^-11 relative or 2^-32 of the largest; 64 truncating steps of 2^-23; the result's rounding
            assert float((o.double() - 1).abs().max()) <= 2.0 ** -11 + n * 2.0 ** -32 + 64 * 2.0 ** -23 + 2.0 ** -11
            assert float((lse.double() - float(torch.logsumexp(x, 0))).abs().max()) <= 2.0 ** -15 + 2.0 ** -21 * float(x.max())
