"""The single-token form against caches of hundreds of thousands of keys: results are not small for being long sums, and
no part of a cache is left out or counted twice."""
import pytest

torch = pytest.importorskip("torch")
from paper_2306_04235_gb300 import mnmt  # noqa: E402
from test_gpu_seq_attn import BF, FP, TYPES, dev  # noqa: E402

pytestmark = pytest.mark.gpu


def token(q, k, v, first, lens, dtype):
    B, d = q.shape[0], q.shape[2]
    s = mnmt.AttentionShape(B, B, k.shape[0], q.shape[1], k.shape[1], d, TYPES[dtype], False, d ** -0.5, None, dev(first), k_len=dev(lens))
    ws = torch.full((mnmt.mnmt_attention_token_workspace(s),), 0xFF, dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty((q.shape[1], B), device="cuda")
    mnmt.mnmt_attention_token(s, mnmt.heads(q), mnmt.heads(k), mnmt.heads(v), mnmt.heads(o), lse, ws)
    torch.cuda.synchronize()
    return o, lse


@pytest.mark.parametrize("dtype", [FP, BF])
@pytest.mark.parametrize("B", [2500, 2])  # a warp per sequence; runs
@pytest.mark.parametrize("n,d", [(1 << 18, 64), (1 << 18, 128), (1 << 20, 64), (200001, 40)])
def test_long_sums(n, d, B, dtype):
    """Values between 1 and 1.25: sums of one sign.  Every tile's sum is added with a rounding of 2^-24 of what is there, to
    either side: over 2^16 tiles 2^-24 2^8 / 3 < 2^-17 as a root of a mean square (the sum grows evenly), with room 2^-14.  A weight's rounding,
    to either side too, is averaged over n: below 2^-14 of o.  Scores, d products: 2^-20.  The result is off by its own half
    step, the mean of d of them by a twelfth's root of a step over the root of d, six times that as room."""
    g = torch.Generator(device="cuda").manual_seed(n + d)
    k = torch.randn((n, 1, d), generator=g, device="cuda").to(dtype)
    v = (1 + 0.25 * torch.rand((n, 1, d), generator=g, device="cuda")).to(dtype)
    q = torch.randn((1, 1, d), generator=g, device="cuda").to(dtype)
    o, lse = token(q.expand(B, 1, d).contiguous(), k, v, [0] * B, [n] * B, dtype)
    x = (k[:, 0].double() @ q[0, 0].double()) * d ** -0.5
    want = torch.softmax(x, 0) @ v[:, 0].double()
    u = torch.finfo(dtype).eps / 2
    for b in (0, B // 2, B - 1):
        far = (o[b, 0].double() - want) / want
        assert float(far.abs().max()) <= u + 2.0 ** -13
        assert abs(float(far.mean())) <= 6 * 2 * u / (12 * d) ** 0.5 + 2.0 ** -13
        assert abs(float(lse[0, b]) - float(torch.logsumexp(x, 0))) <= 2.0 ** -14
    assert torch.equal(o, o[:1].expand_as(o)) or B == 2


def test_every_part_counts_once():
    """More than 2^31 tiles of a shared cache, of equal weights: o is the mean of the values, exactly (sums of whole numbers in
    fp32, below 2^24 steps of what is added), and each element of a value marks another part of the cache."""
    B, rows = 2100, 1 << 25
    at = torch.arange(rows, device="cuda")
    v = torch.zeros((rows, 1, 8), dtype=FP, device="cuda")
    v[:, 0, 0] = (at < rows // 2).to(FP)
    v[:, 0, 1] = ((at >> 20) & 1).to(FP)
    v[:, 0, 2] = ((at >> 22) % 3 == 1).to(FP)
    v[:4096, 0, 3] = 1024.0  # the first and the last rows, some in between
    v[-4096:, 0, 4] = 1024.0
    v[11111111:11111111 + 4096, 0, 5] = 1024.0
    v[:, 0, 6] = 1.0
    v[:, 0, 7] = (at % 37 == 5).to(FP)
    mean = v[:, 0].double().sum(0) / rows
    k, q = torch.zeros_like(v), torch.ones((B, 1, 8), dtype=FP, device="cuda")
    o, lse = token(q, k, v, [0] * B, [rows] * B, FP)
    assert bool(((o[:, 0].double() - mean).abs() <= 2.0 ** -11 * mean).all())
    want = 25 * 0.6931471805599453
    assert float((lse.double() - want).abs().max()) <= 2.0 ** -18
    # parts of it: starts and lengths that are no multiples of anything
    first = [(b * 15485863) % rows for b in range(B)]
    lens = [min(rows - f, 1 + (b * 32452843) % rows) for b, f in zip(range(B), first)]
    o, lse = token(q, k, v, first, lens, FP)
    sums = torch.cat([torch.zeros((1, 8), dtype=torch.float64, device="cuda"), v[:, 0].double().cumsum(0)])
    f, n = dev(first).long(), dev(lens).long()
    mean = (sums[f + n] - sums[f]) / n[:, None]
    assert bool(((o[:, 0].double() - mean).abs() <= 2.0 ** -11 * mean + 2.0 ** -25).all())
    assert float((lse[0].double() - n.double().log()).abs().max()) <= 2.0 ** -18
